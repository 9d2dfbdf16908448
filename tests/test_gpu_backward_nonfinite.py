"""Infinities and NaN in the inputs of the attention core's backward: the filters' gradients take them where the definition does, and planes and channels
without one are as if there were none."""
from __future__ import annotations

import pytest
import torch

import block_reference as ref

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")

# every kernel that sums for the filters: the one for short planes (a grid that fits with its halo, one that does not, width 32), that for values, the general one
SHAPES = [((3, 2, 14, 14, 64, 3), torch.bfloat16, 1), ((3, 2, 1, 100, 64, 3), torch.bfloat16, 0), ((3, 2, 15, 13, 32, 3), torch.bfloat16, 0), ((2, 2, 20, 39, 64, 3), torch.bfloat16, 1),
          ((2, 2, 20, 21, 64, 5), torch.bfloat16, 0), ((2, 2, 37, 21, 32, 3), torch.bfloat16, 1), ((2, 2, 41, 23, 64, 3), torch.float32, 0), ((2, 2, 9, 10, 128, 7), torch.bfloat16, 2),
          ((2, 2, 5, 6, 48, 1), torch.float32, 0), ((2, 2, 33, 6, 16, 5), torch.float32, 1)]


def tensors(shape, dtype, prefix):
    B, H, gh, gw, d, ks = shape
    gen = torch.Generator(device="cuda:0").manual_seed(sum(shape))
    g, q, k, v = (torch.randn(B, H, prefix + gh * gw, d, generator=gen, device="cuda:0").to(dtype) for _ in range(4))
    w = (0.2 * torch.randn(H * d, ks, ks, generator=gen, device="cuda:0")).to(dtype)
    v = torch.where(v == 0, torch.ones_like(v), v)
    return g, q, k, v, w


def filter_grads(g, v, gh, gw, ks, prefix):
    """By the definition: the terms whose token of v lies in the grid, and no others."""
    B, H, _, d = g.shape
    g, v = (t[:, :, prefix:].double().reshape(B, H, gh, gw, d) for t in (g, v))
    dw = torch.zeros(H, d, ks, ks, dtype=torch.float64, device=g.device)
    for y in range(ks):
        for x in range(ks):
            dy, dx = y - ks // 2, x - ks // 2
            y0, y1, x0, x1 = max(0, -dy), min(gh, gh - dy), max(0, -dx), min(gw, gw - dx)
            if y0 < y1 and x0 < x1:
                dw[:, :, y, x] = (g[:, :, y0:y1, x0:x1] * v[:, :, y0 + dy:y1 + dy, x0 + dx:x1 + dx]).sum((0, 2, 3))
    return dw.view(H * d, ks, ks)


def same(got, want, dtype):
    """Infinities and NaN where the definition has them; the rest to the rounding of a sum in fp32 and of the result."""
    got = got.double()
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got.isinf(), want.isinf()) and torch.equal(got[got.isinf()], want[want.isinf()])
    keep = want.isfinite()
    off, top = (got - want)[keep], want[keep]
    assert float(off.norm()) <= (ref.HALF_STEP[dtype] + 64 * 2.0 ** -24) * float(top.norm())


@pytest.mark.parametrize("value", [INF, -INF, NAN])
@pytest.mark.parametrize("which", ["g", "v"])
@pytest.mark.parametrize("shape,dtype,prefix", SHAPES, ids=str)
def test_filters(shape, dtype, prefix, which, value):
    from paper_2211_10526_b200 import CastlingAttn
    B, H, gh, gw, d, ks = shape
    g, q, k, v, w = tensors(shape, dtype, prefix)
    t = {"g": g, "v": v}[which]
    # in channels of their own, images in turn: corners, edges, the middle
    for i, (y, x) in enumerate([(0, 0), (gh - 1, gw - 1), (0, gw - 1), (gh // 2, gw // 2), (gh - 1, gw // 2), (gh // 2, 0), (gh // 2, gw - 1)]):
        t[i % B, i % H, prefix + y * gw + x, 2 * i + 1] = value
    with CastlingAttn(ksize=ks, prefix_tokens=prefix) as attn:
        got = attn.backward(g, q, k, v, w, gh, gw)
        torch.cuda.synchronize()
        assert attn.device_status() == (0, 0)
    same(got[3], filter_grads(g, v, gh, gw, ks, prefix), dtype)
    same(got[4], g[:, :, prefix:].double().sum((0, 2)).reshape(-1), dtype)


@pytest.mark.parametrize("shape,dtype,prefix", SHAPES, ids=str)
def test_other_planes(shape, dtype, prefix):
    """One plane's q, k, v and gradient full of them: the other planes' gradients have the same bits as without."""
    from paper_2211_10526_b200 import CastlingAttn
    B, H, gh, gw, d, ks = shape
    g, q, k, v, w = tensors(shape, dtype, prefix)
    with CastlingAttn(ksize=ks, prefix_tokens=prefix) as attn:
        want = attn.backward(g, q, k, v, w, gh, gw)
        for i, t in enumerate((g, q, k, v)):
            t[0, 0, i::3] = (INF, NAN, -INF, NAN)[i]
        got = attn.backward(g, q, k, v, w, gh, gw)
        torch.cuda.synchronize()
        assert attn.device_status() == (0, 0)
    for a, b in zip(got[:3], want[:3]):
        assert torch.equal(a[0, 1:], b[0, 1:]) and torch.equal(a[1:], b[1:])
    for a, b in zip(got[3:], want[3:]):
        assert torch.equal(a[d:], b[d:])       # the other heads' filters


def test_everything_is_nan():
    from paper_2211_10526_b200 import CastlingAttn
    for shape, dtype in (((8, 4, 14, 14, 64, 3), torch.bfloat16), ((1, 2, 64, 64, 64, 3), torch.bfloat16), ((1, 2, 64, 64, 64, 3), torch.float32)):
        g, q, k, v, w = tensors(shape, dtype, 0)
        with CastlingAttn() as attn:
            got = attn.backward(torch.full_like(g, NAN), q, k, v, w, shape[2], shape[3])
            torch.cuda.synchronize()
            assert all(bool(t.isnan().all()) for t in got)
            assert attn.device_status() == (0, 0)
