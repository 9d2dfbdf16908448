"""Outputs of one call whose strides differ: refused where what they reach overlaps, whatever elements they have."""
from __future__ import annotations

import ctypes
import random

import pytest
import torch

import test_layouts as t
from paper_2211_10526_b200 import binding as b

lib = t.lib     # the fixture


@pytest.mark.parametrize("seed", range(6))
def test_no_shared_element_is_missed(lib, seed):
    rng = random.Random(100 + seed)
    found = {True: 0, False: 0}
    for _ in range(400):
        width = rng.choice([1, 2, 3, 4])
        (axes, reach), (other, more) = t.some(rng, width), t.some(rng, width)
        a, c = (0, axes, width), (rng.randint(-more - 2, reach + 2), other, width)
        want = bool(set(t.elements(a)) & set(t.elements(c)))
        says = [bool(lib.shared(t.packed(x), t.packed(y), ctypes.c_longlong(4))) for x, y in ((a, c), (c, a))]
        assert says[0] == says[1] and (says[0] or not want), (a, c)
        found[says[0]] += 1
    assert min(found.values()) > 20


HEADS, TOKENS = (4 * 6 * 64, 6 * 64, 64), (4 * 6 * 64, 64, 4 * 64)     # [2, 4, 6, 64], head-major and token-major


def test_rotary_outputs_of_other_strides():
    X, K, Y = 0x10000000, 0x20000000, 0x40000000
    size = 4 * 2 * 4 * 6 * 64
    assert t.rotate(X, X, X, X, HEADS, TOKENS) == b.ERR_INVALID_ARG                    # in place, one tensor in two layouts
    assert t.rotate(X, K, Y, Y, HEADS, TOKENS) == b.ERR_INVALID_ARG
    assert t.rotate(X, K, Y, Y + size - 16, HEADS, TOKENS) == b.ERR_INVALID_ARG
    assert t.rotate(X, K, Y, Y + size, HEADS, TOKENS) != b.ERR_INVALID_ARG             # beside one another: no fault of the arguments


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_gradients_of_other_strides(dtype):
    from paper_2211_10526_b200 import CastlingAttn, GridRope
    gen = torch.Generator(device="cuda:0").manual_seed(1)
    g, q, k, v = (torch.randn(2, 3, 64, 32, generator=gen, device="cuda:0").to(dtype) for _ in range(4))
    w = torch.randn(96, 3, 3, generator=gen, device="cuda:0").to(dtype)
    one, two = (torch.full((2, 3, 64, 32), 7.0, device="cuda:0", dtype=dtype) for _ in range(2))
    turned = one.view(2, 64, 3, 32).permute(0, 2, 1, 3)        # the same elements, token-major
    with CastlingAttn(ksize=3) as attn:
        for out in ((one, turned, two), (turned, two, one), (two, one, turned)):
            with pytest.raises(b.CastlingError):
                attn.backward(g, q, k, v, w, 8, 8, out=out)
        torch.cuda.synchronize()
        assert bool((one == 7.0).all()) and bool((two == 7.0).all())
        want = attn.backward(g, q, k, v, w, 8, 8)
        both = torch.empty((2, 2, 3, 64, 32), device="cuda:0", dtype=dtype)
        got = attn.backward(g, q, k, v, w, 8, 8, out=(both[0], both[1].view(2, 64, 3, 32).permute(0, 2, 1, 3), two))
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    with pytest.raises(b.CastlingError):
        GridRope((32,)).forward(one, turned, grid=(64,), inplace=True)
    torch.cuda.synchronize()
    assert bool((one == 7.0).all())
