"""A handle's first backward: captured or not, whatever the calls before it, the same kernels and the same bits; and captured backwards whose splits of a
state meet in memory, replayed."""
from __future__ import annotations

import pytest
import torch

import block_reference as ref

pytestmark = pytest.mark.gpu


def tensors(shape, dtype, seed):
    B, H, gh, gw, d, ks = shape
    gen = torch.Generator(device="cuda:0").manual_seed(seed)
    g, q, k, v = (torch.randn(B, H, gh * gw, d, generator=gen, device="cuda:0").to(dtype) for _ in range(4))
    return g, q, k, v, torch.randn(H * d, ks, ks, generator=gen, device="cuda:0").to(dtype)


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("shape,dtype", [((2, 3, 20, 20, 64, 3), F32), ((2, 3, 14, 14, 64, 3), F32), ((2, 3, 24, 33, 32, 5), F32), ((1, 2, 24, 20, 128, 3), F32), ((2, 2, 20, 20, 64, 7), F32),
                                         ((2, 3, 14, 14, 64, 3), BF16), ((1, 2, 40, 30, 64, 5), BF16), ((2, 2, 9, 9, 48, 3), BF16)], ids=str)
def test_captured_before_anything_else(shape, dtype):
    from paper_2211_10526_b200 import CastlingAttn
    gh, gw, ks = shape[2], shape[3], shape[5]
    a, other = tensors(shape, dtype, 1), tensors(shape, dtype, 2)
    with CastlingAttn(ksize=ks) as used, CastlingAttn(ksize=ks) as fresh:
        used.forward(*other[1:], None, gh, gw)
        want = used.backward(*other, gh, gw)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = fresh.backward(*a, gh, gw)
        assert fresh.last_path() == used.last_path()
        for x, y in zip(a, other):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        assert same(got, want)
        # calls that move the handle's workspace leave the graph as it is
        big = tensors((4, 4, 48, 48, shape[4], ks), dtype, 3)
        fresh.forward(*big[1:], None, 48, 48)
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert same(got, want) and fresh.device_status() == (0, 0)
        del graph


@pytest.mark.parametrize("shape", [(1, 1, 100, 120, 64, 3), (1, 1, 100, 120, 64, 5), (1, 1, 120, 120, 32, 3), (1, 1, 120, 121, 32, 5)], ids=str)
def test_splits_that_meet_in_memory(shape):
    from paper_2211_10526_b200 import CastlingAttn
    gh, gw, ks = shape[2], shape[3], shape[5]
    a, other = tensors(shape, BF16, 4), tensors(shape, BF16, 5)
    with CastlingAttn(ksize=ks) as attn:
        want = [attn.backward(*t, gh, gw) for t in (a, other)]
        x = [t.clone() for t in a]
        graphs, got = [], []
        for _ in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                got.append(attn.backward(*x, gh, gw))
                got.append(attn.backward(*x, gh, gw))
            graphs.append(graph)
        for turn in range(6):
            for t, y in zip(x, (a, other)[turn % 2]):
                t.copy_(y)
            for graph in graphs:
                graph.replay()
            eager = attn.backward(*x, gh, gw)
            torch.cuda.synchronize()
            assert same(eager, want[turn % 2]) and all(same(t, want[turn % 2]) for t in got)
        assert attn.device_status() == (0, 0)
        del graphs
    for name, t, w in zip(("dq", "dk", "dv"), want[0], ref_grads(a, gh, gw)):
        assert float((t.double() - w).norm()) <= 2 * ref.HALF_STEP[BF16] * float(w.norm()), name


def ref_grads(t, gh, gw):
    """Linear in the tokens: these are too many for explicit weights."""
    g, q, k, v, w = (x.double().requires_grad_(i in (1, 2, 3)) for i, x in enumerate(t))
    B, H, N, d = q.shape
    unit = [x / x.norm(dim=-1, keepdim=True) for x in (q, k)]
    out = 0.5 * v.sum(2, keepdim=True) + unit[0] @ (unit[1].transpose(-1, -2) @ v) / torch.pi
    grid = v.view(B, H, gh, gw, d).permute(0, 1, 4, 2, 3).reshape(B, H * d, gh, gw)
    conv = torch.nn.functional.conv2d(grid, w[:, None], padding=w.shape[-1] // 2, groups=H * d)
    out = out + conv.view(B, H, d, N).transpose(-1, -2)
    return torch.autograd.grad(out, (q, k, v), g)


def test_under_a_cap_without_room():
    from paper_2211_10526_b200 import CastlingAttn, binding as b
    for shape, dtype in (((2, 3, 14, 14, 64, 3), BF16), ((2, 3, 20, 20, 32, 3), BF16), ((2, 3, 20, 20, 64, 3), F32)):
        t = tensors(shape, dtype, 6)
        with CastlingAttn(max_workspace=64) as attn:
            got = attn.backward(*t, shape[2], shape[3])
            assert attn.last_path()[0] == b.PATH_SIMT
        for a, w in zip(got, ref.attention_grads(*t, shape[2], shape[3], 0)):
            assert float((a.double() - w).norm()) <= (ref.HALF_STEP[dtype] + 64 * 2.0 ** -24) * float(w.norm())
    t = tensors((2, 3, 14, 14, 64, 3), BF16, 6)
    with CastlingAttn(max_workspace=64, force_path=b.PATH_TENSOR) as attn:
        with pytest.raises(b.CastlingError) as error:
            attn.backward(*t, 14, 14)
        assert error.value.code == b.ERR_OOM


def test_first_calls_at_the_same_time():
    import threading
    from paper_2211_10526_b200 import CastlingAttn
    for shape, dtype in (((2, 3, 14, 14, 64, 3), BF16), ((1, 2, 30, 20, 64, 5), BF16), ((2, 3, 20, 20, 64, 3), F32)):
        t = tensors(shape, dtype, 7)
        with CastlingAttn(ksize=shape[5]) as attn:
            want = attn.backward(*t, shape[2], shape[3])
        torch.cuda.synchronize()
        for _ in range(5):
            with CastlingAttn(ksize=shape[5]) as attn:
                got, start = [None] * 6, threading.Barrier(6)

                def call(i):
                    with torch.cuda.stream(torch.cuda.Stream()):
                        start.wait()
                        got[i] = attn.backward(*t, shape[2], shape[3])
                        torch.cuda.current_stream().synchronize()

                threads = [threading.Thread(target=call, args=(i,)) for i in range(6)]
                for x in threads:
                    x.start()
                for x in threads:
                    x.join()
                torch.cuda.synchronize()
                assert all(g is not None and same(g, want) for g in got)
                assert attn.device_status() == (0, 0)
