"""Strides that no tensor map takes (2^40 bytes and more), of a dimension that has one element: nothing lies there.  A handle that picks its kernels
takes those of the CUDA cores, one that is pinned to the tensor cores says that it cannot."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ksize", [3, 5])
@pytest.mark.parametrize("grid", [(14, 14), (30, 20)], ids=str)
@pytest.mark.parametrize("which", range(7))
def test_one_head_far_from_the_next(which, grid, ksize):
    from paper_2211_10526_b200 import CastlingAttn, binding as b
    gh, gw, d = *grid, 64
    N = gh * gw
    gen = torch.Generator(device="cuda:0").manual_seed(which)
    q, k, v, g = (torch.randn(1, 1, N, d, generator=gen, device="cuda:0").bfloat16() for _ in range(4))
    w = torch.randn(d, ksize, ksize, generator=gen, device="cuda:0").bfloat16()
    strides = [b.castling_attn_strides_t(N * d, N * d, d) for _ in range(7)]
    strides[which] = b.castling_attn_strides_t(1 << 39, 1 << 39, d)
    layout = b.castling_attn_grad_layout_t(*strides)

    def call(attn, layout):
        out = [torch.zeros_like(t) for t in (q, k, v, w)] + [torch.zeros(d, dtype=q.dtype, device="cuda:0")]
        n = b.castling_attn_backward_workspace_bytes(attn.handle, 1, 1, gh, gw, d, b.CASTLING_BF16)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda:0")
        rc = b.castling_attn_backward(attn.handle, *(t.data_ptr() for t in (q, k, v, w, g)), *(t.data_ptr() for t in out), 1, 1, gh, gw, d, b.CASTLING_BF16, layout,
                                      ws.data_ptr(), n)
        torch.cuda.synchronize()
        return rc, out, attn.last_path()[0]

    with CastlingAttn(ksize=ksize, force_path=b.PATH_SIMT) as simt, CastlingAttn(ksize=ksize) as auto, CastlingAttn(ksize=ksize, force_path=b.PATH_TENSOR) as pinned:
        want = call(simt, None)
        assert want[0] == b.OK and call(auto, None)[2] == b.PATH_TENSOR and call(pinned, None)[0] == b.OK
        if N <= 256 and ksize == 3 and which == 6:      # the kernel for short planes writes dv without a map
            assert call(pinned, layout)[0] == b.OK
            return
        rc, got, path = call(auto, layout)
        assert rc == b.OK and path == b.PATH_SIMT
        assert all(torch.equal(x, y) for x, y in zip(got, want[1]))
        assert call(pinned, layout)[0] == b.ERR_UNSUPPORTED
        assert call(pinned, None)[0] == b.OK
