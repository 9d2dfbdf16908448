"""Calls that are the first a thread makes of CUDA take the same kernels as any other, and give the same bits."""
from __future__ import annotations

import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape,dtype", [((2, 3, 14, 14, 64, 3), torch.bfloat16), ((1, 2, 30, 20, 64, 5), torch.bfloat16), ((2, 3, 20, 20, 32, 3), torch.bfloat16),
                                         ((1, 2, 40, 30, 64, 3), torch.bfloat16), ((2, 3, 20, 20, 64, 3), torch.float32), ((1, 2, 30, 33, 128, 3), torch.float32)], ids=str)
@pytest.mark.parametrize("what", ["forward", "backward"])
def test_first_call_of_a_thread(what, shape, dtype):
    from paper_2211_10526_b200 import CastlingAttn
    B, H, gh, gw, d, ks = shape
    gen = torch.Generator(device="cuda:0").manual_seed(1)
    g, q, k, v = (torch.randn(B, H, gh * gw, d, generator=gen, device="cuda:0").to(dtype) for _ in range(4))
    w = torch.randn(H * d, ks, ks, generator=gen, device="cuda:0").to(dtype)
    with CastlingAttn(ksize=ks) as attn:
        outs = [[torch.empty_like(q) for _ in range(3)] for _ in range(2)]       # memory that the calls find ready
        torch.cuda.synchronize()

        def call(i):
            if what == "forward":
                attn.forward(q, k, v, w, None, gh, gw, out=outs[i][0])
            else:
                attn.backward(g, q, k, v, w, gh, gw, out=tuple(outs[i]))
            path.append(attn.last_path())

        path = []
        call(0)
        torch.cuda.synchronize()
        thread = threading.Thread(target=call, args=(1,))
        thread.start()
        thread.join()
        torch.cuda.synchronize()
        assert len(path) == 2 and path[0] == path[1]
        assert all(torch.equal(a, b) for a, b in zip(outs[0][:1 if what == "forward" else 3], outs[1]))
        assert attn.device_status() == (0, 0)
