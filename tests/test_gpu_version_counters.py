"""Tensors that a call writes in place count as changed: autograd refuses to use what it had kept of them."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu


def gauss(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator(device="cuda:0").manual_seed(seed), device="cuda:0")


def test_rows_turned_in_place():
    from paper_2211_10526_b200 import GridRope
    rope = GridRope((16, 16))
    x, y = gauss(2, 3, 20, 32).requires_grad_(), gauss(2, 3, 20, 32, seed=1).requires_grad_()
    q, k = x.exp(), y.exp()           # exp keeps its result for the gradient
    before = q._version, k._version
    out = rope.forward(q.detach(), k.detach(), grid=(4, 5), inplace=True)
    assert out[0]._version > before[0] and out[1]._version > before[1]
    for t in (q, k):
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            t.sum().backward()
    fused = gauss(2, 20, 3, 3, 32)
    before = fused._version
    rope.backward(fused[:, :, 0].permute(0, 2, 1, 3), grid=(4, 5), inplace=True)
    assert fused._version > before
    plain = gauss(2, 3, 20, 32)
    rope.forward(plain, grid=(4, 5))
    assert plain._version == 0


def test_given_outputs():
    from paper_2211_10526_b200 import CastlingAttn
    q, k, v, g = (gauss(2, 3, 64, 32, seed=i) for i in range(4))
    w = gauss(96, 3, 3)
    x = [gauss(2, 3, 64, 32, seed=5 + i).requires_grad_() for i in range(4)]
    out = [t.exp() for t in x]
    with CastlingAttn() as attn:
        attn.backward(g, q, k, v, w, 8, 8, out=tuple(t.detach() for t in out[:3]))
        attn.forward(q, k, v, w, None, 8, 8, out=out[3].detach())
        for t in out:
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                t.sum().backward()
        assert all(t._version == 0 for t in (q, k, v, g, w))


def test_tensors_without_a_counter():
    from paper_2211_10526_b200 import GridRope
    with torch.inference_mode():
        q = gauss(1, 2, 6, 16)
        want = GridRope((16,)).forward(q, grid=(6,))[0]
    got = GridRope((16,)).forward(q, grid=(6,), inplace=True)[0]
    assert torch.equal(got, want)
