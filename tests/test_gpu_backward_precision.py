"""Gradients of the attention core where terms cancel: rows of q and k with a common direction, whose gradients have most of their length taken off along
the row, and gradients of the output whose token sum is nearly nought, which leaves the linear term of dv alone."""
from __future__ import annotations

import pytest
import torch

import block_reference as ref

pytestmark = pytest.mark.gpu

# one kernel for all gradients: planes of one tile and of two, with a token grid that fits a buffer with its halo and without
SHORT = [((2, 3, 14, 14, 64, 3), 1), ((2, 3, 14, 14, 64, 3), 0), ((3, 2, 9, 12, 64, 3), 2), ((2, 2, 1, 200, 64, 3), 0), ((2, 2, 16, 16, 64, 3), 0), ((2, 4, 14, 14, 32, 3), 1),
         ((2, 2, 20, 24, 32, 3), 0), ((160, 2, 7, 7, 64, 3), 0), ((2, 2, 1, 100, 64, 3), 3), ((1, 2, 1, 500, 32, 3), 0)]
# a kernel for the values and one for the rows; other filters
LONG = [((2, 3, 20, 20, 64, 3), 0), ((2, 3, 17, 37, 64, 3), 1), ((1, 2, 80, 70, 64, 3), 0), ((60, 3, 17, 16, 64, 3), 0), ((2, 2, 1, 400, 64, 3), 2), ((1, 3, 30, 33, 32, 3), 1),
        ((2, 3, 14, 14, 64, 5), 1), ((2, 3, 30, 33, 64, 5), 0), ((40, 4, 17, 17, 64, 5), 2), ((2, 3, 30, 33, 32, 5), 1), ((2, 3, 12, 15, 64, 7), 1), ((2, 3, 12, 15, 64, 1), 0)]


def tensors(shape, prefix, cosine, centred, seed):
    B, H, gh, gw, d, ks = shape
    N = prefix + gh * gw
    gen = torch.Generator(device="cuda:0").manual_seed(seed)

    def gauss(*s):
        return torch.randn(*s, generator=gen, device="cuda:0")

    way = gauss(1, H, 1, d)
    way = way / way.norm(dim=-1, keepdim=True) * d ** 0.5
    q, k = ((cosine * way + (1 - cosine ** 2) ** 0.5 * gauss(B, H, N, d)) * torch.exp(0.5 * gauss(B, H, N, 1)) for _ in range(2))
    v, g = gauss(B, H, N, d), gauss(B, H, N, d)
    if centred:
        g = g - g.mean(2, keepdim=True)
    w = (0.02 if centred else 0.2) * gauss(H * d, ks, ks)      # small filters: else the convolution hides the linear term of dv
    return [t.bfloat16() for t in (g, q, k, v, w)]


def check(shape, prefix, cosine, centred):
    """Each gradient is rounded once, which alone is off by `floor` in the 2-norm (the same values' own rounding; other values as close have other roundings of
    the same size: of a few thousand, to 5 %).  What is left over comes from operands kept as two bf16, 2^-17 of their size, and cancellation leaves
    1/8 of the terms or more at the cosines taken here: 2^-14 of the result."""
    from paper_2211_10526_b200 import CastlingAttn
    B, H, gh, gw, d, ks = shape
    g, q, k, v, w = tensors(shape, prefix, cosine, centred, seed=sum(shape) + prefix)
    with CastlingAttn(ksize=ks, prefix_tokens=prefix) as attn:
        got = attn.backward(g, q, k, v, w, gh, gw)
        torch.cuda.synchronize()
        assert attn.device_status() == (0, 0) and attn.last_path()[0] == 2
    off = []
    for name, a, want in zip(("dq", "dk", "dv"), got, ref.attention_grads(g, q, k, v, w, gh, gw, prefix)):
        floor, size = float((want.bfloat16().double() - want).norm()), float(want.norm())
        off.append((name, float((a.double() - want).norm()) / size, floor / size))
    assert all(error <= 1.05 * floor + 2.0 ** -14 for _, error, floor in off), off


@pytest.mark.parametrize("cosine", [0.0, 0.9, 0.97])
@pytest.mark.parametrize("shape,prefix", SHORT + LONG, ids=str)
def test_rows_with_a_common_direction(shape, prefix, cosine):
    check(shape, prefix, cosine, False)


@pytest.mark.parametrize("cosine", [0.0, 0.9])
@pytest.mark.parametrize("shape,prefix", SHORT + LONG, ids=str)
def test_centred_gradients_of_the_output(shape, prefix, cosine):
    check(shape, prefix, cosine, True)
