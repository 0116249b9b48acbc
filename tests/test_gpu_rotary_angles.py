"""Rotary positions on the GPU: cosine and sine as such, from a token (0, 1),
whose rotation gives -sin and cos without a further rounding.

The angle in 64 bits, position x frequency and its reduction to a fraction of a
turn, is off by at most 4 x 2^-53 of the angle.  Cosine and sine are off by at
most 2 float32 steps from the library, and half a step each from rounding the
remainder's product: 3 steps, 3 x 2^-23 of themselves.
"""
import pytest
import torch

from paper_2607_02097_amd import binding as W

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("P", [1, 24, 64])
@pytest.mark.parametrize("top", [50, 5000, 200000, 2 ** 28])
def test_cosine_and_sine_keep_their_own_precision(top, P, adjacent):
    """Near a multiple of a half turn too, where a sine is small."""
    B, S = 2, 600
    gen = torch.Generator().manual_seed(P + top)
    pos = torch.randint(-top, top, (1, B, S), generator=gen)
    freqs = W.wbmm_rotary_frequencies((P,), device="cpu")
    x = torch.zeros(B, S, 1, 2 * P)
    lo, hi = (slice(0, None, 2), slice(1, None, 2)) if adjacent else (slice(0, P), slice(P, None))
    x[..., hi] = 1.0
    y = W.wbmm_rotary_forward(x.cuda(), pos.cuda(), freqs.cuda(), (P,), adjacent).cpu().double()[:, :, 0]
    angle = pos[0].double()[:, :, None] * freqs.double()
    slack = 4 * 2.0 ** -53 * angle.abs()
    for got, want in ((y[..., lo], -angle.sin()), (y[..., hi], angle.cos())):
        assert bool(((got - want).abs() <= 3 * 2.0 ** -23 * want.abs() + slack).all())
