"""Cross attention on the GPU: infinite values and gradients, which keep their
sign whatever fills up the tiles and parts beside them."""
import pytest
import torch

from paper_2607_02097_amd import binding as W

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def inputs(B, Sq, Sk, Hq, Hk, D, dtype, seed):
    """q, k, v, dout on the GPU, scores of order 1 (so no weight underflows)."""
    out = []
    for i, (S, H) in enumerate(((Sq, Hq), (Sk, Hk), (Sk, Hk), (Sq, Hq))):
        g = torch.Generator().manual_seed(seed + i)
        out.append(torch.randn((B, S, H, D), generator=g).to(DT[dtype]).cuda())
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [64, 37])
@pytest.mark.parametrize("Sq", [1, 9])
@pytest.mark.parametrize("Sk", [200, 400, 700, 784, 1001, 1600])
def test_infinite_values_of_states_in_parts(Sk, Sq, D, dtype):
    """One part, 4, 7, 8, 10 and 16 parts: an infinite component of the last
    state (and of one in the middle) comes out as itself, others as before."""
    q, k, v, _ = inputs(2, Sq, Sk, 2, 2, D, dtype, 200)
    clean, lse = W.wbmm_cross_attention_forward(q, k, v)
    v[:, -1, :, 5] = float("inf")
    v[:, Sk // 2, :, 9] = -float("inf")
    out, lse2 = W.wbmm_cross_attention_forward(q, k, v)
    keep = torch.ones(D, dtype=torch.bool, device="cuda")
    keep[5] = keep[9] = False
    assert bool((out[..., 5] == float("inf")).all()) and bool((out[..., 9] == -float("inf")).all())
    assert torch.equal(out[..., keep], clean[..., keep]) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,Sq,Sk,Hq,Hk,D", [
    (2, 5, 90, 4, 2, 64),      # few rows
    (2, 5, 90, 4, 2, 37),
    (1, 64, 90, 2, 2, 32),     # whole tiles
    (2, 50, 70, 2, 2, 128),    # 50 rows: tiles of 32 rows
    (2, 50, 70, 2, 2, 101),
    (25, 100, 70, 8, 8, 64),   # tiles of 64 and 128 rows
    (25, 100, 70, 8, 8, 96),
    (25, 100, 70, 8, 8, 40),
    (1, 400, 90, 1, 1, 64),    # rows in parts
    (1, 399, 90, 3, 1, 72),
])
@pytest.mark.parametrize("mask", [False, True])
def test_infinite_gradients_of_the_last_row(B, Sq, Sk, Hq, Hk, D, mask, dtype):
    """An infinite component of the last query's upstream gradient makes that
    component of the visible states' dv infinite, of its sign; all other
    components, and hidden states, are as before."""
    q, k, v, g = inputs(B, Sq, Sk, Hq, Hk, D, dtype, 210)
    see = torch.ones(B, Sk, dtype=torch.bool, device="cuda")
    if mask:
        see[:, 3::4] = False
    kw = {"key_mask": see} if mask else {}
    out, lse = W.wbmm_cross_attention_forward(q, k, v, **kw)
    clean = W.wbmm_cross_attention_backward(g, q, k, v, out, lse, **kw)[2]
    g[:, -1, Hq // Hk - 1::Hq // Hk, 3] = float("inf")   # the last row of each key head
    g[:, -1, Hq // Hk - 1::Hq // Hk, 6] = -float("inf")
    dv = W.wbmm_cross_attention_backward(g, q, k, v, out, lse, **kw)[2]
    keep = torch.ones(D, dtype=torch.bool, device="cuda")
    keep[3] = keep[6] = False
    assert torch.equal(dv[..., keep], clean[..., keep])
    assert bool((dv[see][..., 3] == float("inf")).all()) and bool((dv[see][..., 6] == -float("inf")).all())
    assert bool((dv[~see] == 0).all())
