"""Rotary positions and cross attention on the GPU against plain 64-bit
implementations on the CPU.

Tolerances are bounds, element by element, from the arithmetic that the
operators document (u = half a step of the type, 2^-24 for float32):

  rotary     y = lo cos - hi sin in float32 from cos and sin that are off by at
             most 2 float32 steps, rounded once: u |y| + 2^-21 (|lo| + |hi|)
  scores     D products and sums in float32: d = scale (D + 4) 2^-24 |q|.|k|;
             with a softmax in float32 each weight is off by at most
             r = 2 d + 2^-20 of itself (both the score's error and that of the
             row's sum; exp2 and its argument's rounding: |s| 2^-22)
  out        weights rounded to the type (u), sums of n terms (n 2^-24):
             (u + r + n 2^-24) sum p |v| + u |out|
  gradients  the same steps for each product, written out in attention_bounds
Weights in 16 bits keep at least 2^-25 of absolute precision next to a largest
weight of 1 (float16's smallest step; bfloat16's is far below), which adds
2^-25 per term.  In every type a weight below 2^-126, float32's smallest normal
number, may come out as zero, which adds 2^-126 to a weight's bound and
2^-126 |dp - delta| to that of ds.
"""
import math

import pytest
import torch

from paper_2607_02097_amd import binding as W

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}  # smallest steps


def draw(shape, dtype, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(DT[dtype])


def check(got, want, bound, dtype, what):
    """|got - want| within the bound everywhere (and no NaN)."""
    got = got.detach().cpu().double()
    err = (got - want).abs()
    limit = bound + TINY[dtype]
    assert got.shape == want.shape, what
    worst = (err / limit).max().item() if err.numel() else 0.0
    bad = ~(err <= limit)
    assert not bad.any(), "%s: %d of %d off, worst %.3g of the bound" % (what, int(bad.sum()), bad.numel(), worst)


# ------------------------------------------------------------------- rotary

def rotary_plain(x, pos, freqs, sections, adjacent, sign=1.0):
    """64-bit rotation and its bound's magnitude."""
    P = sum(sections)
    y, mag = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64)
    i = 0
    for a, n in enumerate(sections):
        for _ in range(n):
            lo, hi = (2 * i, 2 * i + 1) if adjacent else (i, i + P)
            t = sign * pos[a].double() * freqs[i].double()
            c, s = t.cos()[:, :, None], t.sin()[:, :, None]
            xl, xh = x[..., lo].double(), x[..., hi].double()
            y[..., lo], y[..., hi] = xl * c - xh * s, xl * s + xh * c
            mag[..., lo] = mag[..., hi] = xl.abs() + xh.abs()
            i += 1
    return y, mag


def positions(A, B, S, seed, lo=-50, hi=5000, dtype=torch.int64):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(lo, hi, (A, B, S), generator=g).to(dtype)


ROTARY = [
    # B, S, H, D, sections, adjacent
    (1, 1, 1, 2, (1,), False),
    (1, 1, 1, 8, (4,), True),
    (2, 5, 3, 64, (16, 16), False),
    (2, 7, 40, 128, (16, 24, 24), False),
    (1, 33, 6, 80, (20, 20), True),
    (3, 9, 7, 72, (11, 13), False),      # odd pair counts, a tail that stays
    (3, 9, 7, 72, (11, 13), True),
    (2, 4, 5, 96, (8, 16), False),       # whole pieces, a tail that stays
    (2, 4, 5, 96, (8, 16), True),
    (1, 17, 1, 128, (64,), False),
    (2, 3, 2, 512, (100, 0, 56, 100), False),
    (1, 2, 3, 4096, (3,), False),
    (1, 2, 900, 1030, (130,), True),     # heads in several runs
    (4, 1500, 1, 16, (3, 5), False),     # many tokens, little in each
]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,S,H,D,sections,adjacent", ROTARY)
def test_rotary(B, S, H, D, sections, adjacent, dtype):
    x = draw((B, S, H, D), dtype, 1)
    pos = positions(len(sections), B, S, 2)
    freqs = W.wbmm_rotary_frequencies(sections, restart=len(sections) == 2, device="cpu")
    for fn, sign in ((W.wbmm_rotary_forward, 1.0), (W.wbmm_rotary_backward, -1.0)):
        want, mag = rotary_plain(x, pos, freqs, sections, adjacent, sign)
        got = fn(x.cuda(), pos.cuda(), freqs.cuda(), sections, adjacent)
        check(got, want, U[dtype] * want.abs() + 2.0 ** -21 * mag, dtype, fn.__name__)
        P = sum(sections)
        assert torch.equal(got[..., 2 * P:].cpu(), x[..., 2 * P:])


@pytest.mark.parametrize("H,D,S", [(1, 2, (1 << 20) + 3), (2, 2, (1 << 19) + 1), (1, 4, (1 << 19) + 700)])
def test_rotary_many_narrow_tokens(H, D, S):
    """More tokens in a workgroup than it has threads."""
    x, pos, freqs = draw((1, S, H, D), "bf16", 12), positions(1, 1, S, 13), W.wbmm_rotary_frequencies((1,), device="cpu")
    want, mag = rotary_plain(x, pos, freqs, (1,), False)
    got = W.wbmm_rotary_forward(x.cuda(), pos.cuda(), freqs.cuda(), (1,))
    check(got, want, U["bf16"] * want.abs() + 2.0 ** -21 * mag, "bf16", "narrow")


@pytest.mark.parametrize("offset", [0, 1, 2])
def test_rotary_layouts(offset):
    """A slice of a joint projection (offset: unaligned by so many elements),
    [B,H,S,D] order, 32-bit and broadcast positions, and in place."""
    B, S, H, D, sections = 2, 11, 4, 32, (5, 11)
    flat = draw((B * S * (2 * H + 1) * D + 8,), "bf16", 3).cuda()
    joint = flat[offset:offset + B * S * (2 * H + 1) * D].view(B, S, 2 * H + 1, D)
    x = joint[:, :, 1:H + 1]
    pos = positions(2, 1, S, 4, dtype=torch.int32).expand(2, B, S)
    freqs = W.wbmm_rotary_frequencies(sections)
    want, mag = rotary_plain(x.cpu(), pos, freqs.cpu(), sections, False)
    bound = U["bf16"] * want.abs() + 2.0 ** -21 * mag
    before = joint.clone()
    got = W.wbmm_rotary_forward(x, pos.cuda(), freqs, sections)
    check(got, want, bound, "bf16", "slice")
    assert torch.equal(joint, before)
    turned = x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    check(W.wbmm_rotary_forward(turned, pos.cuda(), freqs, sections), want, bound, "bf16", "[B,H,S,D]")
    # into another slice of the same tensor; nothing beside it changes
    W.wbmm_rotary_forward(x, pos.cuda(), freqs, sections, out=joint[:, :, H + 1:])
    assert torch.equal(joint[:, :, H + 1:], got) and torch.equal(joint[:, :, :H + 1], before[:, :, :H + 1])
    W.wbmm_rotary_forward(x, pos.cuda(), freqs, sections, out=x)
    assert torch.equal(joint[:, :, 1:H + 1], got) and torch.equal(joint[:, :, :1], before[:, :, :1])


def test_rotary_far_positions():
    """Angles of positions up to 2^28 keep float32's precision."""
    x = draw((1, 64, 2, 64), "f32", 5)
    pos = positions(1, 1, 64, 6, lo=-2 ** 28, hi=2 ** 28)
    freqs = W.wbmm_rotary_frequencies((32,), device="cpu")
    want, mag = rotary_plain(x, pos, freqs, (32,), False)
    check(W.wbmm_rotary_forward(x.cuda(), pos.cuda(), freqs.cuda(), (32,)), want,
          2.0 ** -24 * want.abs() + 2.0 ** -21 * mag, "f32", "far")


def test_rotary_keeps_inner_products():
    """Scores depend on the distance of the positions only."""
    freqs = W.wbmm_rotary_frequencies((8, 24))
    q, k = draw((1, 1, 1, 64), "f32", 7).cuda(), draw((1, 1, 1, 64), "f32", 8).cuda()

    def score(a, b):
        at = lambda p: torch.tensor(p, device="cuda").view(2, 1, 1)
        qr = W.wbmm_rotary_forward(q, at(a), freqs, (8, 24)).double()
        return (qr * W.wbmm_rotary_forward(k, at(b), freqs, (8, 24)).double()).sum().item()

    # 64 products of components of at most about 3, each off by 2^-21 of both
    tol = 64 * 2 * 2.0 ** -21 * q.abs().max().item() * k.abs().max().item() * 2
    assert abs(score([3, 4], [10, 20]) - score([103, 1004], [110, 1020])) <= tol


def test_rotary_autograd_and_empty():
    x = draw((2, 5, 3, 24), "f32", 9).cuda().requires_grad_(True)
    pos, freqs = positions(2, 2, 5, 10).cuda(), W.wbmm_rotary_frequencies((4, 6))
    y = W.wbmm_rotary(x, pos, freqs, (4, 6), True)
    g = draw(y.shape, "f32", 11).cuda()
    (dx,) = torch.autograd.grad(y, x, g)
    # <g, R x> = <R^T g, x>, each side a float32 rotation of 720 elements
    a, b = (g.double() * y.double()).sum().item(), (dx.double() * x.double()).sum().item()
    assert abs(a - b) <= 2.0 ** -20 * (g.abs().sum() * x.abs().max()).item()
    # a gradient that is a broadcast of one number
    y = W.wbmm_rotary(x, pos, freqs, (4, 6), True)
    (dx,) = torch.autograd.grad(y.sum(), x)
    assert torch.equal(dx, W.wbmm_rotary_backward(torch.ones_like(x), pos, freqs, (4, 6), True))
    for B, S in ((0, 5), (2, 0)):
        e = torch.empty(B, S, 3, 24, device="cuda")
        assert W.wbmm_rotary_forward(e, pos[:, :B, :S], freqs, (4, 6)).shape == (B, S, 3, 24)


# ---------------------------------------------------------------- attention

def attention_plain(q, k, v, lens, mask, scale, dout, dtype):
    """64-bit attention with gradients, and the bounds of this file's head.
    Entries of q, k, v, dout where nothing is visible may be anything."""
    B, Sq, Hq, D = q.shape
    Sk, Hk = k.shape[1], k.shape[2]
    G, u = Hq // Hk, U[dtype]
    least = 2.0 ** -126
    w16 = least if dtype == "f32" else 2.0 ** -25
    res = {n: torch.zeros(s, dtype=torch.float64) for n, s in
           (("out", q.shape), ("dq", q.shape), ("dk", k.shape), ("dv", k.shape), ("lse", (B, Hq, Sq)))}
    bound = {n: torch.zeros_like(t) for n, t in res.items()}
    res["lse"].fill_(-math.inf)
    for b in range(B):
        see = torch.ones(Sk, dtype=torch.bool) if mask is None else mask[b].bool().clone()
        if lens is not None:
            see[max(0, int(lens[b])):] = False
        idx = see.nonzero()[:, 0]
        n = idx.numel()
        if n == 0:
            continue
        for h in range(Hq):
            Q, K, V, dO = (t.double() for t in (q[b, :, h], k[b, idx, h // G], v[b, idx, h // G], dout[b, :, h]))
            s = scale * (Q @ K.T)
            d = scale * (D + 4) * 2.0 ** -24 * (Q.abs() @ K.abs().T).amax(-1, keepdim=True)
            r = 2 * d + 2.0 ** -20 + 2.0 ** -22 * s.abs().amax(-1, keepdim=True)
            p = torch.softmax(s, -1)
            o = p @ V
            A = p @ V.abs()
            bo = (u + r + n * 2.0 ** -24) * A + w16 * V.abs().sum(0) + u * o.abs()
            res["out"][b, :, h], bound["out"][b, :, h] = o, bo
            res["lse"][b, h] = torch.logsumexp(s, -1)
            bound["lse"][b, h] = (d + r)[:, 0] + n * 2.0 ** -24 + 2.0 ** -22 * res["lse"][b, h].abs()
            # gradients: dp and delta in float32, delta from the rounded out
            sums = 2.0 ** -24
            dp = dO @ V.T
            delta = (dO * o).sum(-1, keepdim=True)
            edp = (D + 2) * sums * (dO.abs() @ V.abs().T)
            edelta = (dO.abs() * bo).sum(-1, keepdim=True) + (D + 2) * sums * (dO.abs() * (o.abs() + bo)).sum(-1, keepdim=True)
            ds = p * (dp - delta)
            eds = (2 * r + u) * ds.abs() + p * (1 + u) * (edp + edelta) * (1 + 2 * r) + w16 + least * (dp - delta).abs()
            ep = (2 * r + u) * p + w16
            rows = Sq * G
            res["dq"][b, :, h] = scale * ds @ K
            bound["dq"][b, :, h] = scale * (eds @ K.abs() + n * sums * (ds.abs() + eds) @ K.abs())
            res["dk"][b, idx, h // G] += scale * ds.T @ Q
            bound["dk"][b, idx, h // G] += scale * (eds.T @ Q.abs() + rows * sums * (ds.abs() + eds).T @ Q.abs())
            res["dv"][b, idx, h // G] += p.T @ dO
            bound["dv"][b, idx, h // G] += ep.T @ dO.abs() + rows * sums * (p + ep).T @ dO.abs()
    for m in ("dq", "dk", "dv"):
        bound[m] += u * (res[m].abs() + bound[m])
    return res, bound


def attention_inputs(B, Sq, Sk, Hq, Hk, D, dtype, seed=0, std=1.5):
    q, k, v, g = (draw((B, S, H, D), dtype, seed + i, s) for i, (S, H, s) in
                  enumerate(((Sq, Hq, std), (Sk, Hk, 1.0), (Sk, Hk, 1.0), (Sq, Hq, 1.0))))
    return q, k, v, g


def run_and_check(q, k, v, g, dtype, lens=None, mask=None, scale=None, dev=None, tag=""):
    """Forward and backward on the GPU (dev: the same tensors there, if they
    are laid out in some other way) against the plain results."""
    D = q.shape[3]
    sc = D ** -0.5 if scale is None else scale
    want, bound = attention_plain(q, k, v, lens, mask, sc, g, dtype)
    dq_, dk_, dv_, dg_ = dev if dev is not None else tuple(t.cuda() for t in (q, k, v, g))
    kw = dict(kv_lens=None if lens is None else lens.cuda(), key_mask=None if mask is None else mask.cuda(), scale=scale)
    out, lse = W.wbmm_cross_attention_forward(dq_, dk_, dv_, **kw)
    grads = W.wbmm_cross_attention_backward(dg_, dq_, dk_, dv_, out, lse, **kw)
    empty = want["lse"] == -math.inf
    assert torch.equal(lse.cpu() == -math.inf, empty), tag + " empty rows"
    finite = torch.where(empty, 0.0, lse.cpu().double())
    check(finite, torch.where(empty, 0.0, want["lse"]), bound["lse"], "f32", tag + " lse")
    check(out, want["out"], bound["out"], dtype, tag + " out")
    for n, t in zip(("dq", "dk", "dv"), grads):
        check(t, want[n], bound[n], dtype, tag + " " + n)
    return out, lse, grads


SHAPES = [
    # B, Sq, Sk, Hq, Hk, D
    (1, 1, 1, 1, 1, 1),
    (1, 1, 1, 4, 1, 128),
    (2, 1, 33, 8, 2, 64),
    (1, 1, 700, 8, 2, 128),       # one token, states in parts
    (2, 5, 1601, 4, 1, 96),       # 20 rows, in parts
    (1, 32, 31, 1, 1, 32),
    (2, 33, 65, 2, 2, 40),        # 33 rows: two waves a row tile
    (1, 64, 64, 2, 1, 64),
    (2, 17, 127, 9, 3, 72),
    (1, 129, 129, 3, 1, 128),
    (1, 130, 257, 2, 2, 80),
    (2, 100, 63, 5, 5, 8),
    (1, 43, 300, 6, 2, 7),        # odd components
    (1, 70, 90, 2, 1, 101),
    (3, 257, 40, 2, 2, 33),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,Sq,Sk,Hq,Hk,D", SHAPES)
def test_attention(B, Sq, Sk, Hq, Hk, D, dtype):
    run_and_check(*attention_inputs(B, Sq, Sk, Hq, Hk, D, dtype), dtype)


def hidden(B, Sk, kind, seed=5):
    """Lengths and masks that leave entries empty, full, or with holes."""
    g = torch.Generator().manual_seed(seed)
    lens = mask = None
    if "lens" in kind:
        lens = torch.randint(0, Sk + 1, (B,), generator=g, dtype=torch.int32)
        lens[0], lens[-1] = 0, Sk + 7  # none; past the end: all
    if "mask" in kind:
        mask = torch.rand((B, Sk), generator=g) < 0.6
        mask[B // 2] = False
        mask[-1, Sk // 3:] = False
    return lens, mask


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("kind", ["lens", "mask", "lens+mask"])
@pytest.mark.parametrize("Sq,Sk,Hq,Hk,D", [(1, 600, 4, 2, 64), (7, 100, 8, 2, 128), (60, 200, 2, 2, 72),
                                           (90, 300, 4, 2, 96), (5, 1, 2, 1, 32)])
def test_attention_hidden_states(kind, Sq, Sk, Hq, Hk, D, dtype):
    """Hidden states hold NaN and infinities; nothing of them may show."""
    B = 4
    q, k, v, g = attention_inputs(B, Sq, Sk, Hq, Hk, D, dtype, seed=20)
    lens, mask = hidden(B, Sk, kind)
    see = torch.ones(B, Sk, dtype=torch.bool) if mask is None else mask.clone()
    if lens is not None:
        see &= torch.arange(Sk)[None] < lens[:, None]
    k[~see], v[~see] = float("nan"), float("inf")
    _, _, (dq, dk, dv) = run_and_check(q, k, v, g, dtype, lens, mask)
    assert bool((dk.cpu()[~see] == 0).all()) and bool((dv.cpu()[~see] == 0).all())
    none = ~see.any(1)
    assert bool((dq.cpu()[none] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_layouts(dtype):
    """Slices of joint projections, [B,H,S,D] order, rows that are not whole
    16-byte pieces, and queries broadcast over the batch."""
    B, Sq, Sk, Hq, Hk, D = 2, 50, 75, 4, 2, 48
    q, k, v, g = attention_inputs(B, Sq, Sk, Hq, Hk, D, dtype, seed=30)
    plain = run_and_check(q, k, v, g, dtype, tag="dense")
    kv = torch.stack([k, v], 2).cuda()
    dev = (q.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3), kv[:, :, 0], kv[:, :, 1], g.cuda())
    other = run_and_check(q, k, v, g, dtype, dev=dev, tag="slices")
    assert all(torch.equal(a, b) for a, b in zip(plain[2], other[2])) and torch.equal(plain[0], other[0])

    def shifted(t):  # one element off 16-byte alignment, rows one element apart
        wide = torch.empty(t.shape[0], t.shape[1], t.shape[2], D + 1, dtype=t.dtype, device="cuda")
        wide[..., 1:] = t.cuda()
        return wide[..., 1:]

    odd = run_and_check(q, k, v, g, dtype, dev=tuple(shifted(t) for t in (q, k, v, g)), tag="shifted")
    assert all(torch.equal(a, b) for a, b in zip(plain[2], odd[2])) and torch.equal(plain[0], odd[0])
    q1 = q[:1].expand(B, Sq, Hq, D)
    run_and_check(q1, k, v, g, dtype, dev=(q[:1].cuda().expand(B, Sq, Hq, D), k.cuda(), v.cuda(), g.cuda()), tag="broadcast")


def test_attention_outputs_in_place_of_slices():
    """Outputs into slices of joint tensors; what lies beside them stays."""
    B, Sq, Sk, H, D = 2, 20, 35, 2, 32
    q, k, v, g = (t.cuda() for t in attention_inputs(B, Sq, Sk, H, H, D, "f16", seed=40))
    out, lse = W.wbmm_cross_attention_forward(q, k, v)
    dq, dk, dv = W.wbmm_cross_attention_backward(g, q, k, v, out, lse)
    wide = torch.full((B, Sq, 3, H, D), 7.0, dtype=q.dtype, device="cuda")
    o2, lse2 = W.wbmm_cross_attention_forward(q, k, v, out=wide[:, :, 1])
    assert torch.equal(wide[:, :, 1], out) and torch.equal(lse, lse2) and o2.data_ptr() == wide[:, :, 1].data_ptr()
    assert bool((wide[:, :, ::2] == 7.0).all())
    joint = torch.full((B, Sk, 3, H, D), 7.0, dtype=q.dtype, device="cuda")
    W.wbmm_cross_attention_backward(g, q, k, v, out, lse, dq=wide[:, :, 2], dk=joint[:, :, 0], dv=joint[:, :, 2])
    assert torch.equal(wide[:, :, 2], dq) and torch.equal(joint[:, :, 0], dk) and torch.equal(joint[:, :, 2], dv)
    assert bool((joint[:, :, 1] == 7.0).all()) and torch.equal(wide[:, :, 1], out)


@pytest.mark.parametrize("Sq,Sk", [(0, 5), (5, 0), (0, 0)])
def test_attention_empty_lengths(Sq, Sk):
    q, g = (torch.randn(2, Sq, 4, 16, device="cuda") for _ in range(2))
    k, v = (torch.randn(2, Sk, 2, 16, device="cuda") for _ in range(2))
    out, lse = W.wbmm_cross_attention_forward(q, k, v)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all()) and out.shape == q.shape
    for t, like in zip(W.wbmm_cross_attention_backward(g, q, k, v, out, lse), (q, k, v)):
        assert t.shape == like.shape and bool((t == 0).all())
    e = q[:0]
    assert W.wbmm_cross_attention_forward(e, k[:0], v[:0])[0].shape == e.shape


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_attention_sharp_and_large_scores(dtype):
    """One state that takes everything, scores in the thousands, growing
    along the states so that the running maximum moves in every tile."""
    B, Sq, Sk, H, D = 1, 70, 400, 2, 32
    q, k, v, g = attention_inputs(B, Sq, Sk, H, H, D, dtype, seed=50)
    k = (k * torch.linspace(0.5, 30.0, Sk)[None, :, None, None]).to(DT[dtype])
    run_and_check(q, k, v, g, dtype, scale=2.0, tag="growing")
    run_and_check(q, k.flip(1), v, g, dtype, scale=2.0, tag="falling")
    run_and_check(q[:, :3], k, v, g[:, :3], dtype, scale=2.0, tag="few rows")


def test_attention_nan_stays_in_its_row():
    """A NaN query poisons its own row only; a visible NaN state poisons all
    rows of its entry and head group, and nothing else."""
    q, k, v, _ = (t.cuda() for t in attention_inputs(2, 40, 90, 4, 2, 32, "bf16", seed=60))
    clean, _ = W.wbmm_cross_attention_forward(q, k, v)
    q2 = q.clone()
    q2[0, 3, 1] = float("nan")
    out, lse = W.wbmm_cross_attention_forward(q2, k, v)
    bad = torch.zeros(2, 40, 4, dtype=torch.bool, device="cuda")
    bad[0, 3, 1] = True
    assert bool(out[bad].isnan().all()) and torch.equal(out[~bad], clean[~bad])
    assert torch.equal(lse.permute(0, 2, 1).isnan(), bad)
    k2 = k.clone()
    k2[1, 80, 1] = float("nan")
    out, _ = W.wbmm_cross_attention_forward(q, k2, v)
    bad = torch.zeros(2, 40, 4, dtype=torch.bool, device="cuda")
    bad[1, :, 2:] = True
    assert bool(out[bad].isnan().all()) and torch.equal(out[~bad], clean[~bad])


@pytest.mark.parametrize("Sq,Hq,D", [(3, 4, 32), (60, 2, 64), (40, 2, 128), (150, 2, 64)])
def test_attention_nan_rows_leave_hidden_states_alone(Sq, Hq, D):
    """Rows that hold NaN poison the gradients of what they see; hidden
    states' gradients are zero all the same, and other rows' are untouched."""
    q, k, v, g = (t.cuda() for t in attention_inputs(2, Sq, 90, Hq, 2, D, "bf16", seed=65))
    mask = torch.rand(2, 90, generator=torch.Generator().manual_seed(66)).cuda() < 0.5
    out, lse = W.wbmm_cross_attention_forward(q, k, v, key_mask=mask)
    clean = W.wbmm_cross_attention_backward(g, q, k, v, out, lse, key_mask=mask)
    q[1, 2, 0], g[1, 1, Hq - 1] = float("nan"), float("nan")
    out, lse = W.wbmm_cross_attention_forward(q, k, v, key_mask=mask)
    dq, dk, dv = W.wbmm_cross_attention_backward(g, q, k, v, out, lse, key_mask=mask)
    assert bool((dk[~mask] == 0).all()) and bool((dv[~mask] == 0).all())
    rows = torch.ones(2, Sq, Hq, dtype=torch.bool, device="cuda")
    rows[1, 2, 0] = rows[1, 1, Hq - 1] = False
    assert torch.equal(dq[rows], clean[0][rows]) and bool(dq[~rows].isnan().all())
    assert torch.equal(dk[0], clean[1][0]) and torch.equal(dv[0], clean[2][0])


@pytest.mark.parametrize("Sq,Hq,D", [(3, 4, 32), (60, 2, 64), (40, 2, 128), (150, 2, 64)])
def test_attention_nan_gradient_where_nothing_is_visible(Sq, Hq, D):
    """Rows that see nothing have no gradient, whatever comes from above."""
    q, k, v, g = (t.cuda() for t in attention_inputs(2, Sq, 90, Hq, 2, D, "bf16", seed=67))
    mask = torch.ones(2, 90, dtype=torch.bool, device="cuda")
    mask[1] = False
    g[1], q[1, 0] = float("nan"), float("nan")
    out, lse = W.wbmm_cross_attention_forward(q, k, v, key_mask=mask)
    assert bool((out[1] == 0).all()) and bool((lse[1] == -math.inf).all())
    for t in W.wbmm_cross_attention_backward(g, q, k, v, out, lse, key_mask=mask):
        assert bool((t[1] == 0).all()) and bool(t[0].isfinite().all())


def test_attention_long_cache_offsets():
    """States that lie more than 2^32 bytes into their tensor."""
    B, Sk, H, D = 2, 700, 2, 64
    far = torch.zeros(B, (1 << 31) // (H * D) + Sk, H, D, dtype=torch.bfloat16, device="cuda")
    q, k, v, g = attention_inputs(B, 40, Sk, H, H, D, "bf16", seed=70)
    kd = far[:, -Sk:]
    kd.copy_(k.cuda())
    run_and_check(q, k, v, g, "bf16", dev=(q.cuda(), kd, v.cuda(), g.cuda()), tag="rows")
    run_and_check(q[:, :2], k, v, g[:, :2], "bf16", dev=(q[:, :2].cuda(), kd, v.cuda(), g[:, :2].cuda()), tag="token")


@pytest.mark.parametrize("Sq,Hq", [(2, 4), (50, 2)])
def test_attention_wide_strides(Sq, Hq):
    """States more than 2^31 bytes apart."""
    Sk, D = 3, 16
    wide = torch.zeros(Sk, (1 << 30) + 16, dtype=torch.bfloat16, device="cuda")
    q, k, v, g = attention_inputs(1, Sq, Sk, Hq, 1, D, "bf16", seed=75)
    kd = wide[None, :, None, 8:8 + D]
    kd.copy_(k.cuda())
    run_and_check(q, k, v, g, "bf16", dev=(q.cuda(), kd, v.cuda(), g.cuda()))


def test_attention_same_bits_every_time():
    """Repeated calls, and calls on fewer entries, give the same bits."""
    for Sq, Sk in ((1, 3000), (200, 333)):
        q, k, v, g = (t.cuda() for t in attention_inputs(3, Sq, Sk, 4, 2, 64, "bf16", seed=80))

        def both():
            out, lse = W.wbmm_cross_attention_forward(q, k, v)
            return (out, lse) + W.wbmm_cross_attention_backward(g, q, k, v, out, lse)

        first = both()
        for _ in range(3):
            assert all(torch.equal(a, b) for a, b in zip(first, both()))


def test_attention_other_stream():
    """Calls on a stream given by argument or made current."""
    q, k, v, g = (t.cuda() for t in attention_inputs(2, 1, 2000, 8, 2, 64, "bf16", seed=90))
    want, lse = W.wbmm_cross_attention_forward(q, k, v)
    grads = W.wbmm_cross_attention_backward(g, q, k, v, want, lse)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    a, la = W.wbmm_cross_attention_forward(q, k, v, stream=s)
    ga = W.wbmm_cross_attention_backward(g, q, k, v, a, la, stream=s)
    with torch.cuda.stream(s):
        b, _ = W.wbmm_cross_attention_forward(q, k, v)
    s.synchronize()
    assert torch.equal(a, want) and torch.equal(b, want) and all(torch.equal(x, y) for x, y in zip(ga, grads))


def test_attention_graphs_share_nothing():
    """Two graphs captured on one stream, replayed on two streams at once, and
    replays between eager calls."""
    sets = [tuple(t.cuda() for t in attention_inputs(2, 1, 4000, 8, 2, 64, "bf16", seed=s)) for s in (100, 110)]
    want = []
    for q, k, v, g in sets:
        out, lse = W.wbmm_cross_attention_forward(q, k, v)
        want.append((out, lse) + W.wbmm_cross_attention_backward(g, q, k, v, out, lse))
    torch.cuda.synchronize()
    cap = torch.cuda.Stream()
    graphs, outs = [], []
    for q, k, v, g in sets:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=cap):
            out, lse = W.wbmm_cross_attention_forward(q, k, v)
            outs.append((out, lse) + W.wbmm_cross_attention_backward(g, q, k, v, out, lse))
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(4):
        for o in outs:
            for t in o:
                t.zero_()
        torch.cuda.synchronize()
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert all(torch.equal(a, b) for a, b in zip(o, w))
        again, _ = W.wbmm_cross_attention_forward(*sets[0][:3])
        assert torch.equal(again, want[0][0])


def test_attention_refuses():
    q, k = torch.zeros(2, 3, 4, 16, device="cuda"), torch.zeros(2, 5, 2, 16, device="cuda")
    f, b = W.wbmm_cross_attention_forward, W.wbmm_cross_attention_backward
    for bad in (k[:1], k[..., :8], k.half(), k.cpu(), k.transpose(2, 3)):
        with pytest.raises(ValueError):
            f(q, k, bad)
        with pytest.raises(ValueError):
            f(q, bad, k)
    with pytest.raises(ValueError):
        f(q[:, :, :3], k, k)                                      # heads do not divide
    with pytest.raises(TypeError):
        f(q.double(), k.double(), k.double())
    with pytest.raises(TypeError):
        f(q, k, k, kv_lens=torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        f(q, k, k, kv_lens=torch.zeros(3, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        f(q, k, k, kv_lens=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(TypeError):
        f(q, k, k, key_mask=torch.zeros(2, 5, device="cuda"))     # additive masks
    with pytest.raises(ValueError):
        f(q, k, k, key_mask=torch.zeros(2, 4, dtype=torch.bool, device="cuda"))
    for scale in (0.0, -1.0, float("nan")):
        with pytest.raises(W.WbmmError):
            f(q, k, k, scale=scale)
    wide = torch.zeros(2, 3, 4, 136, device="cuda")
    with pytest.raises(W.WbmmError):
        f(wide, wide, wide)
    with pytest.raises(W.WbmmError):
        f(q, k, k, out=q)
    out, lse = f(q, k, k)
    with pytest.raises(ValueError):
        b(out[:1], q, k, k, out, lse)
    with pytest.raises(ValueError):
        b(out, q, k, k, out, lse.half())
    with pytest.raises(W.WbmmError):
        b(out, q, k, k, out, lse, dk=k)
    with pytest.raises(ValueError):
        W.wbmm_rotary_forward(q, torch.zeros(1, 2, 4, dtype=torch.int64, device="cuda"), torch.ones(4, device="cuda"), (4,))
    with pytest.raises(TypeError):
        W.wbmm_rotary_forward(q, torch.zeros(1, 2, 3, device="cuda"), torch.ones(4, device="cuda"), (4,))
    with pytest.raises(W.WbmmError):
        W.wbmm_rotary_forward(q, torch.zeros(1, 2, 3, dtype=torch.int64, device="cuda"), torch.ones(9, device="cuda"), (9,))


def test_attention_gradient_by_differences():
    """Directional derivatives of a float32 loss by central differences,
    through rotation and attention together."""
    B, Sq, Sk, Hq, Hk, D, sections = 2, 6, 40, 4, 2, 16, (3, 5)
    q, k, v, g = (t.cuda() for t in attention_inputs(B, Sq, Sk, Hq, Hk, D, "f32", seed=120))
    pq, pk = positions(2, B, Sq, 121, 0, 20).cuda(), positions(2, B, Sk, 122, 0, 20).cuda()
    freqs = W.wbmm_rotary_frequencies(sections)
    lens = torch.tensor([Sk, 17], dtype=torch.int32, device="cuda")

    def layer(q, k, v):
        return W.wbmm_cross_attention(W.wbmm_rotary(q, pq, freqs, sections), W.wbmm_rotary(k, pk, freqs, sections), v, lens)

    leaves = [t.requires_grad_(True) for t in (q, k, v)]
    grads = torch.autograd.grad(layer(*leaves), leaves, g)
    step = 2.0 ** -7
    for i in range(3):
        d = draw(leaves[i].shape, "f32", 130 + i).cuda()
        at = lambda e: [t.detach() + (e * d if j == i else 0.0) for j, t in enumerate(leaves)]
        up, down = ((layer(*at(e)).double() * g.double()).sum().item() for e in (step, -step))
        slope = (up - down) / (2 * step)
        want = (grads[i].double() * d.double()).sum().item()
        # float32 sums of the two losses over the step, and the differences' own
        # error: step^2 / 6 of a third derivative, of the order of the slope's
        # terms times the third power of the score's change (below 4 here)
        size = (grads[i].double().abs() * d.double().abs()).sum().item()
        loss = (layer(*leaves).double().abs() * g.double().abs()).sum().item()
        assert abs(slope - want) <= 2.0 ** -20 * loss / step + step * step / 6 * 64 * size


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layer_of_both_operators(dtype):
    """A decoder's tokens read a map, as they would in training: window
    products on the map, rotation of queries and keys, attention; outputs and
    gradients against 64 bits, and a captured step equal to the eager one."""
    B, Sq, Hh, Ww, Hq, Hk, D, sections = 2, 24, 14, 14, 4, 2, 32, (4, 6, 6)
    Sk, C = Hh * Ww, Hk * D
    x = draw((B, 2 * C, Hh, Ww), dtype, 140).cuda()
    table = (draw((2 * C, 27 * 27), "f32", 141) * 0.02).to(DT[dtype]).cuda()
    q, g = draw((B, Sq, Hq, D), dtype, 142, 1.5).cuda(), draw((B, Sq, Hq, D), dtype, 143).cuda()
    freqs = W.wbmm_rotary_frequencies(sections)
    pq = positions(3, B, Sq, 144, 0, 40).cuda()
    at = torch.arange(Sk, device="cuda")
    pk = torch.stack([at * 0, at // Ww, at % Ww])[:, None].expand(3, B, Sk)

    def step(x, table, q):
        kv = W.wbmm(x, table, 14).flatten(2).transpose(1, 2).reshape(B, Sk, 2, Hk, D)
        kr = W.wbmm_rotary(kv[:, :, 0], pk, freqs, sections)
        qr = W.wbmm_rotary(q, pq, freqs, sections)
        v = kv[:, :, 1]
        out = W.wbmm_cross_attention(qr, kr, v)
        return (out, qr, kr, v) + torch.autograd.grad(out, (qr, kr, v, x, table, q), g)

    leaves = [t.requires_grad_(True) for t in (x, table, q)]
    out, qr, kr, v, dqr, dkr, dv, dx, dt, dq = step(*leaves)
    # the attention on its own inputs, and the rotation's gradient on its own
    want, bound = attention_plain(*(t.detach().cpu() for t in (qr, kr, v)), None, None, D ** -0.5, g.cpu(), dtype)
    for name, t in (("out", out), ("dq", dqr), ("dk", dkr), ("dv", dv)):
        check(t, want[name], bound[name], dtype, name)
    wq, mag = rotary_plain(dqr.cpu(), pq.cpu(), freqs.cpu(), sections, False, -1.0)
    check(dq, wq, U[dtype] * wq.abs() + 2.0 ** -21 * mag, dtype, "dq of the leaf")
    dkv = torch.stack([W.wbmm_rotary_backward(dkr, pk, freqs, sections), dv], 2)
    dmap = dkv.reshape(B, Sk, 2 * C).transpose(1, 2).reshape(B, 2 * C, Hh, Ww).contiguous()
    ex, et = W.wbmm_backward(x.detach(), dmap, table.detach(), 14)
    assert torch.equal(dx, ex) and torch.equal(dt, et.to(dt.dtype))
    eager = [t.detach().clone() for t in (out, dx, dt, dq)]
    del out, qr, kr, v, dqr, dkr, dv, dx, dt, dq
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*leaves)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = step(*leaves)
        caught = [r[0], r[7], r[8], r[9]]
    for _ in range(3):
        for t in caught:
            t.detach().zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(caught, eager))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,Sk", [(32, 100), (64, 470), (96, 200), (128, 64), (128, 330)])
def test_attention_a_tile_for_each_unit(Sk, D, dtype):
    """Tiles of 128 rows, about one for each compute unit, of one to eight
    tiles of states, the last one partial, straight to LDS."""
    run_and_check(*attention_inputs(25, 128, Sk, 8, 8, D, dtype, seed=150), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("kind", ["", "lens+mask"])
@pytest.mark.parametrize("Sq,D", [(40, 24), (50, 37), (64, 72), (33, 128), (100, 64), (65, 37), (128, 72), (90, 128)])
def test_attention_tiles_of_64_and_128_rows(Sq, D, kind, dtype):
    """As many heads as take whole tiles of rows, in rows of whole 16-byte
    pieces and others, masked and not, two tiles of states."""
    B, H, Sk = 48, 4, 77
    lens, mask = hidden(B, Sk, kind)
    run_and_check(*attention_inputs(B, Sq, Sk, 2 * H if Sq == 33 else H, H, D, dtype, seed=160), dtype, lens, mask)


def test_attention_small_and_large_scales():
    """Weights that are all alike, and one state that takes everything."""
    for dtype in DT:
        q, k, v, g = attention_inputs(2, 70, 50, 2, 2, 32, dtype, seed=170)
        for scale in (1e-30, 1e-4, 16.0):
            run_and_check(q, k, v, g, dtype, scale=scale, tag="scale %g" % scale)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("kind", ["", "lens", "lens+mask", "gap"])
@pytest.mark.parametrize("Sq,Sk,Hq,Hk,D", [(130, 700, 1, 1, 64), (100, 330, 2, 1, 128), (70, 500, 3, 1, 37),
                                           (520, 130, 2, 1, 72)])
def test_attention_gradients_in_parts(Sq, Sk, Hq, Hk, D, kind, dtype):
    """Few heads: states and rows both in parts, whose partial sums share a
    workspace; hidden states, whole tiles of them too, hold NaN."""
    B = 3
    q, k, v, g = attention_inputs(B, Sq, Sk, Hq, Hk, D, dtype, seed=180)
    lens, mask = hidden(B, Sk, kind)
    if kind == "gap":
        mask = torch.ones(B, Sk, dtype=torch.bool)
        mask[0, 30:Sk - 3] = mask[1, :64] = mask[2, 64:128] = False
    see = torch.ones(B, Sk, dtype=torch.bool) if mask is None else mask.clone()
    if lens is not None:
        see &= torch.arange(Sk)[None] < lens[:, None]
    k[~see], v[~see] = float("nan"), float("nan")
    _, _, (_, dk, dv) = run_and_check(q, k, v, g, dtype, lens, mask)
    assert bool((dk.cpu()[~see] == 0).all()) and bool((dv.cpu()[~see] == 0).all())


@pytest.mark.parametrize("Sq,D", [(128, 128), (128, 72), (50, 64), (1, 64)])
def test_attention_infinite_values_keep_their_sign(Sq, D):
    """An infinite component of a visible state's values comes out as itself,
    the last state's too, beside which a tile is filled up."""
    q, k, v, _ = (t.cuda() for t in attention_inputs(25, Sq, 70, 8, 8, D, "bf16", seed=190))
    clean, _ = W.wbmm_cross_attention_forward(q, k, v)
    v[:, -1, :, 5] = float("inf")
    out, _ = W.wbmm_cross_attention_forward(q, k, v)
    keep = torch.arange(D, device="cuda") != 5
    assert bool((out[..., 5] == float("inf")).all()) and torch.equal(out[..., keep], clean[..., keep])
