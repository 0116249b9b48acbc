"""CPU-side checks of the rotary and cross attention entry points: refusals
of the C ABI (only calls that fail validation, or have no work, are sent, so
no kernel is ever launched here) and of the Python binding."""
import ctypes

import pytest
import torch

from paper_2607_02097_amd import binding as W

E, U, OK = W.WBMM_ERR_INVALID_ARG, W.WBMM_ERR_UNSUPPORTED, W.WBMM_OK
FAR = 1 << 32  # addresses that are never dereferenced, this far apart


@pytest.fixture(scope="module")
def lib():
    return W.load_library()


def dense(at, S, H, D):
    return (at, S * H * D, H * D, D)


def rotary(lib, fn="wbmm_rotary_forward", x=None, y=None, pos=8 * FAR, pos_bytes=8, pos_strides=None, freqs=9 * FAR,
           axes=3, sections=(2, 3, 3), adjacent=0, B=2, S=5, H=4, D=16, dtype=1):
    x = dense(FAR, S, H, D) if x is None else x
    y = dense(2 * FAR, S, H, D) if y is None else y
    pos_strides = (B * S, S, 1) if pos_strides is None else pos_strides
    sections = tuple(sections) + (0,) * (4 - len(sections))
    args = W._ROTARY_ARGS.pack(*x, *y, pos, pos_bytes, *pos_strides, freqs, axes, *sections, adjacent, B, S, H, D, dtype)
    return getattr(lib, fn)(args, None)


@pytest.mark.parametrize("fn", ["wbmm_rotary_forward", "wbmm_rotary_backward"])
def test_rotary_refusals(lib, fn):
    def call(**kw):
        return rotary(lib, fn, **kw)

    assert getattr(lib, fn)(None, None) == E
    assert call(dtype=3) == U and call(dtype=-1) == U
    assert call(x=dense(0, 5, 4, 16)) == E and call(y=dense(0, 5, 4, 16)) == E
    assert call(x=dense(FAR + 1, 5, 4, 16)) == E                    # misaligned
    assert call(pos=0) == E and call(freqs=0) == E
    assert call(pos=8 * FAR + 4) == E and call(pos_bytes=2) == E and call(freqs=9 * FAR + 2) == E
    assert call(axes=0) == E and call(axes=5) == U
    assert call(sections=(2, -1, 3)) == E and call(sections=(0, 0, 0)) == E
    assert call(sections=(3, 3, 3)) == E                            # 2 P > D
    assert call(sections=(200, 100, 0), D=1024) == U                # P > 256
    assert call(D=8192) == U
    assert call(B=-1) == E and call(S=-1) == E and call(H=0) == E
    assert call(x=(FAR, 320, 64, -16)) == E and call(pos_strides=(10, -5, 1)) == E
    assert call(x=(FAR, 1 << 62, 64, 16)) == E                      # past any memory
    # ranges that meet: shifted copies, entries folded onto one address, the positions
    assert call(y=dense(FAR + 32, 5, 4, 16)) == E
    assert call(y=(2 * FAR, 0, 64, 16)) == E and call(y=(2 * FAR, 320, 64, 8)) == E
    assert call(y=dense(8 * FAR, 5, 4, 16)) == E and call(y=dense(9 * FAR, 5, 4, 16)) == E
    # one tensor, other strides: not in place
    assert call(x=(FAR, 320, 64, 16), y=(FAR, 320, 16, 80)) == E
    # too many tokens for a launch
    assert call(B=1 << 14, S=1 << 14, H=64, D=128, x=(FAR, 0, 0, 0), y=(1 << 44, (1 << 14) * 8192, 8192, 128)) == U
    # nothing to do
    assert call(B=0) == OK and call(S=0, x=(0, 0, 64, 16), y=(0, 0, 64, 16)) == OK


def attention(lib, fn="forward", size=False, **kw):
    # (float32 gradients need a workspace for the rows' statistics)
    p = dict(B=2, Sq=3, Sk=5, Hq=8, Hk=4, D=64, scale=0.125, dtype=0 if fn == "backward" else 1, lse=20 * FAR, lens=0, mask=0, mask_b=5, mask_s=1,
             ws=21 * FAR, ws_bytes=1 << 30)
    names = ("q", "k", "v", "out", "dout", "dq", "dk", "dv")
    p.update({k: v for k, v in kw.items() if k not in names})
    tok = []
    for i, n in enumerate(names):
        S, H = (p["Sk"], p["Hk"]) if n in ("k", "v", "dk", "dv") else (p["Sq"], p["Hq"])
        tok += list(kw.get(n, dense((i + 1) * FAR, S, H, p["D"])))
    args = W._ATTENTION_ARGS.pack(*tok, p["lse"], p["lens"], p["mask"], p["mask_b"], p["mask_s"], p["B"], p["Sq"],
                                  p["Sk"], p["Hq"], p["Hk"], p["D"], p["scale"], p["dtype"], p["ws"], p["ws_bytes"])
    if size:
        return getattr(lib, "wbmm_cross_attention_%s_workspace_bytes" % fn)(args)
    return getattr(lib, "wbmm_cross_attention_" + fn)(args, None)


@pytest.mark.parametrize("fn", ["forward", "backward"])
def test_attention_refusals(lib, fn):
    def call(**kw):
        return attention(lib, fn, **kw)

    assert getattr(lib, "wbmm_cross_attention_" + fn)(None, None) == E
    assert call(dtype=7) == U
    assert call(D=129) == U and call(D=0) == E
    assert call(Hq=9) == E and call(Hk=0) == E and call(Hq=0) == E
    assert call(B=-1) == E and call(Sq=-1) == E and call(Sk=-1) == E
    assert call(Sq=1 << 30) == U and call(Sk=1 << 31) == U
    for scale in (0.0, -1.0, float("inf"), float("nan"), 1e-60, 1e-31, 3e38):
        assert call(scale=scale) == E, scale
    for n in ("q", "k", "v", "out") + (("dout", "dq", "dk", "dv") if fn == "backward" else ()):
        S, H = (5, 4) if n in ("k", "v", "dk", "dv") else (3, 8)
        assert call(**{n: dense(0, S, H, 64)}) == E, n
        assert call(**{n: dense(FAR * 30 + 1, S, H, 64)}) == E, n
        assert call(**{n: (FAR * 30, -1, H * 64, 64)}) == E, n
    assert call(lens=22 * FAR + 2) == E and call(lse=20 * FAR + 1) == E
    assert call(mask=22 * FAR, mask_b=-5) == E and call(mask=22 * FAR, mask_b=1 << 60) == E
    # outputs on inputs, on each other or on themselves
    for o in ("out",) if fn == "forward" else ("dq", "dk", "dv"):
        S, H = (5, 4) if o in ("dk", "dv") else (3, 8)
        assert call(**{o: dense(FAR + 64, S, H, 64)}) == E, o        # on q
        assert call(**{o: dense(20 * FAR, S, H, 64)}) == E, o        # on lse
        assert call(**{o: (FAR * 30, 0, H * 64, 64)}) == E, o        # entries folded
        assert call(**{o: (FAR * 30, S * H * 64, H * 64, 32)}) == E, o
        assert call(lens=FAR * 30, **{o: dense(FAR * 30, S, H, 64)}) == E, o
        assert call(mask=FAR * 30, **{o: dense(FAR * 30, S, H, 64)}) == E, o
    if fn == "backward":
        assert call(dk=dense(FAR * 30, 5, 4, 64), dv=dense(FAR * 30 + 128, 5, 4, 64)) == E
        assert call(lse=0) == E
        # slices of one joint tensor are taken apart, but not if they reach into each other
        joint = (5 * 512, 512, 64)
        assert call(dk=(FAR * 30, *joint), dv=(FAR * 30 + 2 * 192, *joint)) == E
        assert attention(lib, fn, size=True) > 0
        assert call(dk=(FAR * 30, *joint), dv=(FAR * 30 + 2 * 256, *joint), ws=0) == E
        assert call(ws_bytes=attention(lib, fn, size=True) - 1) == E and call(ws=21 * FAR + 8) == E
        assert call(ws=FAR) == E                                     # workspace on q
        assert call(Sq=0, Sk=0) == OK
    else:
        assert call(Sq=0) == OK
    assert call(B=0) == OK
    # more tiles than a launch holds (broadcast inputs; outputs far apart)
    wide = {n: ((8 + i) << 41, 0, 0, 0) for i, n in enumerate(("q", "k", "v", "dout"))}
    wide["dk"], wide["dv"] = (30 << 41, 1 << 30, 1, 0), (31 << 41, 1 << 30, 1, 0)
    if fn == "forward":
        assert call(B=1, Sq=1 << 29, Sk=1, Hq=4, Hk=4, D=1, **{**wide, "out": (20 << 41, 0, 4, 1)}) == U
    else:
        assert call(B=2, Sq=1, Sk=1 << 30, Hq=1, Hk=1, D=1, **{**wide, "out": (20 << 41, 1, 0, 0), "dq": (21 << 41, 1, 0, 0)},
                    ws=40 << 41, ws_bytes=1 << 40) == U


def slices(lib, fn, B, S, H, D, order, first, second):
    """A rotary call from one slice of a joint bfloat16 tensor to another that
    fails on its positions alone, if not on the slices."""
    if order == "bshd":
        strides = (S * 3 * H * D, 3 * H * D, D)
        at = lambda i: FAR + int(2 * i * H * D)
    else:  # [B, 3 H, S, D]
        strides = (3 * H * S * D, D, S * D)
        at = lambda i: FAR + int(2 * i * H * S * D)
    kw = dict(B=B, S=S, H=H, D=D, sections=(2,), axes=1)
    clash = rotary(lib, fn, x=(at(first),) + strides, y=(at(second),) + strides, **kw) == E
    return clash


@pytest.mark.parametrize("order", ["bshd", "bhsd"])
@pytest.mark.parametrize("B,S", [(2, 5), (8, 1), (1, 7)])
def test_slices_of_one_tensor(lib, order, B, S):
    """Slices that are apart pass the overlap check in every order (the calls
    then fail on the launch, there being no GPU); ones that meet do not."""
    if torch.cuda.is_available():
        pytest.skip("would launch")
    fn = "wbmm_rotary_forward"
    assert not slices(lib, fn, B, S, 4, 16, order, 0, 1)
    assert not slices(lib, fn, B, S, 4, 16, order, 2, 0)
    assert slices(lib, fn, B, S, 4, 16, order, 0, 0.5)
    assert slices(lib, fn, B, S, 4, 16, order, 1, 0.75)


def test_attention_workspace_query(lib):
    assert attention(lib, "forward", size=True, dtype=9) == 0
    assert attention(lib, "backward", size=True, D=200) == 0
    # nor does a call that is past the launch limits
    assert attention(lib, "backward", size=True, B=1 << 15, Hq=1 << 15, Hk=1 << 15, Sq=1 << 30, Sk=1 << 30) == 0
    # one token over many states goes in parts; the parts' results take space
    long = dict(B=1, Sq=1, Sk=100000, Hq=8, Hk=8, D=128)
    need = attention(lib, "forward", size=True, **long)
    assert need > 0 and need % (8 * 129 * 4) == 0
    assert attention(lib, "forward", ws=0, **long) == E
    assert attention(lib, "forward", ws_bytes=need - 16, **long) == E
    # a row's statistics: two float32 values; none where one kernel does it all
    assert attention(lib, "backward", size=True, dtype=1, B=64, Sq=128, Sk=4096, Hq=16, Hk=16) == 64 * 128 * 16 * 8
    assert attention(lib, "backward", size=True, dtype=1, B=64, Sq=64, Sk=4096, Hq=16, Hk=16) == 0


def test_binding_refusals():
    """Arguments that the binding refuses before the library sees them (host
    tensors never reach it)."""
    x = torch.zeros(1, 2, 3, 8)
    pos, f = torch.zeros(1, 1, 2, dtype=torch.int64), torch.ones(4)
    with pytest.raises(ValueError, match="GPU"):
        W.wbmm_rotary_forward(x, pos, f, (4,))
    with pytest.raises(ValueError, match="GPU"):
        W.wbmm_cross_attention_forward(x, x, x)
    with pytest.raises(TypeError):
        W.wbmm_rotary_forward([1.0], pos, f, (4,))
    for sections in ((), (0, 0), (3, -1)):
        with pytest.raises(ValueError):
            W.wbmm_rotary_frequencies(sections, device="cpu")
    with pytest.raises(ValueError):
        W.wbmm_rotary_frequencies((2,), base=0.0, device="cpu")


def test_rotary_frequencies():
    f = W.wbmm_rotary_frequencies((1, 3), base=16.0, device="cpu")
    assert f.dtype == torch.float32 and torch.allclose(f, torch.tensor([1.0, 0.5, 0.25, 0.125]), rtol=1e-6, atol=0.0)
    g = W.wbmm_rotary_frequencies((2, 0, 1), base=16.0, restart=True, device="cpu")
    assert torch.allclose(g, torch.tensor([1.0, 0.25, 1.0]), rtol=1e-6, atol=0.0)


def test_argument_structs_match_the_header():
    """The packed formats have the sizes of the C structs (8-byte fields)."""
    assert W._ROTARY_ARGS.size == 25 * 8
    assert W._ATTENTION_ARGS.size == 47 * 8
    assert ctypes.sizeof(ctypes.c_void_p) == 8
