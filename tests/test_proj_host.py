"""Host side of the projection entry points: symbols, refusals, workspace sizes and frequencies, without a GPU."""
import ctypes as C
import math
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def pda():
    import paper_2511_12056_amd as pda
    return pda


def test_every_declared_symbol_is_exported(pda):
    text = open(os.path.join(ROOT, "include", "pipedit_proj.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\bint (pda_[a-z0-9_]+)\s*\(", text)))
    assert names == ["pda_fp8_matmul", "pda_fp8_matmul_workspace", "pda_fp8_quant", "pda_pack_heads_rope", "pda_pack_heads_rope_bwd", "pda_rms_norm_bwd",
                     "pda_rms_norm_bwd_workspace", "pda_rms_norm_fwd", "pda_rope_frequencies"]
    lib = C.CDLL(pda.lib_path())
    for n in names:
        assert getattr(lib, n) is not None


# Made-up device addresses, far apart; every call below fails its checks before one of them is used.
def _addr(i):
    return (i + 1) << 34


def _quant(pda, x=_addr(0), xt=1, rows=300, cols=200, ldx=200, ft=2, block=1, q=_addr(1), qs=_addr(2), qt=_addr(3), qts=_addr(4)):
    return pda.lib.pda_fp8_quant(x, xt, rows, cols, ldx, ft, block, q, qs, qt, qts, None)


@pytest.mark.parametrize("change,code,word", [
    (dict(xt=2), 1, "x_type"), (dict(ft=1), 1, "fp8_type"), (dict(ft=4), 1, "fp8_type"), (dict(block=2), 1, "block_rows"), (dict(rows=-1), 1, "rows"),
    (dict(cols=-1), 1, "cols"), (dict(ldx=199), 1, "ldx"), (dict(rows=1 << 31), 2, "2^31"), (dict(rows=1 << 30, ldx=1 << 20), 2, "2^40"), (dict(qs=None), 1, "together"),
    (dict(qt=None), 1, "together"), (dict(q=None, qs=None, qt=None, qts=None), 1, "nothing"), (dict(x=None), 1, "null x"), (dict(x=_addr(0) + 1), 2, "aligned"),
    (dict(q=_addr(1) + 4), 2, "16-byte"), (dict(qts=_addr(4) + 2), 2, "4-byte"), (dict(q=_addr(0) + 256), 1, "q overlaps x"), (dict(qts=_addr(1) + 16), 1, "overlaps"),
    (dict(qt=_addr(1) + 300 * 256 - 16), 1, "q overlaps qt"), (dict(qs=_addr(3)), 1, "q_scales overlaps qt"),
])
def test_quant_refuses(pda, change, code, word):
    assert _quant(pda, **change) == code and word in pda.last_error(), pda.last_error()


def test_quant_with_nothing_to_do(pda):
    assert _quant(pda, x=None, rows=0) == 0 and _quant(pda, x=None, cols=0, ldx=0) == 0


def _mm(pda, a=_addr(0), at=2, sa=_addr(1), b=_addr(2), sb=_addr(3), block=128, bias=_addr(4), out=_addr(5), M=300, N=200, K=256, ldo=200, ws=_addr(6), wb=1 << 30):
    return pda.lib.pda_fp8_matmul(a, at, sa, b, sb, block, bias, out, M, N, K, ldo, ws, wb, None)


@pytest.mark.parametrize("change,code,word", [
    (dict(M=-1), 1, "negative"), (dict(K=-128), 1, "negative"), (dict(K=200), 1, "multiple of 128"), (dict(K=1 << 24), 2, "2^24"), (dict(N=1 << 31, ldo=1 << 31), 2, "2^31"),
    (dict(M=1 << 30, N=1 << 12, ldo=1 << 12), 2, "2^40"), (dict(at=0), 1, "a_type"), (dict(block=64), 1, "b_block_rows"), (dict(ldo=199), 1, "ldo"),
    (dict(ldo=1 << 40), 1, "ldo"), (dict(out=None), 1, "null"), (dict(sb=None), 1, "null"), (dict(a=_addr(0) + 8), 2, "16-byte"), (dict(out=_addr(5) + 2), 2, "16-byte"),
    (dict(sa=_addr(1) + 1), 2, "4-byte"), (dict(bias=_addr(4) + 2), 2, "4-byte"), (dict(out=_addr(0) + 300 * 256 - 16), 1, "out overlaps a"), (dict(bias=_addr(5) + 64), 1, "out overlaps bias"),
])
def test_matmul_refuses(pda, change, code, word):
    assert _mm(pda, **change) == code and word in pda.last_error(), pda.last_error()


def test_matmul_with_nothing_to_do(pda):
    assert _mm(pda, M=0, a=None, out=None) == 0 and _mm(pda, N=0, ldo=0, b=None, out=None) == 0


def test_matmul_workspace(pda):
    size = pda.fp8_matmul_workspace_bytes
    assert size(1, 4608, 1536, n_cu=256) == 0 and size(119056, 4608, 1536, n_cu=256) == 0 and size(0, 5, 5, n_cu=256) == 0 and size(100, 5, 0, n_cu=256) == 0
    assert size(4608, 1536, 119056, n_cu=256) == size(4608, 1536, 119168, n_cu=256) > 0
    f = pda.lib.pda_fp8_matmul_workspace
    assert f(8, 8, 128, 256, None) == 1 and f(8, 8, 128, -1, C.byref(C.c_int64())) == 1 and f(8, 8, 100, 256, C.byref(C.c_int64())) == 1


@pytest.mark.parametrize("n_cu", [1, 64, 256, 304])
def test_matmul_workspace_of_extreme_sizes(pda, n_cu):
    """At most 32 parts, of results padded to tiles of 256."""
    top = 2 ** 31 - 1
    for M, N, K in ((1, 1, 2 ** 24 - 128), (top, 1, 128), (1, top, 128), (top, 256, 128), (256, 256, 2 ** 24 - 128), (4000, 4000, 65536), (1, 1, 128), (17, 1, 4096), (65536, 65536, 4096)):
        n = pda.fp8_matmul_workspace_bytes(M, N, K, n_cu=n_cu)
        assert 0 <= n <= 32 * 4 * (-(-M // 256) * 256) * (-(-N // 256) * 256)
        assert n == 0 or K > 128


def _rms(pda, x=_addr(0), xt=1, res=_addr(1), rt=0, w=_addr(2), h=_addr(3), y=_addr(4), yt=2, ys=_addr(5), rstd=_addr(6), rows=8, groups=1, D=200, eps=1e-6):
    return pda.lib.pda_rms_norm_fwd(x, xt, res, rt, w, h, y, yt, ys, rstd, rows, groups, D, eps, None)


@pytest.mark.parametrize("change,code,word", [
    (dict(xt=2), 1, "type"), (dict(rt=3), 1, "type"), (dict(yt=3), 1, "type"), (dict(rows=-1), 1, "rows"), (dict(groups=0), 1, "groups"), (dict(groups=3), 1, "multiple"),
    (dict(D=0), 1, "D=0"), (dict(D=8193), 2, "MAX"), (dict(rows=70000, groups=70000), 2, "65535"), (dict(rows=1 << 31), 2, "2^31"), (dict(eps=-1.0), 1, "eps"),
    (dict(eps=float("nan")), 1, "eps"), (dict(h=None), 1, "together"), (dict(res=None), 1, "together"), (dict(ys=None), 1, "y_scales"), (dict(yt=1), 1, "y_scales"),
    (dict(x=None), 1, "null"), (dict(y=None), 1, "null"), (dict(res=_addr(1) + 8), 2, "16-byte"), (dict(w=_addr(2) + 4), 2, "16-byte"), (dict(ys=_addr(5) + 1), 2, "4-byte"),
    (dict(rstd=_addr(6) + 2), 2, "4-byte"), (dict(h=_addr(0)), 1, "h overlaps x"), (dict(h=_addr(1) + 16), 1, "h overlaps res"), (dict(y=_addr(0)), 1, "y overlaps x"),
    (dict(y=_addr(3) + 64), 1, "y overlaps h"), (dict(ys=_addr(4) + 8 * 256 - 4), 1, "y overlaps y_scales"), (dict(rstd=_addr(2)), 1, "rstd overlaps weight"),
])
def test_rms_norm_fwd_refuses(pda, change, code, word):
    assert _rms(pda, **change) == code and word in pda.last_error(), pda.last_error()


def _rms_bwd(pda, dy=_addr(0), yt=1, h=_addr(1), ht=0, w=_addr(2), rstd=_addr(3), dres=_addr(4), dh=_addr(5), dw=_addr(6), rows=8, groups=1, D=64):
    return pda.lib.pda_rms_norm_bwd(dy, yt, h, ht, w, rstd, dres, dh, dw, rows, groups, D, None, 0, None)


@pytest.mark.parametrize("change,code,word", [
    (dict(yt=2), 1, "type"), (dict(ht=-1), 1, "type"), (dict(rows=9, groups=2), 1, "multiple"), (dict(D=9000), 2, "MAX"), (dict(dh=None, dw=None), 1, "nothing"),
    (dict(dy=None), 1, "null"), (dict(rstd=None), 1, "null"), (dict(dw=_addr(6) + 4), 2, "16-byte"), (dict(dres=_addr(4) + 4), 2, "16-byte"), (dict(rstd=_addr(3) + 1), 2, "4-byte"),
    (dict(dh=_addr(0)), 1, "dh overlaps dy"), (dict(dh=_addr(4) + 32), 1, "dh overlaps dres"), (dict(dw=_addr(1)), 1, "dweight overlaps h"), (dict(dw=_addr(2)), 1, "dweight overlaps weight"),
])
def test_rms_norm_bwd_refuses(pda, change, code, word):
    assert _rms_bwd(pda, **change) == code and word in pda.last_error(), pda.last_error()


def test_norm_with_nothing_to_do(pda):
    assert _rms(pda, x=None, res=None, w=None, h=None, y=None, ys=None, rstd=None, rows=0) == 0 and _rms_bwd(pda, dw=None, rows=0) == 0


def test_rms_norm_bwd_workspace(pda):
    size = pda.rms_norm_bwd_workspace_bytes
    assert size(0, 64, n_cu=256) == 0 and size(4, 64, n_cu=256) == 0 and size(4096, 1536, n_cu=256) > 0 and size(64, 64, groups=64, n_cu=256) == 0
    f = pda.lib.pda_rms_norm_bwd_workspace
    assert f(8, 1, 64, 256, None) == 1 and f(8, 1, 64, -1, C.byref(C.c_int64())) == 1 and f(8, 3, 64, 256, C.byref(C.c_int64())) == 1


def _struct(rot=64, layout=0, axes=1, pairs=(32, 0, 0, 0), freqs=True, positions=None, pos_batch=0, first=0, bad=None):
    from paper_2511_12056_amd.binding import RopeStruct
    f = (C.c_double * 64)(*[0.5] * 64)
    if bad is not None:
        f[3] = bad
    s = RopeStruct(rot, layout, axes, (C.c_int * 4)(*pairs), C.cast(f, C.POINTER(C.c_double)) if freqs else None, positions, pos_batch, first)
    s.keep = f
    return s


def _rope(pda, x=_addr(0), xt=1, xb=8 * 192, xtok=192, y=_addr(1), yb=3 * 8 * 64, yh=8 * 64, B=2, S=8, H=3, d=64, rope=None, rms=1, premul=1.0, **kw):
    return pda.lib.pda_pack_heads_rope(x, xt, xb, xtok, y, yb, yh, B, S, H, d, C.byref(_struct(**kw)) if rope is None else rope or None, rms, premul, None)


ROPE_BAD = [
    (dict(B=-1), 1, "negative"), (dict(d=96), 2, "head dim"), (dict(xt=2), 1, "x_type"), (dict(rope=False), 1, "null rope"), (dict(rot=4), 1, "rot"), (dict(rot=72), 1, "rot"),
    (dict(rot=-8), 1, "rot"), (dict(layout=2), 1, "layout"), (dict(axes=0), 1, "axes"), (dict(axes=5), 1, "axes"), (dict(pairs=(31, 0, 0, 0)), 1, "sum"),
    (dict(axes=2, pairs=(40, -8, 0, 0), positions=_addr(3)), 1, "negative"), (dict(freqs=False), 1, "null freqs"), (dict(bad=float("inf")), 1, "freqs[3]"),
    (dict(axes=2, pairs=(16, 16, 0, 0)), 1, "null positions"), (dict(first=-1), 1, "first"), (dict(positions=_addr(3) + 2), 2, "4-byte"),
    (dict(positions=_addr(3), pos_batch=-1), 1, "pos_batch"), (dict(premul=float("nan")), 1, "premul"), (dict(S=1 << 31), 2, "2^31"), (dict(H=1 << 24, S=1, B=1, xtok=1 << 30, yh=64), 2, "2^24"),
    (dict(x=None), 1, "null"), (dict(y=None), 1, "null"), (dict(xb=-8), 1, "stride of x"), (dict(xtok=196), 2, "strides of x"), (dict(yh=516), 2, "strides of y"),
    (dict(yh=-8), 1, "stride of y"), (dict(x=_addr(0) + 8), 2, "16-byte"), (dict(y=_addr(1) + 8), 2, "16-byte"), (dict(yh=504), 1, "heads of y"), (dict(yb=1024), 1, "batches of y"),
    (dict(y=_addr(0) + 1024), 1, "y overlaps x"), (dict(positions=_addr(1) + 64), 1, "y overlaps positions"), (dict(xtok=1 << 39, S=1 << 20, yh=1 << 26, yb=1 << 28), 2, "2^42"),
]


@pytest.mark.parametrize("change,code,word", ROPE_BAD)
def test_pack_heads_rope_refuses(pda, change, code, word):
    assert _rope(pda, **change) == code and word in pda.last_error(), pda.last_error()


def _rope_bwd(pda, dy=_addr(0), yb=3 * 8 * 64, yh=8 * 64, x=_addr(1), xt=0, xb=8 * 192, xtok=192, dx=_addr(2), db=8 * 192, dtok=192, B=2, S=8, H=3, d=64, rms=1, premul=1.0, **kw):
    return pda.lib.pda_pack_heads_rope_bwd(dy, yb, yh, x, xt, xb, xtok, dx, db, dtok, B, S, H, d, C.byref(_struct(**kw)), rms, premul, None)


@pytest.mark.parametrize("change,code,word", [
    (dict(d=32), 2, "head dim"), (dict(dy=None), 1, "null"), (dict(x=None), 1, "null"), (dict(dx=None), 1, "null"), (dict(dtok=184), 1, "tokens of dx overlap"),
    (dict(db=800), 1, "batches of dx overlap"), (dict(dx=_addr(1) + 64), 1, "dx overlaps x"), (dict(dx=_addr(1), dtok=200, db=1600), 1, "dx overlaps x"),
    (dict(dx=_addr(0)), 1, "dx overlaps dy"), (dict(dtok=194), 2, "strides of dx"), (dict(rot=20), 1, "rot"),
])
def test_pack_heads_rope_bwd_refuses(pda, change, code, word):
    assert _rope_bwd(pda, **change) == code and word in pda.last_error(), pda.last_error()


def test_rope_with_nothing_to_do(pda):
    assert _rope(pda, x=None, y=None, S=0) == 0 and _rope(pda, x=None, y=None, H=0) == 0 and _rope_bwd(pda, dy=None, x=None, dx=None, B=0) == 0


def test_frequencies(pda):
    n = 32
    plain, one = pda.rope_frequencies(n)
    assert one == 1.0 and all(abs(f - 10000.0 ** (-i / n)) < 1e-15 for i, f in enumerate(plain))
    assert all(abs(f - p / 4) < 1e-15 for f, p in zip(pda.rope_frequencies(n, scaling="linear", factor=4)[0], plain))
    base, _ = pda.rope_frequencies(n, scaling="base", factor=4)
    assert base[0] == 1.0 and abs(base[-1] / plain[-1] - 1 / 4) < 1e-12 and all(x > y for x, y in zip(base, base[1:]))
    blend, magnitude = pda.rope_frequencies(n, scaling="blend", factor=16, original=4096, slow_turns=1, fast_turns=32)
    assert abs(magnitude - (0.1 * math.log(16) + 1)) < 1e-15
    for f, p in zip(blend, plain):
        turns = 4096 * p / (2 * math.pi)
        keep = min(1, max(0, (turns - 1) / 31))
        assert abs(f - (p * keep + p / 16 * (1 - keep))) < 1e-15
    assert blend[0] == plain[0] and abs(blend[-1] - plain[-1] / 16) < 1e-18
    assert pda.rope_frequencies(1, scaling="base", factor=4)[0] == [1.0]


@pytest.mark.parametrize("kw", [dict(n=0), dict(n=4, base=1.0), dict(n=4, base=float("inf")), dict(n=4, scaling="linear", factor=0.5), dict(n=4, scaling="blend", factor=2, original=0),
                                dict(n=4, scaling="blend", factor=2, slow_turns=3, fast_turns=3), dict(n=4, scaling="base", factor=float("nan"))])
def test_frequencies_refuses(pda, kw):
    with pytest.raises(pda.PdaError):
        pda.rope_frequencies(**kw)


def test_rope_object_refuses(pda):
    for kw in (dict(freqs=[1.0] * 6), dict(freqs=[1.0] * 68), dict(freqs=[1.0] * 8, layout="other"), dict(freqs=[1.0] * 8, axis_pairs=[4, 3]),
               dict(freqs=[1.0] * 8, axis_pairs=[8, 0, 0, 0, 0]), dict(freqs=[1.0] * 8, axis_pairs=[9, -1])):
        with pytest.raises(ValueError):
            pda.Rope(**kw)
    with pytest.raises(ValueError):
        pda.rope_frequencies(4, scaling="other")
    assert pda.Rope([]).rot == 0


def test_wrappers_refuse_tensors_of_the_cpu(pda):
    import torch
    x = torch.zeros(2, 128)
    q, s = torch.zeros(2, 128, dtype=torch.float8_e4m3fn), torch.zeros(2, 4, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    with pytest.raises(ValueError):
        pda.fp8_quant(x, q, s)
    with pytest.raises(ValueError):
        pda.fp8_matmul(q, s, q, s, torch.zeros(2, 2, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        pda.rms_norm_fwd(x, None, x)
    with pytest.raises(ValueError):
        pda.pack_heads_rope(torch.zeros(1, 2, 1, 64), torch.zeros(1, 1, 2, 64, dtype=torch.bfloat16), pda.Rope([]))
