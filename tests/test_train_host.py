"""Host side of the training entry points: symbols, refusals and workspace sizes, without a GPU."""
import ctypes as C
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def pda():
    import paper_2511_12056_amd as pda
    return pda


def test_every_declared_symbol_is_exported(pda):
    text = open(os.path.join(ROOT, "include", "pipedit_train.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\bint (pda_[a-z0-9_]+)\s*\(", text)))
    assert names == ["pda_attn_bwd", "pda_attn_bwd_strided", "pda_attn_bwd_workspace", "pda_layer_norm_bwd",
                     "pda_layer_norm_bwd_workspace", "pda_layer_norm_fwd", "pda_pack_heads_bwd"]
    lib = C.CDLL(pda.lib_path())
    for n in names:
        assert getattr(lib, n) is not None


# Made-up device addresses, far apart; every call below fails its checks before one of them is used.
def _addr(i):
    return (i + 1) << 32


ATTN = dict(dout=_addr(0), q=_addr(1), k=_addr(2), v=_addr(3), out=_addr(4), out_type=0, lse=_addr(5), dq=_addr(6), dk=_addr(7), dv=_addr(8),
            B=1, H=2, Sq=8, Skv=8, d=64, scale=1.0, n_v=8, ws=_addr(9), ws_bytes=0)


def _bwd(pda, strides=None, **kw):
    a = dict(ATTN, **kw)
    head = [a[n] for n in ("dout", "q", "k", "v", "out", "out_type", "lse", "dq", "dk", "dv", "B", "H", "Sq", "Skv", "d")]
    tail = [a["scale"], a["n_v"], a["ws"], a["ws_bytes"], None]
    if strides is None:
        return pda.lib.pda_attn_bwd(*head, *tail)
    return pda.lib.pda_attn_bwd_strided(*head, strides and C.byref(strides), *tail)


@pytest.mark.parametrize("change,code,word", [
    (dict(d=32), 2, "head dim"), (dict(n_v=9), 1, "kv_valid_len"), (dict(n_v=-1), 1, "kv_valid_len"), (dict(Sq=-1), 1, "negative"),
    (dict(B=-1), 1, "negative"), (dict(scale=-0.5), 1, "scale"), (dict(scale=float("nan")), 1, "scale"), (dict(scale=float("inf")), 1, "scale"),
    (dict(out_type=2), 1, "out_type"), (dict(dout=None), 1, "null"), (dict(lse=None), 1, "null"), (dict(dq=None), 1, "null"),
    (dict(k=None), 1, "null"), (dict(dv=None), 1, "null"), (dict(q=_addr(1) + 8), 2, "16-byte"), (dict(dk=_addr(7) + 2), 2, "16-byte"),
    (dict(lse=_addr(5) + 2), 2, "4-byte"), (dict(B=70000), 2, "65535"), (dict(Sq=1 << 31), 2, "2^31"),
    (dict(H=60000, Sq=1 << 30, d=128), 2, "2^40"), (dict(dq=_addr(1)), 1, "dq overlaps q"), (dict(dk=_addr(7), dv=_addr(7) + 16), 1, "dv overlaps dk"),
    (dict(dq=_addr(4) + 2 * 8 * 64 * 4 - 16), 1, "dq overlaps out"), (dict(ws=None), 1, "workspace"), (dict(ws_bytes=64), 1, "workspace"),
    (dict(ws=_addr(9) + 16, ws_bytes=1 << 40), 2, "256-byte"),
])
def test_attn_bwd_refuses(pda, change, code, word):
    assert _bwd(pda, **change) == code and word in pda.last_error(), pda.last_error()


def test_attn_bwd_with_nothing_to_do(pda):
    none = dict(dout=None, q=None, k=None, v=None, out=None, lse=None, dq=None, dk=None, dv=None, ws=None)
    assert _bwd(pda, **none, B=0) == 0 and _bwd(pda, **none, H=0) == 0 and _bwd(pda, **none, Sq=0, Skv=0, n_v=0) == 0


def _strides(pda, **kw):
    from paper_2511_12056_amd.binding import AttnBwdStrides
    s = AttnBwdStrides(*([2 * 8 * 64, 8 * 64] * 4 + [16, 8] + [2 * 8 * 64, 8 * 64] * 2))
    for n, x in kw.items():
        setattr(s, n, x)
    return s


@pytest.mark.parametrize("change,kw,code,word", [
    (dict(q_head=-8), {}, 1, "stride"), (dict(kv_batch=1 << 40), {}, 1, "stride"), (dict(dout_head=8 * 64 + 4), {}, 2, "multiples of 8"),
    (dict(out_head=514), {}, 2, "16 bytes"), (dict(out_head=516), dict(out_type=1), 2, "16 bytes"), (dict(dq_head=504), {}, 1, "heads of dq"),
    (dict(dkv_head=504), {}, 1, "heads of dk/dv"), (dict(dq_batch=1016), dict(B=2), 1, "batches of dq"), (dict(dkv_batch=0), dict(B=2), 1, "batches of dk/dv"),
    ({}, dict(dk=_addr(8)), 1, "overlaps"), ({}, dict(d=96), 2, "head dim"), ({}, dict(out_type=7), 1, "out_type"),
])
def test_attn_bwd_strided_refuses(pda, change, kw, code, word):
    assert _bwd(pda, strides=_strides(pda, **change), **kw) == code and word in pda.last_error(), pda.last_error()


def test_attn_bwd_strided_refuses_no_strides(pda):
    a = [ATTN[n] for n in ("dout", "q", "k", "v", "out", "out_type", "lse", "dq", "dk", "dv", "B", "H", "Sq", "Skv", "d")]
    assert pda.lib.pda_attn_bwd_strided(*a, None, 1.0, 8, ATTN["ws"], 0, None) == 1 and "strides" in pda.last_error()


def test_attn_bwd_workspace(pda):
    size = pda.attn_bwd_workspace_bytes
    for a in ((1, 2, 1024, 1024, 64, 1024), (1, 24, 9600, 9600, 128, 9600), (2, 3, 1, 1, 64, 1), (1, 1, 100000, 70, 128, 3)):
        n = size(*a, n_cu=256)
        assert n >= a[0] * a[1] * a[2] * 8 and n % 256 == 0
    assert size(1, 2, 0, 0, 64, n_cu=256) == 0
    f = pda.lib.pda_attn_bwd_workspace
    assert f(1, 1, 8, 8, 64, 8, 256, None) == 1 and f(1, 1, 8, 8, 64, 8, -1, C.byref(C.c_int64())) == 1
    assert f(1, 1, 8, 8, 80, 8, 256, C.byref(C.c_int64())) == 2 and f(1, 1, -8, 8, 64, 8, 256, C.byref(C.c_int64())) == 1


def _ln(pda, x=_addr(0), x_type=0, w=_addr(1), b=_addr(2), y=_addr(3), y_type=1, mean=_addr(4), rstd=_addr(5), rows=8, groups=1, D=64, eps=1e-6):
    return pda.lib.pda_layer_norm_fwd(x, x_type, w, b, y, y_type, mean, rstd, rows, groups, D, eps, None)


@pytest.mark.parametrize("change,code,word", [
    (dict(x_type=2), 1, "type"), (dict(y_type=-1), 1, "type"), (dict(rows=-1), 1, "rows"), (dict(groups=0), 1, "groups"), (dict(groups=3), 1, "multiple"),
    (dict(D=0), 1, "D=0"), (dict(D=8193), 2, "MAX"), (dict(rows=70000, groups=70000), 2, "65535"), (dict(rows=1 << 31), 2, "2^31"),
    (dict(eps=-1.0), 1, "eps"), (dict(eps=float("nan")), 1, "eps"), (dict(mean=None), 1, "together"), (dict(rstd=None), 1, "together"),
    (dict(x=None), 1, "null"), (dict(y=None), 1, "null"), (dict(x=_addr(0) + 8), 2, "16-byte"), (dict(b=_addr(2) + 4), 2, "16-byte"),
    (dict(mean=_addr(4) + 2), 2, "4-byte"), (dict(y=_addr(0)), 1, "overlaps"), (dict(y=_addr(0) + 64, y_type=0), 1, "overlaps"),
])
def test_layer_norm_fwd_refuses(pda, change, code, word):
    assert _ln(pda, **change) == code and word in pda.last_error(), pda.last_error()


def test_layer_norm_with_nothing_to_do(pda):
    assert _ln(pda, x=None, y=None, w=None, b=None, mean=None, rstd=None, rows=0) == 0
    assert _ln_bwd(pda, dw=None, db=None, rows=0) == 0


def _ln_bwd(pda, dy=_addr(0), y_type=1, x=_addr(1), x_type=0, w=_addr(2), mean=_addr(3), rstd=_addr(4), dx=_addr(5), dw=_addr(6), db=_addr(7),
            rows=8, groups=1, D=64):
    return pda.lib.pda_layer_norm_bwd(dy, y_type, x, x_type, w, mean, rstd, dx, dw, db, rows, groups, D, None, 0, None)


@pytest.mark.parametrize("change,code,word", [
    (dict(x_type=2), 1, "type"), (dict(rows=-1), 1, "rows"), (dict(rows=9, groups=2), 1, "multiple"), (dict(D=9000), 2, "MAX"),
    (dict(dx=None, dw=None, db=None), 1, "nothing"), (dict(dy=None), 1, "null"), (dict(rstd=None), 1, "null"), (dict(dw=_addr(6) + 4), 2, "16-byte"),
    (dict(dx=_addr(5) + 4), 2, "16-byte"), (dict(mean=_addr(3) + 1), 2, "4-byte"), (dict(dx=_addr(0)), 1, "dx overlaps dy"), (dict(dx=_addr(1) + 32), 1, "dx overlaps x"),
])
def test_layer_norm_bwd_refuses(pda, change, code, word):
    assert _ln_bwd(pda, **change) == code and word in pda.last_error(), pda.last_error()


def test_layer_norm_bwd_workspace(pda):
    size = pda.layer_norm_bwd_workspace_bytes
    assert size(0, 64, n_cu=256) == 0 and size(4, 64, n_cu=256) == 0 and size(4096, 1536, n_cu=256) > 0
    assert size(64, 64, groups=64, n_cu=256) == 0                  # one row a group
    f = pda.lib.pda_layer_norm_bwd_workspace
    assert f(8, 1, 64, 256, None) == 1 and f(8, 1, 64, -1, C.byref(C.c_int64())) == 1 and f(8, 3, 64, 256, C.byref(C.c_int64())) == 1


def _pack(pda, dy=_addr(0), x=_addr(1), dx=_addr(2), B=1, S=8, H=2, d=64, rms=1, premul=1.0):
    return pda.lib.pda_pack_heads_bwd(dy, x, dx, B, S, H, d, rms, premul, None)


@pytest.mark.parametrize("change,code,word", [
    (dict(B=-1), 1, "negative"), (dict(d=96), 2, "head dim"), (dict(S=1 << 40), 2, "2^40"), (dict(dy=None), 1, "null"), (dict(x=None), 1, "null"),
    (dict(dx=None), 1, "null"), (dict(dy=_addr(0) + 8), 2, "16-byte"), (dict(dx=_addr(0) + 1024), 1, "dx overlaps dy"), (dict(dx=_addr(1) + 16), 1, "dx overlaps x"),
    (dict(premul=float("inf")), 1, "premul"),
])
def test_pack_heads_bwd_refuses(pda, change, code, word):
    assert _pack(pda, **change) == code and word in pda.last_error(), pda.last_error()


def test_pack_heads_bwd_with_nothing_to_do(pda):
    assert _pack(pda, dy=None, x=None, dx=None, S=0) == 0 and _pack(pda, dy=None, x=None, dx=None, B=0) == 0


def test_binding_checks_tensors(pda):
    import torch
    t = torch.zeros(1, 1, 8, 64, dtype=torch.bfloat16)
    lse = torch.zeros(1, 1, 8)
    with pytest.raises(ValueError):
        pda.attn_bwd(t, t, t, t, t, lse, t, t, t, 1.0)             # not on the GPU
    with pytest.raises(ValueError):
        pda.attn_bwd_strided(t, t, t, t, t.double(), lse, t, t, t, 1.0)
    with pytest.raises(ValueError):
        pda.layer_norm_fwd(torch.zeros(4, 8), None, None, torch.zeros(4, 8))
    with pytest.raises(ValueError):
        pda.layer_norm_bwd(torch.zeros(4, 8), torch.zeros(4, 8), None, torch.zeros(4), torch.zeros(4), None, None, None)
    with pytest.raises(ValueError):
        pda.pack_heads_bwd(t, None, torch.zeros(1, 8, 1, 64), False)


@pytest.mark.parametrize("change,word", [
    (dict(y=_addr(1)), "y overlaps weight"), (dict(b=_addr(3) + 1008), "y overlaps bias"), (dict(mean=_addr(0)), "mean overlaps x"),
    (dict(rstd=_addr(3) + 1020), "rstd overlaps y"), (dict(rstd=_addr(4) + 28), "mean overlaps rstd"), (dict(mean=_addr(1) + 252), "mean overlaps weight"),
])
def test_layer_norm_fwd_refuses_results_over_other_tensors(pda, change, word):
    assert _ln(pda, **change) == 1 and word in pda.last_error(), pda.last_error()


@pytest.mark.parametrize("change,word", [         # 8 rows of 64: dy 1024 bytes, dx 2048, mean and rstd 32, the parameters 256
    (dict(dw=_addr(2)), "dweight overlaps weight"), (dict(db=_addr(3) + 16), "dbias overlaps mean"), (dict(dw=_addr(0) + 1008), "dweight overlaps dy"),
    (dict(db=_addr(5)), "dbias overlaps dx"), (dict(db=_addr(6) + 240), "dbias overlaps dweight"), (dict(dx=_addr(4) - 2032), "dx overlaps rstd"),
])
def test_layer_norm_bwd_refuses_results_over_other_tensors(pda, change, word):
    assert _ln_bwd(pda, **change) == 1 and word in pda.last_error(), pda.last_error()


def test_attn_bwd_refuses_a_workspace_over_a_tensor(pda):
    for i in range(9):
        assert _bwd(pda, ws=_addr(i), ws_bytes=1 << 20) == 1 and "workspace overlaps" in pda.last_error(), pda.last_error()


class _Elsewhere:
    """What the wrappers ask of a tensor, of one on device 1."""
    is_cuda = True
    device = 1

    def __init__(self, dtype, *shape):
        import torch
        self.dtype, self.shape = dtype, torch.Size(shape)

    def is_contiguous(self):
        return True

    def stride(self):
        return [int(self.shape[i + 1:].numel()) for i in range(len(self.shape))]

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def get_device(self):
        return self.device

    def data_ptr(self):
        raise AssertionError("its address was asked for")


def test_tensors_of_another_device_are_refused(pda, monkeypatch):
    import torch
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    bf16, fp32 = torch.bfloat16, torch.float32
    q, lse = _Elsewhere(bf16, 1, 2, 8, 64), _Elsewhere(fp32, 1, 2, 8)
    x, w, s = _Elsewhere(fp32, 8, 64), _Elsewhere(fp32, 64), _Elsewhere(fp32, 8)
    for call in (lambda: pda.attn_bwd(q, q, q, q, q, lse, q, q, q, 1.0), lambda: pda.attn_bwd_strided(q, q, q, q, q, lse, q, q, q, 1.0),
                 lambda: pda.layer_norm_fwd(x, w, w, x, s, s), lambda: pda.layer_norm_bwd(x, x, w, s, s, x, w, w),
                 lambda: pda.pack_heads_bwd(q, None, _Elsewhere(fp32, 1, 8, 2, 64), False)):
        with pytest.raises(ValueError, match="device 1, the current device is 0"):
            call()


def test_layer_norm_parameters_that_do_not_fit(pda, monkeypatch):
    import torch
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    f32 = torch.float32
    x, y, s, w = _Elsewhere(f32, 8, 64), _Elsewhere(f32, 8, 64), _Elsewhere(f32, 8), _Elsewhere(f32, 64)
    for bad in (_Elsewhere(f32, 0, 64), _Elsewhere(f32, 32), _Elsewhere(f32, 1, 1, 64), _Elsewhere(torch.bfloat16, 64), _Elsewhere(f32)):
        with pytest.raises(ValueError, match="weight"):
            pda.layer_norm_fwd(x, bad, None, y)
    for call in (lambda: pda.layer_norm_fwd(x, _Elsewhere(f32, 2, 64), w, y), lambda: pda.layer_norm_bwd(y, x, _Elsewhere(f32, 2, 64), s, s, x, w, None)):
        with pytest.raises(ValueError, match="1 groups, another parameter has 2"):
            call()
    for call in (lambda: pda.layer_norm_fwd(x, w, w, y, w, w), lambda: pda.layer_norm_fwd(x, w, w, y, s, _Elsewhere(torch.bfloat16, 8))):
        with pytest.raises(ValueError, match="one entry per row"):
            call()
