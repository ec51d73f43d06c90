"""ctypes binding of libpipedit_attn: same names as the C entry points, argument marshalling only.

Tensors are torch tensors on the GPU (torch is used for device memory and
streams); the binding passes raw device pointers and sizes across the C ABI.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libpipedit_attn.so")

PDA_OK, PDA_ERR_INVALID_ARG, PDA_ERR_UNSUPPORTED, PDA_ERR_HIP, PDA_ERR_NOMEM = 0, 1, 2, 3, 4
PDA_MAX_PARTIALS = 16
PDA_NOALLOC_MAX_SLOTS = 576
PDA_MAX_KEY_RANGES = 16
PDA_MAX_LOCAL_HEADS = 64
PDA_SINK_HEAD_MAJOR, PDA_SINK_TOKEN_ARRIVAL, PDA_SINK_TOKEN_FINAL = 0, 1, 2
PDA_F32, PDA_BF16, PDA_E4M3, PDA_E5M2 = 0, 1, 2, 3
PDA_LAYER_NORM_MAX = 8192
PDA_ANY_LEN = -1
PDA_ROPE_MAX_AXES = 4
ROPE_LAYOUTS = {"interleaved": 0, "half": 1}
ROPE_SCALINGS = {"plain": 0, "linear": 1, "base": 2, "blend": 3}


class AttnBwdStrides(C.Structure):
    """pda_attn_bwd_strides: batch and head strides in elements."""
    _fields_ = [(n + "_" + a, C.c_int64) for n in ("dout", "q", "kv", "out", "lse", "dq", "dkv") for a in ("batch", "head")]


class RopeStruct(C.Structure):
    """pda_rope."""
    _fields_ = [("rot", C.c_int), ("layout", C.c_int), ("axes", C.c_int), ("axis_pairs", C.c_int * PDA_ROPE_MAX_AXES),
                ("freqs", C.POINTER(C.c_double)), ("positions", C.c_void_p), ("pos_batch", C.c_int64), ("first", C.c_int64)]


class PdaError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"libpipedit_attn error {code}: {message}")
        self.code = code


def lib_path() -> str:
    return _LIB_PATH


def _load() -> C.CDLL:
    if not os.path.exists(_LIB_PATH):
        raise ImportError(
            f"{_LIB_PATH} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()' "
            "or python paper_2511_12056_amd/build.py). There is no fallback path.")
    lib = C.CDLL(_LIB_PATH)
    vp, fp, i32, i64, f32 = C.c_void_p, C.c_void_p, C.c_int, C.c_int64, C.c_float
    lib.pda_attn_fwd.argtypes = [vp, vp, vp, fp, fp, i32, i32, i64, i64, i32, f32, i64, i64, vp]
    lib.pda_attn_fwd.restype = i32
    lib.pda_attn_fwd_strided.argtypes = [vp, vp, vp, fp, fp, i32, i32, i64, i64, i32] + [i64] * 8 + [f32, i64, i64, vp]
    lib.pda_attn_fwd_strided.restype = i32
    lib.pda_attn_fwd_noalloc.argtypes = [vp, vp, vp, fp, fp, i32, i32, i64, i64, i32, f32, i64, i64, vp]
    lib.pda_attn_fwd_noalloc.restype = i32
    lib.pda_attn_fwd_variant.argtypes = [vp, vp, vp, fp, fp, i32, i32, i64, i64, i32, f32, i64, i32, vp]
    lib.pda_attn_fwd_variant.restype = i32
    lib.pda_attn_tail_plan.argtypes = [i32, i32, i64, i64, i32, i32, C.POINTER(i64), C.POINTER(i64), C.POINTER(i32),
                                       C.POINTER(i64), C.POINTER(i64)]
    lib.pda_attn_tail_plan.restype = i32
    lib.pda_attn_merge.argtypes = [C.POINTER(vp), C.POINTER(vp), i32, fp, fp, i64, i32, vp]
    lib.pda_attn_merge.restype = i32
    lib.pda_headchunk_run.argtypes = [vp, vp, vp, fp, fp, i32, i32, i64, i64, i32, f32, i64, i32, vp, vp, fp,
                                      C.POINTER(f32), C.POINTER(f32)]
    lib.pda_headchunk_run.restype = i32
    lib.pda_headchunk_run_ex.argtypes = [vp, vp, vp, fp, fp, i32, i32, i64, i64, i32, f32, i64, C.POINTER(i32), i32,
                                         i32, i32, vp, vp, fp, C.POINTER(f32), C.POINTER(f32)]
    lib.pda_headchunk_run_ex.restype = i32
    lib.pda_pipesp_postprocess.argtypes = [C.POINTER(vp), i32, i32, i64, fp, i64, i32, vp]
    lib.pda_pipesp_postprocess.restype = i32
    lib.pda_pack_heads.argtypes = [fp, vp, i32, i64, i32, i32, i32, f32, vp]
    lib.pda_attn_fwd_bf16out.argtypes = [vp, vp, vp, vp, fp, i32, i32, i64, i64, i32, f32, i64, vp]
    lib.pda_attn_fwd_bf16out.restype = i32
    lib.pda_attn_fwd_base2.argtypes = [vp, vp, vp, fp, fp, i32, i32, i64, i64, i32, i64, vp]
    lib.pda_attn_fwd_base2.restype = i32
    lib.pda_pack_heads.restype = i32
    f64 = C.c_double
    lib.pda_plan_n_decode.argtypes = [f64, f64, i32, C.POINTER(i32)]
    lib.pda_plan_n_decode.restype = i32
    lib.pda_plan_aco.argtypes = [f64, f64, i32, i32, C.POINTER(f64), C.POINTER(f64), C.POINTER(f64)]
    lib.pda_plan_aco.restype = i32
    lib.pda_plan_head_padding.argtypes = [i32, i32, C.POINTER(i32), C.POINTER(i32), C.POINTER(i32)]
    lib.pda_plan_head_padding.restype = i32
    lib.pda_plan_ragged_groups.argtypes = [i32, i32, C.POINTER(i32)]
    lib.pda_plan_ragged_groups.restype = i32
    lib.pda_probe_mfma_rate.argtypes = [vp, i64, i64, C.POINTER(f32), C.POINTER(f32), vp]
    lib.pda_probe_mfma_rate.restype = i32
    lib.pda_probe_loop_rate.argtypes = [vp, i64, i64, i32, C.POINTER(f32), C.POINTER(f32), vp]
    lib.pda_probe_loop_rate.restype = i32
    lib.pda_attn_bwd.argtypes = [vp] * 5 + [i32, fp, vp, vp, vp, i32, i32, i64, i64, i32, f32, i64, vp, i64, vp]
    lib.pda_attn_bwd.restype = i32
    lib.pda_attn_bwd_strided.argtypes = [vp] * 5 + [i32, fp, vp, vp, vp, i32, i32, i64, i64, i32, C.POINTER(AttnBwdStrides), f32, i64, vp, i64, vp]
    lib.pda_attn_bwd_strided.restype = i32
    lib.pda_attn_bwd_workspace.argtypes = [i32, i32, i64, i64, i32, i64, i32, C.POINTER(i64)]
    lib.pda_attn_bwd_workspace.restype = i32
    lib.pda_layer_norm_fwd.argtypes = [vp, i32, fp, fp, vp, i32, fp, fp, i64, i64, i32, f32, vp]
    lib.pda_layer_norm_fwd.restype = i32
    lib.pda_layer_norm_bwd.argtypes = [vp, i32, vp, i32, fp, fp, fp, vp, fp, fp, i64, i64, i32, vp, i64, vp]
    lib.pda_layer_norm_bwd.restype = i32
    lib.pda_layer_norm_bwd_workspace.argtypes = [i64, i64, i32, i32, C.POINTER(i64)]
    lib.pda_layer_norm_bwd_workspace.restype = i32
    lib.pda_pack_heads_bwd.argtypes = [vp, fp, fp, i32, i64, i32, i32, i32, f32, vp]
    lib.pda_pack_heads_bwd.restype = i32
    lib.pda_fp8_quant.argtypes = [vp, i32, i64, i64, i64, i32, i32, vp, vp, vp, vp, vp]
    lib.pda_fp8_quant.restype = i32
    lib.pda_fp8_matmul.argtypes = [vp, i32, vp, vp, vp, i32, fp, vp, i64, i64, i64, i64, vp, i64, vp]
    lib.pda_fp8_matmul.restype = i32
    lib.pda_fp8_matmul_workspace.argtypes = [i64, i64, i64, i32, C.POINTER(i64)]
    lib.pda_fp8_matmul_workspace.restype = i32
    lib.pda_rms_norm_fwd.argtypes = [vp, i32, vp, i32, fp, vp, vp, i32, vp, fp, i64, i64, i32, f32, vp]
    lib.pda_rms_norm_fwd.restype = i32
    lib.pda_rms_norm_bwd.argtypes = [vp, i32, vp, i32, fp, fp, vp, vp, fp, i64, i64, i32, vp, i64, vp]
    lib.pda_rms_norm_bwd.restype = i32
    lib.pda_rms_norm_bwd_workspace.argtypes = [i64, i64, i32, i32, C.POINTER(i64)]
    lib.pda_rms_norm_bwd_workspace.restype = i32
    lib.pda_pack_heads_rope.argtypes = [vp, i32, i64, i64, vp, i64, i64, i32, i64, i32, i32, C.POINTER(RopeStruct), i32, f32, vp]
    lib.pda_pack_heads_rope.restype = i32
    lib.pda_pack_heads_rope_bwd.argtypes = [vp, i64, i64, vp, i32, i64, i64, vp, i64, i64, i32, i64, i32, i32, C.POINTER(RopeStruct), i32, f32, vp]
    lib.pda_pack_heads_rope_bwd.restype = i32
    lib.pda_rope_frequencies.argtypes = [i32, f64, i32, f64, f64, f64, f64, C.POINTER(f64), C.POINTER(f64)]
    lib.pda_rope_frequencies.restype = i32
    lib.pda_last_error.argtypes = []
    lib.pda_last_error.restype = C.c_char_p
    lib.pda_version.argtypes = []
    lib.pda_version.restype = i32
    return lib


lib = _load()


def last_error() -> str:
    return lib.pda_last_error().decode()


def version() -> int:
    return lib.pda_version()


def _check(rc: int) -> None:
    if rc != PDA_OK:
        raise PdaError(rc, last_error())


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream_handle(stream) -> Optional[int]:
    if stream is None:
        # The handle without the Stream object around it: a call on a short sequence is bound by host time, and
        # torch.cuda.current_stream() was 3.0 of its 14 us (2 x 1 024, d = 64), the tensor checks 2.8.
        import torch
        raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
        if raw is not None and device is not None and torch.cuda.is_initialized():     # neither is a public name
            return raw(device()) or None
        stream = torch.cuda.current_stream()
    return stream.cuda_stream or None


def _expect(t, dtype, shape, name):
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or not t.is_cuda:
        raise ValueError(f"{name}: expected contiguous cuda {dtype} of shape {tuple(shape)}, "
                         f"got {t.dtype} {tuple(t.shape)} contiguous={t.is_contiguous()} cuda={t.is_cuda}")


def attn_fwd(q, k, v, out, lse, scale: float, kv_valid_len: Optional[int] = None, q_offset: int = 0, stream=None):
    """pda_attn_fwd: q [B,H,Sq,d] bf16, k/v [B,H,Skv,d] bf16 -> out [B,H,Sq,d] fp32, lse [B,H,Sq] fp32."""
    import torch
    B, H, Sq, d = q.shape
    Skv = k.shape[2]
    _expect(q, torch.bfloat16, (B, H, Sq, d), "q")
    _expect(k, torch.bfloat16, (B, H, Skv, d), "k")
    _expect(v, torch.bfloat16, (B, H, Skv, d), "v")
    _expect(out, torch.float32, (B, H, Sq, d), "out")
    _expect(lse, torch.float32, (B, H, Sq), "lse")
    n_v = Skv if kv_valid_len is None else int(kv_valid_len)
    _check(lib.pda_attn_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), B, H, Sq, Skv, d, float(scale),
                            n_v, int(q_offset), _stream_handle(stream)))
    return out, lse


def attn_fwd_noalloc(q, k, v, out, lse, scale: float, kv_valid_len: Optional[int] = None, q_offset: int = 0, stream=None):
    """pda_attn_fwd_noalloc: attn_fwd with the partials of cut tiles in the library's static device buffer."""
    import torch
    B, H, Sq, d = q.shape
    Skv = k.shape[2]
    _expect(q, torch.bfloat16, (B, H, Sq, d), "q")
    _expect(k, torch.bfloat16, (B, H, Skv, d), "k")
    _expect(v, torch.bfloat16, (B, H, Skv, d), "v")
    _expect(out, torch.float32, (B, H, Sq, d), "out")
    _expect(lse, torch.float32, (B, H, Sq), "lse")
    n_v = Skv if kv_valid_len is None else int(kv_valid_len)
    _check(lib.pda_attn_fwd_noalloc(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), B, H, Sq, Skv, d, float(scale),
                                    n_v, int(q_offset), _stream_handle(stream)))
    return out, lse


def attn_fwd_variant(q, k, v, out, lse, scale: float, variant: int, kv_valid_len: Optional[int] = None, stream=None):
    """pda_attn_fwd_variant: attn_fwd with an explicit kernel choice (testing aid)."""
    import torch
    B, H, Sq, d = q.shape
    Skv = k.shape[2]
    _expect(q, torch.bfloat16, (B, H, Sq, d), "q")
    _expect(k, torch.bfloat16, (B, H, Skv, d), "k")
    _expect(v, torch.bfloat16, (B, H, Skv, d), "v")
    _expect(out, torch.float32, (B, H, Sq, d), "out")
    _expect(lse, torch.float32, (B, H, Sq), "lse")
    n_v = Skv if kv_valid_len is None else int(kv_valid_len)
    _check(lib.pda_attn_fwd_variant(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), B, H, Sq, Skv, d, float(scale),
                                    n_v, int(variant), _stream_handle(stream)))
    return out, lse


def attn_tail_plan(B: int, H: int, Sq: int, kv_valid_len: int, d: int, n_cu: int = 0):
    """pda_attn_tail_plan: dict(n_tiles, n_cut, split, part_offsets, workspace_slots); part_offsets lists the
    split + 1 boundaries of the key ranges of a cut tile ([] if nothing is cut); n_cu = 0 asks the current device."""
    a, b, c, f = C.c_int64(0), C.c_int64(0), C.c_int(0), C.c_int64(0)
    offs = (C.c_int64 * (PDA_MAX_KEY_RANGES + 1))()
    _check(lib.pda_attn_tail_plan(int(B), int(H), int(Sq), int(kv_valid_len), int(d), int(n_cu),
                                  C.byref(a), C.byref(b), C.byref(c), offs, C.byref(f)))
    return {"n_tiles": a.value, "n_cut": b.value, "split": c.value,
            "part_offsets": [offs[j] for j in range(c.value + 1)] if c.value > 1 else [], "workspace_slots": f.value}


def attn_fwd_bf16out(q, k, v, out, lse, scale: float, kv_valid_len: Optional[int] = None, stream=None):
    """pda_attn_fwd_bf16out: as attn_fwd with out [B,H,Sq,d] in bf16."""
    import torch
    B, H, Sq, d = q.shape
    Skv = k.shape[2]
    _expect(q, torch.bfloat16, (B, H, Sq, d), "q")
    _expect(k, torch.bfloat16, (B, H, Skv, d), "k")
    _expect(v, torch.bfloat16, (B, H, Skv, d), "v")
    _expect(out, torch.bfloat16, (B, H, Sq, d), "out")
    _expect(lse, torch.float32, (B, H, Sq), "lse")
    n_v = Skv if kv_valid_len is None else int(kv_valid_len)
    _check(lib.pda_attn_fwd_bf16out(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), B, H, Sq, Skv, d, float(scale),
                                    n_v, _stream_handle(stream)))
    return out, lse


def attn_fwd_base2(q, k, v, out, lse, kv_valid_len: Optional[int] = None, stream=None):
    """pda_attn_fwd_base2: as attn_fwd with the scores q.k already in log2 units (weights 2^(q.k))."""
    import torch
    B, H, Sq, d = q.shape
    Skv = k.shape[2]
    _expect(q, torch.bfloat16, (B, H, Sq, d), "q")
    _expect(k, torch.bfloat16, (B, H, Skv, d), "k")
    _expect(v, torch.bfloat16, (B, H, Skv, d), "v")
    _expect(out, torch.float32, (B, H, Sq, d), "out")
    _expect(lse, torch.float32, (B, H, Sq), "lse")
    n_v = Skv if kv_valid_len is None else int(kv_valid_len)
    _check(lib.pda_attn_fwd_base2(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), B, H, Sq, Skv, d, n_v,
                                  _stream_handle(stream)))
    return out, lse


def _view_strides(t, inner, name):
    """(batch stride, head stride) of a [B,H,S,...] view whose rows are compact."""
    if not t.is_cuda:
        raise ValueError(f"{name}: expected a cuda tensor")
    st = t.stride()
    if inner == 2 and (st[3] != 1 or st[2] != t.shape[3]):
        raise ValueError(f"{name}: rows must be compact (stride {st})")
    if inner == 1 and st[2] != 1:
        raise ValueError(f"{name}: rows must be compact (stride {st})")
    return int(st[0]), int(st[1])


def attn_fwd_strided(q, k, v, out, lse, scale: float, kv_valid_len: Optional[int] = None, q_offset: int = 0, stream=None):
    """pda_attn_fwd_strided: as attn_fwd, on [B,H,S,d] VIEWS (e.g. x[:, :, a:b]) with compact rows; no copies."""
    import torch
    B, H, Sq, d = q.shape
    Skv = k.shape[2]
    if q.dtype != torch.bfloat16 or k.dtype != torch.bfloat16 or v.dtype != torch.bfloat16:
        raise ValueError("q/k/v: expected bf16")
    if out.dtype != torch.float32 or lse.dtype != torch.float32:
        raise ValueError("out/lse: expected fp32")
    if tuple(k.shape) != (B, H, Skv, d) or tuple(v.shape) != (B, H, Skv, d) or tuple(out.shape) != (B, H, Sq, d) \
            or tuple(lse.shape) != (B, H, Sq):
        raise ValueError("shape mismatch")
    qs, ks, vs, os_, ls = (_view_strides(q, 2, "q"), _view_strides(k, 2, "k"), _view_strides(v, 2, "v"),
                           _view_strides(out, 2, "out"), _view_strides(lse, 1, "lse"))
    if ks != vs:
        raise ValueError("k and v must share their strides")
    n_v = Skv if kv_valid_len is None else int(kv_valid_len)
    _check(lib.pda_attn_fwd_strided(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), B, H, Sq, Skv, d,
                                    qs[0], qs[1], ks[0], ks[1], os_[0], os_[1], ls[0], ls[1],
                                    float(scale), n_v, int(q_offset), _stream_handle(stream)))
    return out, lse


def attn_merge(partials: Sequence, lses: Sequence, out, lse_out=None, stream=None):
    """pda_attn_merge: partials n x [rows,d] fp32, lses n x [rows] fp32 -> out [rows,d] (+ lse_out [rows])."""
    import torch
    n = len(partials)
    if len(lses) != n:
        raise ValueError("partials and lses differ in length")
    d = out.shape[-1]
    rows = out.numel() // d if d else 0
    for i, (pt, lt) in enumerate(zip(partials, lses)):
        if pt.dtype != torch.float32 or lt.dtype != torch.float32 or not pt.is_contiguous() or not lt.is_contiguous():
            raise ValueError(f"partial {i}: expected contiguous fp32")
        if pt.numel() != rows * d or lt.numel() != rows:
            raise ValueError(f"partial {i}: size mismatch")
    if lse_out is not None and (lse_out.dtype != torch.float32 or lse_out.numel() != rows):
        raise ValueError("lse_out: expected fp32 with one entry per row")
    arr_p = (C.c_void_p * max(n, 1))(*[pt.data_ptr() for pt in partials])
    arr_l = (C.c_void_p * max(n, 1))(*[lt.data_ptr() for lt in lses])
    _check(lib.pda_attn_merge(arr_p, arr_l, n, _ptr(out), _ptr(lse_out), rows, d, _stream_handle(stream)))
    return out, lse_out


def headchunk_run(q, k, v, out, lse, scale: float, heads_per_group: int, compute_stream, drain_stream,
                  kv_valid_len: Optional[int] = None, sink=None, timed: bool = False):
    """pda_headchunk_run.  Returns (group_ms list, total_ms) when timed, else None (caller syncs both streams)."""
    import torch
    B, H, Sq, d = q.shape
    Skv = k.shape[2]
    _expect(q, torch.bfloat16, (B, H, Sq, d), "q")
    _expect(k, torch.bfloat16, (B, H, Skv, d), "k")
    _expect(v, torch.bfloat16, (B, H, Skv, d), "v")
    _expect(out, torch.float32, (B, H, Sq, d), "out")
    _expect(lse, torch.float32, (B, H, Sq), "lse")
    if sink is not None:
        _expect(sink, torch.float32, (B, H, Sq, d), "sink")
    n_v = Skv if kv_valid_len is None else int(kv_valid_len)
    n_groups = (H + heads_per_group - 1) // heads_per_group if heads_per_group > 0 and H > 0 else 0
    gms = (C.c_float * max(n_groups, 1))() if timed else None
    tms = C.c_float(0.0) if timed else None
    _check(lib.pda_headchunk_run(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), B, H, Sq, Skv, d, float(scale),
                                 n_v, int(heads_per_group), _stream_handle(compute_stream),
                                 _stream_handle(drain_stream), _ptr(sink),
                                 gms if timed else None, C.byref(tms) if timed else None))
    if timed:
        return [gms[i] for i in range(n_groups)], tms.value
    return None


def headchunk_run_ex(q, k, v, out, lse, scale: float, group_sizes: Sequence[int], compute_stream, drain_stream,
                     kv_valid_len: Optional[int] = None, sink=None, sp_ranks: int = 1,
                     sink_layout: int = PDA_SINK_HEAD_MAJOR, timed: bool = False):
    """pda_headchunk_run_ex.  sink is [B,H,Sq,d] (head-major layout) or [B,Sq,H,d] (token-major layouts)."""
    import torch
    B, H, Sq, d = q.shape
    Skv = k.shape[2]
    _expect(q, torch.bfloat16, (B, H, Sq, d), "q")
    _expect(k, torch.bfloat16, (B, H, Skv, d), "k")
    _expect(v, torch.bfloat16, (B, H, Skv, d), "v")
    _expect(out, torch.float32, (B, H, Sq, d), "out")
    _expect(lse, torch.float32, (B, H, Sq), "lse")
    if sink is not None:
        _expect(sink, torch.float32, (B, H, Sq, d) if sink_layout == PDA_SINK_HEAD_MAJOR else (B, Sq, H, d), "sink")
    n_v = Skv if kv_valid_len is None else int(kv_valid_len)
    n_groups = len(group_sizes)
    sizes = (C.c_int * max(n_groups, 1))(*[int(x) for x in group_sizes])
    gms = (C.c_float * max(n_groups, 1))() if timed else None
    tms = C.c_float(0.0) if timed else None
    _check(lib.pda_headchunk_run_ex(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), B, H, Sq, Skv, d, float(scale),
                                    n_v, sizes, n_groups, int(sp_ranks), int(sink_layout),
                                    _stream_handle(compute_stream), _stream_handle(drain_stream), _ptr(sink),
                                    gms if timed else None, C.byref(tms) if timed else None))
    if timed:
        return [gms[i] for i in range(n_groups)], tms.value
    return None


def pipesp_postprocess(chunks: Sequence, h: int, n: int, hidden, chunk_row_stride: Optional[int] = None, stream=None):
    """pda_pipesp_postprocess: h chunks [rows,n,D] fp32 -> hidden [rows,n*h,D] fp32.

    chunks may also be ONE concatenated tensor [rows,h*n,D]; its h slices are then passed with the
    concatenated tensor's row stride.
    """
    import torch
    rows, HH, D = hidden.shape
    if HH != h * n:
        raise ValueError("hidden: middle axis must be n*h")
    _expect(hidden, torch.float32, (rows, h * n, D), "hidden")
    if hasattr(chunks, "data_ptr"):
        _expect(chunks, torch.float32, (rows, h * n, D), "t_mod")
        ptrs = [chunks.data_ptr() + j * n * D * 4 for j in range(h)]
        stride = h * n * D if chunk_row_stride is None else int(chunk_row_stride)
    else:
        if len(chunks) != h:
            raise ValueError("need h chunks")
        for j, c in enumerate(chunks):
            _expect(c, torch.float32, (rows, n, D), f"chunk {j}")
        ptrs = [c.data_ptr() for c in chunks]
        stride = n * D if chunk_row_stride is None else int(chunk_row_stride)
    arr = (C.c_void_p * max(h, 1))(*ptrs)
    _check(lib.pda_pipesp_postprocess(arr, int(h), int(n), stride, _ptr(hidden), rows, D, _stream_handle(stream)))
    return hidden


def pack_heads(x, y, unit_rms: bool, premul: float = 1.0, stream=None):
    """pda_pack_heads: x [B,S,H,d] fp32 -> y [B,H,S,d] bf16 (every element times premul before rounding)."""
    import torch
    B, S, H, d = x.shape
    _expect(x, torch.float32, (B, S, H, d), "x")
    _expect(y, torch.bfloat16, (B, H, S, d), "y")
    _check(lib.pda_pack_heads(_ptr(x), _ptr(y), B, S, H, d, 1 if unit_rms else 0, float(premul), _stream_handle(stream)))
    return y


# ---- training: gradients, layer norm (include/pipedit_train.h) ----------------------------------------------

@functools.lru_cache(maxsize=None)
def _torch():
    """torch, without an import statement's search in every check: a call on few rows is bound by host time."""
    import torch
    return torch


@functools.lru_cache(maxsize=None)
def _type_codes():
    torch = _torch()
    return {torch.float32: PDA_F32, torch.bfloat16: PDA_BF16}, {torch.float8_e4m3fn: PDA_E4M3, torch.float8_e5m2: PDA_E5M2}


def _type_code(t, name):
    code = _type_codes()[0].get(t.dtype)
    if code is None:
        raise ValueError(f"{name}: expected fp32 or bf16, got {t.dtype}")
    return code


def _elsewhere(t):
    import torch
    return ValueError(f"a tensor on device {t.get_device()}, the current device is {torch.cuda.current_device()}")


def _stream_of(current: int, stream):
    """A kernel on another device's stream would run there, and so would a workspace that is taken on it."""
    device = getattr(stream, "device", None)                    # (anything with a cuda_stream is a stream here)
    if device is not None and device.index != current:
        raise ValueError(f"a stream of device {device.index}, the current device is {current}")


def _on_current_device(stream, *tensors):
    """A kernel runs on the current device and would follow another device's addresses there."""
    torch = _torch()
    current = torch.cuda.current_device()
    _stream_of(current, stream)
    for t in tensors:
        if t is not None and t.get_device() != current:
            raise _elsewhere(t)


def _workspace(nbytes: int, workspace, stream):
    """The given workspace, checked, or a new one from torch's allocator, on the stream of the call that is to use it."""
    torch = _torch()
    if workspace is None:
        if nbytes == 0:
            return None
        with torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream()):
            return torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    if workspace.dtype is not torch.uint8 or not workspace.is_contiguous() or not workspace.is_cuda:
        raise ValueError("workspace: expected a contiguous cuda uint8 tensor")
    return workspace


def attn_bwd_workspace_bytes(B: int, H: int, Sq: int, Skv: int, d: int, kv_valid_len: Optional[int] = None, n_cu: int = 0) -> int:
    """pda_attn_bwd_workspace; n_cu = 0 asks the current device.  kv_valid_len: None is Skv, PDA_ANY_LEN gives what serves every call of at
    most these sizes (a call on fewer keys or rows may need more than one on all of them)."""
    n = C.c_int64(0)
    _check(lib.pda_attn_bwd_workspace(int(B), int(H), int(Sq), int(Skv), int(d), int(Skv if kv_valid_len is None else kv_valid_len),
                                      int(n_cu), C.byref(n)))
    return n.value


def attn_bwd_workspace(B: int, H: int, Sq: int, Skv: int, d: int, kv_valid_len: Optional[int] = None):
    """A workspace on the current device for programs that keep it: for attn_bwd calls of at most these sizes and any valid length, or with
    kv_valid_len for calls of exactly these."""
    import torch
    return torch.empty(attn_bwd_workspace_bytes(B, H, Sq, Skv, d, PDA_ANY_LEN if kv_valid_len is None else kv_valid_len), dtype=torch.uint8, device="cuda")


def attn_bwd(dout, q, k, v, out, lse, dq, dk, dv, scale: float, kv_valid_len: Optional[int] = None, workspace=None, stream=None):
    """pda_attn_bwd: dout, q [B,H,Sq,d], k, v [B,H,Skv,d] bf16, out fp32 or bf16 and lse of the forward call -> dq, dk, dv bf16.

    workspace: a uint8 tensor of attn_bwd_workspace_bytes (attn_bwd_workspace makes one); None takes one from torch's allocator.
    """
    import torch
    B, H, Sq, d = q.shape
    Skv = k.shape[2]
    bf16 = torch.bfloat16
    _expect(q, bf16, (B, H, Sq, d), "q")
    _expect(k, bf16, (B, H, Skv, d), "k")
    _expect(v, bf16, (B, H, Skv, d), "v")
    _expect(dout, bf16, (B, H, Sq, d), "dout")
    out_type = _type_code(out, "out")
    _expect(out, out.dtype, (B, H, Sq, d), "out")
    _expect(lse, torch.float32, (B, H, Sq), "lse")
    _expect(dq, bf16, (B, H, Sq, d), "dq")
    _expect(dk, bf16, (B, H, Skv, d), "dk")
    _expect(dv, bf16, (B, H, Skv, d), "dv")
    _on_current_device(stream, dout, q, k, v, out, lse, dq, dk, dv, workspace)
    n_v = Skv if kv_valid_len is None else int(kv_valid_len)
    if workspace is None:
        workspace = _workspace(attn_bwd_workspace_bytes(B, H, Sq, Skv, d, n_v), None, stream)
    else:
        _workspace(0, workspace, stream)
    _check(lib.pda_attn_bwd(_ptr(dout), _ptr(q), _ptr(k), _ptr(v), _ptr(out), out_type, _ptr(lse), _ptr(dq), _ptr(dk), _ptr(dv),
                            B, H, Sq, Skv, d, float(scale), n_v, _ptr(workspace), 0 if workspace is None else workspace.numel(),
                            _stream_handle(stream)))
    return dq, dk, dv


def attn_bwd_strided(dout, q, k, v, out, lse, dq, dk, dv, scale: float, kv_valid_len: Optional[int] = None, workspace=None, stream=None):
    """pda_attn_bwd_strided: as attn_bwd, on [B,H,S,d] VIEWS (e.g. x[:, :, a:b]) with compact rows; no copies."""
    import torch
    B, H, Sq, d = q.shape
    Skv = k.shape[2]
    for t, name in ((q, "q"), (k, "k"), (v, "v"), (dout, "dout"), (dq, "dq"), (dk, "dk"), (dv, "dv")):
        if t.dtype != torch.bfloat16:
            raise ValueError(f"{name}: expected bf16")
    out_type = _type_code(out, "out")
    if lse.dtype != torch.float32:
        raise ValueError("lse: expected fp32")
    if any(tuple(t.shape) != (B, H, Sq, d) for t in (dout, out, dq)) or any(tuple(t.shape) != (B, H, Skv, d) for t in (k, v, dk, dv)) \
            or tuple(lse.shape) != (B, H, Sq):
        raise ValueError("shape mismatch")
    st = [_view_strides(t, 2, name) for t, name in ((dout, "dout"), (q, "q"), (k, "k"), (out, "out"))]
    st += [_view_strides(lse, 1, "lse"), _view_strides(dq, 2, "dq"), _view_strides(dk, 2, "dk")]
    if _view_strides(v, 2, "v") != st[2] or _view_strides(dv, 2, "dv") != st[6]:
        raise ValueError("k and v must share their strides, and dk and dv theirs")
    _on_current_device(stream, dout, q, k, v, out, lse, dq, dk, dv, workspace)
    n_v = Skv if kv_valid_len is None else int(kv_valid_len)
    if workspace is None:
        workspace = _workspace(attn_bwd_workspace_bytes(B, H, Sq, Skv, d, n_v), None, stream)
    else:
        _workspace(0, workspace, stream)
    _check(lib.pda_attn_bwd_strided(_ptr(dout), _ptr(q), _ptr(k), _ptr(v), _ptr(out), out_type, _ptr(lse), _ptr(dq), _ptr(dk), _ptr(dv),
                                    B, H, Sq, Skv, d, C.byref(AttnBwdStrides(*(x for s in st for x in s))), float(scale), n_v,
                                    _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream_handle(stream)))
    return dq, dk, dv


def _norm_sizes(stream, x, per_row, params, others):
    """Rows, D and groups of a call, and that all tensors and the stream are of the current device (others: of the shape of x, a workspace).  per_row: fp32 with an entry per row; params: fp32 [D] or [groups, D], which must agree; None: not wanted.
    (One function: a call on few rows is bound by host time.)"""
    torch = _torch()
    f32, device = torch.float32, x.get_device()
    if device < 0 or x.dim() < 1 or not x.is_contiguous():
        raise ValueError("x: expected a contiguous cuda tensor of at least one axis")
    if device != torch.cuda.current_device():
        raise _elsewhere(x)
    _stream_of(device, stream)
    for t in others:
        if t is not None and t.get_device() != device:
            raise _elsewhere(t)
    D = x.shape[-1]
    rows = x.numel() // D if D else 0
    for t, name in per_row:
        if t is None:
            continue
        if t.get_device() != device:
            raise _elsewhere(t)
        if t.dtype is not f32 or t.numel() != rows or not t.is_contiguous():
            raise ValueError(f"{name}: expected contiguous cuda fp32 with one entry per row")
    groups = 0
    for t, name in params:
        if t is None:
            continue
        shape = t.shape
        n = 1 if len(shape) == 1 else shape[0] if len(shape) == 2 else -1
        if t.get_device() != device:
            raise _elsewhere(t)
        if n < 1 or t.dtype is not f32 or shape[-1] != D or not t.is_contiguous():
            raise ValueError(f"{name}: expected contiguous cuda fp32 [{D}] or [groups, {D}], got {t.dtype} {tuple(shape)}")
        if groups not in (0, n):
            raise ValueError(f"{name}: {n} groups, another parameter has {groups}")
        groups = n
    return rows, D, groups or 1


def layer_norm_fwd(x, weight, bias, y, mean=None, rstd=None, eps: float = 1e-6, stream=None):
    """pda_layer_norm_fwd: x [..., D] -> y [..., D] (fp32 or bf16 each), mean and rstd [rows] fp32 for the backward call.

    weight, bias: [D], or [groups, D] with one row for every rows/groups consecutive rows of x, or None.
    """
    rows, D, groups = _norm_sizes(stream, x, ((mean, "mean"), (rstd, "rstd")), ((weight, "weight"), (bias, "bias")), (y,))
    _expect(y, y.dtype, x.shape, "y")
    _check(lib.pda_layer_norm_fwd(_ptr(x), _type_code(x, "x"), _ptr(weight), _ptr(bias), _ptr(y), _type_code(y, "y"), _ptr(mean), _ptr(rstd),
                                  rows, groups, D, float(eps), _stream_handle(stream)))
    return y, mean, rstd


def layer_norm_bwd_workspace_bytes(rows: int, D: int, groups: int = 1, n_cu: int = 0) -> int:
    """pda_layer_norm_bwd_workspace; n_cu = 0 asks the current device."""
    n = C.c_int64(0)
    _check(lib.pda_layer_norm_bwd_workspace(int(rows), int(groups), int(D), int(n_cu), C.byref(n)))
    return n.value


def layer_norm_bwd_workspace(rows: int, D: int, groups: int = 1):
    """A workspace for layer_norm_bwd calls of these sizes on the current device, for programs that keep it."""
    import torch
    return torch.empty(layer_norm_bwd_workspace_bytes(rows, D, groups), dtype=torch.uint8, device="cuda")


def layer_norm_bwd(dy, x, weight, mean, rstd, dx, dweight, dbias, workspace=None, stream=None):
    """pda_layer_norm_bwd: dy like y, x, weight, mean, rstd of the forward call -> dx like x, dweight and dbias [D] or [groups, D].

    dx, dweight and dbias may be None; weight is None where the forward call had none.
    """
    rows, D, groups = _norm_sizes(stream, x, ((mean, "mean"), (rstd, "rstd")), ((weight, "weight"), (dweight, "dweight"), (dbias, "dbias")),
                                  (dy, dx, workspace))
    _expect(dy, dy.dtype, x.shape, "dy")
    if dx is not None:
        _expect(dx, x.dtype, x.shape, "dx")
    if workspace is None:
        need = layer_norm_bwd_workspace_bytes(rows, D, groups) if dweight is not None or dbias is not None else 0
        workspace = _workspace(need, None, stream)
    else:
        _workspace(0, workspace, stream)
    _check(lib.pda_layer_norm_bwd(_ptr(dy), _type_code(dy, "dy"), _ptr(x), _type_code(x, "x"), _ptr(weight), _ptr(mean), _ptr(rstd),
                                  _ptr(dx), _ptr(dweight), _ptr(dbias), rows, groups, D,
                                  _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream_handle(stream)))
    return dx, dweight, dbias


def pack_heads_bwd(dy, x, dx, unit_rms: bool, premul: float = 1.0, stream=None):
    """pda_pack_heads_bwd: dy [B,H,S,d] bf16, the pack's x [B,S,H,d] fp32 (None without unit_rms) -> dx [B,S,H,d] fp32."""
    import torch
    B, H, S, d = dy.shape
    _expect(dy, torch.bfloat16, (B, H, S, d), "dy")
    if x is not None:
        _expect(x, torch.float32, (B, S, H, d), "x")
    _expect(dx, torch.float32, (B, S, H, d), "dx")
    _on_current_device(stream, dy, x, dx)
    _check(lib.pda_pack_heads_bwd(_ptr(dy), _ptr(x), _ptr(dx), B, S, H, d, 1 if unit_rms else 0, float(premul), _stream_handle(stream)))
    return dx


# ---- projections: RMS norm, 8-bit matrices and their product, rotary positions (include/pipedit_proj.h) -------

def _fp8_code(t, name):
    code = _type_codes()[1].get(t.dtype)
    if code is None:
        raise ValueError(f"{name}: expected float8_e4m3fn or float8_e5m2, got {t.dtype}")
    return code


def _up(n: int, m: int) -> int:
    return (n + m - 1) // m * m


def _expect_fp8(q, scales, rows: int, cols: int, block_rows: int, name: str):
    """q [rows, cols padded to 128] and its scales [blocks of rows, blocks of columns padded to 4] -> the code of its type."""
    code = _fp8_code(q, name)
    width = -(-cols // 128)
    shape = (rows, 128 * width)
    if q.shape != shape or not q.is_contiguous() or not q.is_cuda:
        raise ValueError(f"{name}: expected contiguous cuda {shape}, got {tuple(q.shape)} contiguous={q.is_contiguous()} cuda={q.is_cuda}")
    shape = (rows if block_rows == 1 else -(-rows // block_rows), width + 3 & ~3)
    if scales is None or scales.dtype is not _torch().float8_e8m0fnu or scales.shape != shape or not scales.is_contiguous() or not scales.is_cuda:
        raise ValueError(f"{name}_scales: expected contiguous cuda float8_e8m0fnu {shape}, got " +
                         ("None" if scales is None else f"{scales.dtype} {tuple(scales.shape)} contiguous={scales.is_contiguous()} cuda={scales.is_cuda}"))
    return code


def fp8_empty(rows: int, cols: int, block_rows: int = 1, dtype=None):
    """(q, scales) for an 8-bit matrix [rows, cols] on the current device, not filled; dtype: torch.float8_e4m3fn (default) or torch.float8_e5m2."""
    import torch
    q = torch.empty(rows, _up(cols, 128), dtype=torch.float8_e4m3fn if dtype is None else dtype, device="cuda")
    return q, torch.empty(_up(rows, block_rows) // block_rows, _up(_up(cols, 128) // 128, 4), dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)


def fp8_quant(x, q=None, q_scales=None, qt=None, qt_scales=None, block_rows: int = 1, stream=None):
    """pda_fp8_quant: x [rows, cols] fp32 or bf16 (rows may lie apart, not share elements) -> q, q_scales and/or qt, qt_scales (of the transposed matrix), as fp8_empty makes them.

    block_rows: 1 (a scale per row and 128 columns of what is written) or 128 (per 128 x 128, the same in both orders).
    """
    if x.dim() != 2 or not x.is_cuda or (x.shape[1] > 1 and x.stride(1) != 1):
        raise ValueError(f"x: expected a cuda matrix with compact rows, got {tuple(x.shape)} stride {x.stride()}")
    rows, cols = x.shape
    ldx = x.stride(0) if rows > 1 and cols > 0 else cols
    if ldx < cols:
        raise ValueError(f"x: rows that share elements (stride {x.stride()} of {tuple(x.shape)}); a row that is repeated needs .contiguous()")
    if q is None and qt is None:
        raise ValueError("neither q nor qt: nothing to compute")
    if block_rows not in (1, 128):
        raise ValueError(f"block_rows: expected 1 or 128, got {block_rows}")
    if q is not None:
        code = _expect_fp8(q, q_scales, rows, cols, block_rows, "q")
    if qt is not None:
        code = _expect_fp8(qt, qt_scales, cols, rows, block_rows, "qt")
        if q is not None and q.dtype is not qt.dtype:
            raise ValueError("q and qt: expected one type")
    if (q is None and q_scales is not None) or (qt is None and qt_scales is not None):
        raise ValueError("scales without their values")
    _on_current_device(stream, x, q, q_scales, qt, qt_scales)
    _check(lib.pda_fp8_quant(_ptr(x), _type_code(x, "x"), rows, cols, ldx, code, block_rows,
                             _ptr(q), _ptr(q_scales), _ptr(qt), _ptr(qt_scales), _stream_handle(stream)))
    return q, q_scales, qt, qt_scales


def fp8_matmul_workspace_bytes(M: int, N: int, K: int, n_cu: int = 0) -> int:
    """pda_fp8_matmul_workspace (K is rounded up to 128); n_cu = 0 asks the current device."""
    n = C.c_int64(0)
    _check(lib.pda_fp8_matmul_workspace(int(M), int(N), _up(int(K), 128), int(n_cu), C.byref(n)))
    return n.value


def fp8_matmul_workspace(M: int, N: int, K: int):
    """A workspace for fp8_matmul calls of these sizes on the current device, for programs that keep it."""
    import torch
    return torch.empty(fp8_matmul_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda")


@functools.lru_cache(maxsize=4096)
def _fp8_matmul_bytes(M: int, N: int, K: int, device: int) -> int:
    """fp8_matmul_workspace_bytes on the current device, `device`: a call on few rows is bound by host time."""
    return fp8_matmul_workspace_bytes(M, N, K)


def fp8_matmul(a, a_scales, b, b_scales, out, bias=None, workspace=None, stream=None):
    """pda_fp8_matmul: a [M, K] (blocks of one row), b [N, K] (blocks of one row or of 128, as its scales say) -> out [M, N] bf16 = a b^T + bias [N] fp32.

    K is the padded length of the rows.  out may be a view whose rows lie apart.
    """
    torch = _torch()
    if a.dim() != 2 or b.dim() != 2 or a.shape[1] != b.shape[1] or a.shape[1] % 128:
        raise ValueError(f"a, b: expected [M, K] and [N, K] with rows padded to 128, got {tuple(a.shape)} and {tuple(b.shape)}")
    M, K = a.shape
    N = b.shape[0]
    block = 1 if b_scales is not None and b_scales.dim() == 2 and b_scales.shape[0] == N else 128
    code = _expect_fp8(a, a_scales, M, K, 1, "a")
    if _expect_fp8(b, b_scales, N, K, block, "b") != PDA_E4M3:
        raise ValueError(f"b: expected float8_e4m3fn, got {b.dtype}")
    if out.dtype is not torch.bfloat16 or out.shape != (M, N) or not out.is_cuda or (N > 1 and out.stride(1) != 1) or (M > 1 and out.stride(0) < N):
        raise ValueError(f"out: expected cuda bf16 {(M, N)} with compact rows, got {out.dtype} {tuple(out.shape)} stride {out.stride()}")
    if bias is not None:
        _expect(bias, torch.float32, (N,), "bias")
    _on_current_device(stream, a, a_scales, b, b_scales, out, bias, workspace)
    if workspace is None:
        nbytes = _fp8_matmul_bytes(M, N, K, a.get_device())
        workspace = _workspace(nbytes, None, stream) if nbytes else None
    else:
        _workspace(0, workspace, stream)
    _check(lib.pda_fp8_matmul(_ptr(a), code, _ptr(a_scales), _ptr(b), _ptr(b_scales), block, _ptr(bias), _ptr(out), M, N, K,
                              out.stride(0) if M > 1 else N, _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream_handle(stream)))
    return out


def rms_norm_fwd(x, weight, y, res=None, h=None, y_scales=None, rstd=None, eps: float = 1e-6, stream=None):
    """pda_rms_norm_fwd: h = res + x (res and h of one type, both or neither), y = the norm of h times weight; x [..., D].

    weight: [D], or [groups, D] with one row for every rows/groups consecutive rows, or None.  y: fp32 or bf16 of the shape of x, or
    float8_e4m3fn [rows, D padded to 128] with y_scales (fp8_empty(rows, D)).  rstd [rows] fp32, for rms_norm_bwd, or None.
    """
    torch = _torch()
    rows, D, groups = _norm_sizes(stream, x, ((rstd, "rstd"),), ((weight, "weight"),), (res, h, y, y_scales))
    if (res is None) != (h is None):
        raise ValueError("res and h go together")
    if res is not None:
        _expect(res, res.dtype, x.shape, "res")
        _expect(h, res.dtype, x.shape, "h")
    if y.dtype is torch.float8_e4m3fn:
        _expect_fp8(y, y_scales, rows, D, 1, "y")
        code = PDA_E4M3
    else:
        _expect(y, y.dtype, x.shape, "y")
        code = _type_code(y, "y")
        if y_scales is not None:
            raise ValueError("y_scales go with an 8-bit y")
    _check(lib.pda_rms_norm_fwd(_ptr(x), _type_code(x, "x"), _ptr(res), 0 if res is None else _type_code(res, "res"), _ptr(weight), _ptr(h), _ptr(y), code,
                                _ptr(y_scales), _ptr(rstd), rows, groups, D, float(eps), _stream_handle(stream)))
    return h, y, y_scales, rstd


def rms_norm_bwd_workspace_bytes(rows: int, D: int, groups: int = 1, n_cu: int = 0) -> int:
    """pda_rms_norm_bwd_workspace; n_cu = 0 asks the current device."""
    n = C.c_int64(0)
    _check(lib.pda_rms_norm_bwd_workspace(int(rows), int(groups), int(D), int(n_cu), C.byref(n)))
    return n.value


def rms_norm_bwd_workspace(rows: int, D: int, groups: int = 1):
    """A workspace for rms_norm_bwd calls of these sizes on the current device, for programs that keep it."""
    import torch
    return torch.empty(rms_norm_bwd_workspace_bytes(rows, D, groups), dtype=torch.uint8, device="cuda")


def rms_norm_bwd(dy, h, weight, rstd, dh, dweight, dres=None, workspace=None, stream=None):
    """pda_rms_norm_bwd: dy (fp32 or bf16), h, weight, rstd of the forward call, dres (the gradient that reaches h past the norm, or None)
    -> dh like h, the gradient of res and x, and dweight [D] or [groups, D]; dh or dweight may be None.
    """
    rows, D, groups = _norm_sizes(stream, h, ((rstd, "rstd"),), ((weight, "weight"), (dweight, "dweight")), (dy, dres, dh, workspace))
    _expect(dy, dy.dtype, h.shape, "dy")
    for t, name in ((dres, "dres"), (dh, "dh")):
        if t is not None:
            _expect(t, h.dtype, h.shape, name)
    if workspace is None:
        workspace = _workspace(rms_norm_bwd_workspace_bytes(rows, D, groups) if dweight is not None else 0, None, stream)
    else:
        _workspace(0, workspace, stream)
    _check(lib.pda_rms_norm_bwd(_ptr(dy), _type_code(dy, "dy"), _ptr(h), _type_code(h, "h"), _ptr(weight), _ptr(rstd), _ptr(dres), _ptr(dh), _ptr(dweight),
                                rows, groups, D, _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream_handle(stream)))
    return dh, dweight


def rope_frequencies(n: int, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0, original: float = 4096, slow_turns: float = 1.0,
                     fast_turns: float = 32.0):
    """pda_rope_frequencies: (n radians a position, what queries and keys are multiplied by).  scaling: plain, linear, base or blend."""
    out, magnitude = (C.c_double * max(int(n), 1))(), C.c_double(0)
    if scaling not in ROPE_SCALINGS:
        raise ValueError(f"scaling: expected one of {sorted(ROPE_SCALINGS)}, got {scaling!r}")
    _check(lib.pda_rope_frequencies(int(n), float(base), ROPE_SCALINGS[scaling], float(factor), float(original), float(slow_turns), float(fast_turns),
                                    out, C.byref(magnitude)))
    return list(out), magnitude.value


class Rope:
    """What turns: freqs (radians a position, one for each pair of columns), the layout of the pairs (interleaved or half) and how many of them
    turn with each axis of a position (default: all with one).  No frequencies: nothing turns.  Made once, used by every call."""

    def __init__(self, freqs, layout: str = "interleaved", axis_pairs: Optional[Sequence[int]] = None):
        if layout not in ROPE_LAYOUTS:
            raise ValueError(f"layout: expected one of {sorted(ROPE_LAYOUTS)}, got {layout!r}")
        freqs = [float(f) for f in freqs]
        pairs = [len(freqs)] if axis_pairs is None else [int(n) for n in axis_pairs]
        if not 1 <= len(pairs) <= PDA_ROPE_MAX_AXES or any(n < 0 for n in pairs) or sum(pairs) != len(freqs):
            raise ValueError(f"axis_pairs: expected up to {PDA_ROPE_MAX_AXES} counts that sum to {len(freqs)}, got {pairs}")
        if len(freqs) % 4 or len(freqs) > 64:
            raise ValueError(f"freqs: expected a multiple of 4 of them, at most 64, got {len(freqs)}")
        self.rot, self.layout, self.axes = 2 * len(freqs), layout, len(pairs)
        self._freqs = (C.c_double * max(len(freqs), 1))(*freqs)
        self._struct = bytes(RopeStruct(self.rot, ROPE_LAYOUTS[layout], self.axes, (C.c_int * PDA_ROPE_MAX_AXES)(*pairs), C.cast(self._freqs, C.POINTER(C.c_double)), None, 0, 0))

    def at(self, positions, first: int, B: int, S: int) -> RopeStruct:
        """The description for one call (positions, checked, must outlive it)."""
        torch = _torch()
        pos_batch = 0
        if positions is not None:
            if first:
                raise ValueError("positions and first: expected one of them")
            shape = tuple(positions.shape)
            if positions.dtype is not torch.int32 or not positions.is_cuda or not positions.is_contiguous() or \
                    shape not in ((S, self.axes), (B, S, self.axes), (1, S, self.axes)):
                raise ValueError(f"positions: expected contiguous cuda int32 {(S, self.axes)} or {(B, S, self.axes)}, got {positions.dtype} {shape}")
            pos_batch = S * self.axes if len(shape) == 3 and shape[0] == B else 0
        r = RopeStruct.from_buffer_copy(self._struct)
        if positions is not None:
            r.positions, r.pos_batch = positions.data_ptr(), pos_batch
        r.first = int(first)
        return r


def _token_strides(t, B, S, H, d, name):
    """(batch stride, token stride) of a [B,S,H,d] view whose tokens are compact."""
    st = t.stride()
    if tuple(t.shape) != (B, S, H, d) or not t.is_cuda or (d > 1 and st[3] != 1) or (H > 1 and st[2] != d):
        raise ValueError(f"{name}: expected cuda {(B, S, H, d)} with compact tokens, got {tuple(t.shape)} stride {st}")
    return (int(st[0]) if B > 1 else 0), (int(st[1]) if S > 1 else 0)


def _head_strides(t, B, H, S, d, name):
    """(batch stride, head stride) of a bf16 [B,H,S,d] view whose heads are compact."""
    torch = _torch()
    if t.dtype is not torch.bfloat16 or tuple(t.shape) != (B, H, S, d):
        raise ValueError(f"{name}: expected bf16 {(B, H, S, d)}, got {t.dtype} {tuple(t.shape)}")
    st = t.stride()
    if not t.is_cuda or st[3] != 1 or (S > 1 and st[2] != d):
        raise ValueError(f"{name}: rows must be compact on the GPU (stride {st})")
    return (int(st[0]) if B > 1 else 0), (int(st[1]) if H > 1 else 0)


def pack_heads_rope(x, y, rope: Rope, positions=None, first: int = 0, unit_rms: bool = False, premul: float = 1.0, stream=None):
    """pda_pack_heads_rope: x [B,S,H,d] fp32 or bf16 (a view with compact tokens, e.g. a third of a fused projection) -> y [B,H,S,d] bf16 (a view
    with compact heads, e.g. a part of a longer sequence), normalised as by pack_heads and turned by rope.

    positions: int32 [S, axes] or [B, S, axes]; None: token s is at first + s.
    """
    B, S, H, d = x.shape
    xs = _token_strides(x, B, S, H, d, "x")
    ys = _head_strides(y, B, H, S, d, "y")
    _on_current_device(stream, x, y, positions)
    _check(lib.pda_pack_heads_rope(_ptr(x), _type_code(x, "x"), *xs, _ptr(y), *ys, B, S, H, d, C.byref(rope.at(positions, first, B, S)),
                                   1 if unit_rms else 0, float(premul), _stream_handle(stream)))
    return y


def pack_heads_rope_bwd(dy, x, dx, rope: Rope, positions=None, first: int = 0, unit_rms: bool = False, premul: float = 1.0, stream=None):
    """pda_pack_heads_rope_bwd: dy [B,H,S,d] bf16, the pack's x (None without unit_rms) -> dx [B,S,H,d] of x's type; views as for pack_heads_rope."""
    B, S, H, d = dx.shape
    ds = _token_strides(dx, B, S, H, d, "dx")
    gs = _head_strides(dy, B, H, S, d, "dy")
    xs = (0, 0)
    if unit_rms:
        if x is None:
            raise ValueError("x: needed with unit_rms")
        if x.dtype is not dx.dtype:
            raise ValueError(f"x and dx: expected one type, got {x.dtype} and {dx.dtype}")
        xs = _token_strides(x, B, S, H, d, "x")
    _on_current_device(stream, dy, x, dx, positions)
    _check(lib.pda_pack_heads_rope_bwd(_ptr(dy), *gs, _ptr(x) if unit_rms else None, _type_code(dx, "dx"), *xs, _ptr(dx), *ds, B, S, H, d,
                                       C.byref(rope.at(positions, first, B, S)), 1 if unit_rms else 0, float(premul), _stream_handle(stream)))
    return dx


def plan_n_decode(t_denoise: float, t_decode: float, N: int) -> int:
    out = C.c_int(0)
    _check(lib.pda_plan_n_decode(float(t_denoise), float(t_decode), int(N), C.byref(out)))
    return out.value


def plan_aco(t_L: float, t_A: float, n_denoise: int, n_decode: int):
    """(T_baseline, T_coop, speed-up S)."""
    a, b, c = C.c_double(0), C.c_double(0), C.c_double(0)
    _check(lib.pda_plan_aco(float(t_L), float(t_A), int(n_denoise), int(n_decode), C.byref(a), C.byref(b), C.byref(c)))
    return a.value, b.value, c.value


def plan_head_padding(H: int, n_denoise: int):
    """(padded heads, heads per GPU, GPUs effectively needed)."""
    a, b, c = C.c_int(0), C.c_int(0), C.c_int(0)
    _check(lib.pda_plan_head_padding(int(H), int(n_denoise), C.byref(a), C.byref(b), C.byref(c)))
    return a.value, b.value, c.value


def plan_ragged_groups(H: int, n: int):
    arr = (C.c_int * max(int(n), 1))()
    _check(lib.pda_plan_ragged_groups(int(H), int(n), arr))
    return [arr[i] for i in range(int(n))]


def probe_mfma_rate(operands, mfma_per_wave: int = 1 << 20, stream=None):
    """pda_probe_mfma_rate on a bf16 tensor: (TFLOP/s, ms) of an MFMA-only loop fed with its values."""
    import torch
    if operands.dtype != torch.bfloat16 or not operands.is_contiguous() or not operands.is_cuda:
        raise ValueError("operands: expected a contiguous cuda bf16 tensor")
    tf, ms = C.c_float(0.0), C.c_float(0.0)
    _check(lib.pda_probe_mfma_rate(_ptr(operands), operands.numel(), int(mfma_per_wave), C.byref(tf), C.byref(ms),
                                   _stream_handle(stream)))
    return tf.value, ms.value


def probe_loop_rate(operands, mix: int, mfma_per_wave: int = 1 << 20, stream=None):
    """pda_probe_loop_rate: (TFLOP/s, ms) of the MFMA loop with the attention loop's other instruction classes (mix 0..3)."""
    import torch
    if operands.dtype != torch.bfloat16 or not operands.is_contiguous() or not operands.is_cuda:
        raise ValueError("operands: expected a contiguous cuda bf16 tensor")
    tf, ms = C.c_float(0.0), C.c_float(0.0)
    _check(lib.pda_probe_loop_rate(_ptr(operands), operands.numel(), int(mfma_per_wave), int(mix), C.byref(tf), C.byref(ms),
                                   _stream_handle(stream)))
    return tf.value, ms.value
