"""Thin ctypes binding of liblookme.so (the C ABI in include/lookme.h).

Argument marshalling only: every step of the path runs in the library's
gfx950 kernels.  If the library has not been built this module raises on
first use; there is no other implementation to fall back to.

The functions keep the C names and order of arguments; tensors are torch
tensors (device memory), converted to raw pointers here.
"""

from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblookme.so")

LOOKME_OK, LOOKME_ERR_INVALID, LOOKME_ERR_UNSUPPORTED, LOOKME_ERR_WORKSPACE, LOOKME_ERR_HIP = range(5)
LOOKME_F32, LOOKME_BF16 = 0, 1
LOOKME_SCORE_DOT, LOOKME_SCORE_COS = 0, 1
LOOKME_KMAX = 32
LOOKME_NOALLOC_MAX_ROWS = 131072
LOOKME_MAX_GROUPS = 16384
LOOKME_ATTENTION_WORKSPACE = 64 << 20
INT32 = 1 << 31     # one past the largest int32_t, as which the library takes most sizes

STATUS_NAMES = {0: "OK", 1: "INVALID", 2: "UNSUPPORTED", 3: "WORKSPACE", 4: "HIP"}

EXPORTED = ("lookme_create", "lookme_workspace_size", "lookme_set_workspace", "lookme_route",
            "lookme_lookup", "lookme_inject", "lookme_select", "lookme_inject_kept",
            "lookme_set_relevance", "lookme_lookup_relevance", "lookme_set_fusion",
            "lookme_inject_fused", "lookme_set_propagation", "lookme_inject_propagated",
            "lookme_set_multiscale", "lookme_inject_multiscale",
            "lookme_inject_multiscale_gated", "lookme_gate",
            "lookme_inject_gated", "lookme_inject_fused_gated", "lookme_inject_propagated_gated",
            "lookme_inject_text", "lookme_lookup_select", "lookme_lookup_gate",
            "lookme_scene_keys", "lookme_index_errors",
            "lookme_destroy", "lookme_last_error",
            "lookme_profile_enable", "lookme_profile_read", "lookme_inject_noalloc",
            "lookme_residual_norm", "lookme_group_rows", "lookme_grouped_product",
            "lookme_grouped_product_quant", "lookme_quant_product", "lookme_quant_swiglu",
            "lookme_head_norm_rotary", "lookme_cache_write", "lookme_cache_read",
            "lookme_cache_attention", "lookme_cache_attention_workspace")

GROUPS = ("project", "route", "bucket", "score", "norm", "select", "inject")


class LookmeError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"LOOKME_ERR_{STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


class lookme_desc_t(ctypes.Structure):
    _fields_ = [("num_scenes", ctypes.c_int32), ("prims_per_scene", ctypes.c_int32),
                ("key_dim", ctypes.c_int32), ("value_dim", ctypes.c_int32),
                ("top_k", ctypes.c_int32), ("dtype", ctypes.c_int32), ("score", ctypes.c_int32)]


_lib = None
_vp = ctypes.c_void_p


def load():
    """Load liblookme.so once; raise if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                           "`python -m paper_2607_16305_amd.build` (no fallback path exists)")
    lib = ctypes.CDLL(LIB_PATH)
    st = ctypes.c_int
    sig = {
        "lookme_create": [ctypes.POINTER(lookme_desc_t), _vp, _vp, _vp, _vp, ctypes.POINTER(_vp)],
        "lookme_workspace_size": [_vp, ctypes.c_int32, ctypes.c_int64,
                                  ctypes.POINTER(ctypes.c_size_t)],
        "lookme_set_workspace": [_vp, _vp, ctypes.c_size_t],
        "lookme_route": [_vp, ctypes.c_int32, ctypes.c_int64, ctypes.c_int32, _vp, _vp, _vp, _vp,
                         _vp],
        "lookme_lookup": [_vp, ctypes.c_int32, ctypes.c_int64, _vp, _vp, _vp, _vp, _vp],
        "lookme_inject": [_vp, ctypes.c_int32, ctypes.c_int64, ctypes.c_int64, _vp,
                          ctypes.c_int32, _vp, _vp, _vp, _vp, ctypes.c_int32, _vp, _vp],
        "lookme_select": [_vp, ctypes.c_int32, ctypes.c_int64, ctypes.c_int64, _vp,
                          ctypes.c_int32, _vp, _vp],
        "lookme_inject_noalloc": [_vp, ctypes.c_int32, ctypes.c_int64, ctypes.c_int64, _vp,
                                  ctypes.c_int32, _vp, _vp, _vp, _vp, ctypes.c_int32, _vp, _vp],
        "lookme_inject_kept": [_vp, ctypes.c_int32, ctypes.c_int64, ctypes.c_int64, _vp, _vp, _vp,
                               _vp, _vp, ctypes.c_int32, _vp],
        "lookme_set_relevance": [_vp, ctypes.c_int32, _vp, _vp, _vp, _vp],
        "lookme_lookup_relevance": [_vp, ctypes.c_int32, ctypes.c_int64, _vp, _vp, _vp, _vp, _vp,
                                    _vp],
        "lookme_set_fusion": [_vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, _vp, _vp,
                              _vp],
        "lookme_inject_fused": [_vp, ctypes.c_int32, ctypes.c_int64, ctypes.c_int64, _vp, _vp,
                                _vp, _vp, _vp, ctypes.c_int32, _vp],
        "lookme_set_propagation": [_vp, ctypes.c_int32, _vp],
        "lookme_set_multiscale": [_vp, ctypes.c_int32, ctypes.c_int32, _vp],
        "lookme_inject_multiscale": [_vp, ctypes.c_int64, ctypes.c_int64, _vp, _vp, _vp, _vp, _vp,
                                     ctypes.c_int32, _vp],
        "lookme_inject_propagated": [_vp, ctypes.c_int32, ctypes.c_int64, ctypes.c_int64, _vp,
                                     _vp, _vp, _vp, _vp, ctypes.c_int32, _vp],
        "lookme_gate": [_vp, ctypes.c_int32, ctypes.c_int64, _vp, ctypes.c_int64, ctypes.c_int32,
                        _vp, _vp, _vp, _vp, _vp],
        "lookme_inject_multiscale_gated": [_vp, ctypes.c_int64, _vp, _vp, _vp, _vp, _vp, _vp,
                                           ctypes.c_int32, _vp],
        "lookme_inject_gated": [_vp, ctypes.c_int32, ctypes.c_int64, _vp, _vp, _vp, _vp, _vp,
                                _vp, ctypes.c_int32, _vp],
        "lookme_inject_fused_gated": [_vp, ctypes.c_int32, ctypes.c_int64, _vp, _vp, _vp, _vp,
                                      _vp, _vp, ctypes.c_int32, _vp],
        "lookme_inject_propagated_gated": [_vp, ctypes.c_int32, ctypes.c_int64, _vp, _vp, _vp,
                                           _vp, _vp, _vp, ctypes.c_int32, _vp],
        "lookme_scene_keys": [ctypes.POINTER(lookme_desc_t), _vp, _vp, _vp],
        "lookme_index_errors": [_vp, ctypes.POINTER(ctypes.c_uint64)],
        "lookme_inject_text": [ctypes.c_int32, _vp, ctypes.c_int64, ctypes.c_int32,
                               ctypes.c_int64, _vp, _vp, _vp, _vp, _vp, ctypes.c_int64,
                               ctypes.c_int32, _vp],
        "lookme_lookup_select": [_vp, ctypes.c_int32, ctypes.c_int64, _vp, _vp, _vp, _vp,
                                 ctypes.c_int64, _vp, ctypes.c_int32, _vp, _vp],
        "lookme_lookup_gate": [_vp, ctypes.c_int32, ctypes.c_int64, _vp, _vp, _vp, _vp, _vp,
                               ctypes.c_int32, _vp, _vp, _vp, _vp],
        "lookme_residual_norm": [ctypes.c_int32, ctypes.c_int64, ctypes.c_int32, _vp,
                                 ctypes.c_int32, _vp, _vp, _vp, ctypes.c_float, _vp, _vp, _vp,
                                 _vp, _vp],
        "lookme_group_rows": [ctypes.c_int32, ctypes.c_int64, _vp, _vp, _vp, _vp],
        "lookme_grouped_product": [ctypes.c_int32, ctypes.c_int32, ctypes.c_int64,
                                   ctypes.c_int32, ctypes.c_int32, _vp, ctypes.c_int64, _vp,
                                   ctypes.c_int32, _vp, _vp, _vp, _vp, ctypes.c_int32, _vp],
        "lookme_grouped_product_quant": [ctypes.c_int32, ctypes.c_int64, ctypes.c_int32,
                                         ctypes.c_int32, _vp, _vp, ctypes.c_int64, _vp,
                                         ctypes.c_int32, _vp, _vp, _vp, _vp, _vp, _vp,
                                         ctypes.c_int32, _vp],
        "lookme_quant_product": [ctypes.c_int32, ctypes.c_int64, ctypes.c_int32, ctypes.c_int32,
                                 ctypes.c_int32, _vp, _vp, _vp, _vp, _vp, _vp, _vp],
        "lookme_quant_swiglu": [ctypes.c_int32, ctypes.c_int64, ctypes.c_int32, ctypes.c_int32,
                                ctypes.c_int32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp],
        "lookme_head_norm_rotary": [ctypes.c_int32, ctypes.c_int64, ctypes.c_int32,
                                    ctypes.c_int32, _vp, ctypes.c_int64, _vp, ctypes.c_int64,
                                    ctypes.c_int32, _vp, ctypes.c_int64, _vp, ctypes.c_int64,
                                    ctypes.c_int32, _vp, _vp, ctypes.c_float, ctypes.c_int32,
                                    ctypes.c_int32, ctypes.c_int32, _vp, _vp, _vp,
                                    ctypes.c_float, _vp],
        "lookme_cache_write": [ctypes.c_int32, ctypes.c_int64, ctypes.c_int32, ctypes.c_int32,
                               _vp, ctypes.c_int64, _vp, ctypes.c_int64, _vp, ctypes.c_int64,
                               ctypes.c_int32, _vp, _vp],
        "lookme_cache_read": [ctypes.c_int32, ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, _vp,
                              ctypes.c_int64, ctypes.c_int32, _vp, _vp, ctypes.c_int64, _vp,
                              ctypes.c_int64, _vp],
        "lookme_cache_attention": [ctypes.c_int32, ctypes.c_int64, ctypes.c_int32, ctypes.c_int32,
                                   ctypes.c_int32, ctypes.c_int32, _vp, ctypes.c_int64, _vp, _vp,
                                   _vp, ctypes.c_int32, ctypes.c_int64, ctypes.c_int32, _vp,
                                   ctypes.c_float, ctypes.c_int32, _vp, ctypes.c_int64, _vp,
                                   ctypes.c_size_t, _vp],
        "lookme_cache_attention_workspace": [ctypes.c_int32, ctypes.c_int64, ctypes.c_int32,
                                             ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                             ctypes.c_int32, ctypes.c_int32,
                                             ctypes.POINTER(ctypes.c_size_t)],
        "lookme_destroy": [_vp],
        "lookme_profile_enable": [_vp, ctypes.c_int32],
        "lookme_profile_read": [_vp, ctypes.c_int32, ctypes.POINTER(ctypes.c_int64),
                                ctypes.POINTER(ctypes.c_double), ctypes.c_int32],
    }
    for name, args in sig.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = st
    lib.lookme_last_error.argtypes = []
    lib.lookme_last_error.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _check(status: int):
    if status != LOOKME_OK:
        raise LookmeError(status, load().lookme_last_error().decode())


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        # the current stream's handle without a Stream object around it (7 us a call)
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


DTYPE_CODE = {torch.float32: LOOKME_F32, torch.bfloat16: LOOKME_BF16}


def lookme_create(desc: lookme_desc_t, scene_keys, prim_keys, values, scene_bias=None):
    """Returns an opaque handle (int).  The table tensors are borrowed."""
    h = _vp()
    _check(load().lookme_create(ctypes.byref(desc), _ptr(scene_keys), _ptr(prim_keys),
                                _ptr(values), _ptr(scene_bias), ctypes.byref(h)))
    return h.value


def lookme_workspace_size(h, layers: int, n_tokens: int) -> int:
    out = ctypes.c_size_t()
    _check(load().lookme_workspace_size(h, layers, n_tokens, ctypes.byref(out)))
    return out.value


def lookme_set_workspace(h, ws, nbytes: int):
    _check(load().lookme_set_workspace(h, _ptr(ws), nbytes))


def lookme_route(h, layers, n, d_in, x, w_proj, q_out, scene_out, stream=None):
    _check(load().lookme_route(h, layers, n, d_in, _ptr(x), _ptr(w_proj), _ptr(q_out),
                               _ptr(scene_out), _stream(stream)))


def lookme_lookup(h, layers, n, q, scene, prim_out, w_out, stream=None):
    _check(load().lookme_lookup(h, layers, n, _ptr(q), _ptr(scene), _ptr(prim_out),
                                _ptr(w_out), _stream(stream)))


def lookme_inject(h, layers, n, n_keep, crit, d_c, scene, prim, w, hidden, d_h, kept_out=None,
                  stream=None):
    _check(load().lookme_inject(h, layers, n, n_keep, _ptr(crit), d_c, _ptr(scene), _ptr(prim),
                                _ptr(w), _ptr(hidden), d_h, _ptr(kept_out), _stream(stream)))


def lookme_inject_noalloc(h, layers, n, n_keep, crit, d_c, scene, prim, w, hidden, d_h,
                          kept_out=None, stream=None):
    _check(load().lookme_inject_noalloc(h, layers, n, n_keep, _ptr(crit), d_c, _ptr(scene),
                                        _ptr(prim), _ptr(w), _ptr(hidden), d_h, _ptr(kept_out),
                                        _stream(stream)))


def lookme_select(h, layers, n, n_keep, crit, d_c, kept_out, stream=None):
    _check(load().lookme_select(h, layers, n, n_keep, _ptr(crit), d_c, _ptr(kept_out),
                                _stream(stream)))


def lookme_inject_kept(h, layers, n, n_keep, kept, scene, prim, w, hidden, d_h, stream=None):
    _check(load().lookme_inject_kept(h, layers, n, n_keep, _ptr(kept), _ptr(scene), _ptr(prim),
                                     _ptr(w), _ptr(hidden), d_h, _stream(stream)))


def lookme_set_relevance(h, hidden, w1, b1, w2, b2):
    _check(load().lookme_set_relevance(h, hidden, _ptr(w1), _ptr(b1), _ptr(w2), _ptr(b2)))


def lookme_lookup_relevance(h, layers, n, q, scene, act_out, prim_out, w_out, stream=None):
    _check(load().lookme_lookup_relevance(h, layers, n, _ptr(q), _ptr(scene), _ptr(act_out),
                                          _ptr(prim_out), _ptr(w_out), _stream(stream)))


def lookme_set_fusion(h, layers, d_ff, d_h, w_gate, w_up, w_down):
    _check(load().lookme_set_fusion(h, layers, d_ff, d_h, _ptr(w_gate), _ptr(w_up),
                                    _ptr(w_down)))


def lookme_inject_fused(h, layers, n, n_keep, kept, scene, prim, w, hidden, d_h, stream=None):
    _check(load().lookme_inject_fused(h, layers, n, n_keep, _ptr(kept), _ptr(scene), _ptr(prim),
                                      _ptr(w), _ptr(hidden), d_h, _stream(stream)))


def lookme_set_propagation(h, steps, w_p_t):
    _check(load().lookme_set_propagation(h, steps, _ptr(w_p_t)))


def lookme_inject_propagated(h, steps, n, n_keep, kept, scene, prim, w, hidden, d_h,
                             stream=None):
    _check(load().lookme_inject_propagated(h, steps, n, n_keep, _ptr(kept), _ptr(scene),
                                           _ptr(prim), _ptr(w), _ptr(hidden), d_h,
                                           _stream(stream)))


def lookme_set_multiscale(h, scales, d_h, w_he_t):
    _check(load().lookme_set_multiscale(h, scales, d_h, _ptr(w_he_t)))


def lookme_inject_multiscale(h, n, n_keep, kept, scene, prim, w, hidden, d_h, stream=None):
    _check(load().lookme_inject_multiscale(h, n, n_keep, _ptr(kept), _ptr(scene), _ptr(prim),
                                           _ptr(w), _ptr(hidden), d_h, _stream(stream)))


def lookme_lookup_select(h, layers, n, q, scene, prim_out, w_out, n_keep, crit, d_c, kept_out,
                         stream=None):
    _check(load().lookme_lookup_select(h, layers, n, _ptr(q), _ptr(scene), _ptr(prim_out),
                                       _ptr(w_out), n_keep, _ptr(crit), d_c, _ptr(kept_out),
                                       _stream(stream)))


def lookme_lookup_gate(h, layers, n, q, scene, prim_out, w_out, delta, d_c, w_g, kept_out,
                       count_out, stream=None):
    _check(load().lookme_lookup_gate(h, layers, n, _ptr(q), _ptr(scene), _ptr(prim_out),
                                     _ptr(w_out), _ptr(delta), d_c, _ptr(w_g), _ptr(kept_out),
                                     _ptr(count_out), _stream(stream)))


def lookme_gate(h, layers, n, delta, delta_rows, d_c, pos, w_g, kept_out, count_out,
                stream=None):
    _check(load().lookme_gate(h, layers, n, _ptr(delta), delta_rows, d_c, _ptr(pos), _ptr(w_g),
                              _ptr(kept_out), _ptr(count_out), _stream(stream)))


def lookme_inject_gated(h, layers, n, kept, count, scene, prim, w, hidden, d_h, stream=None):
    _check(load().lookme_inject_gated(h, layers, n, _ptr(kept), _ptr(count), _ptr(scene),
                                      _ptr(prim), _ptr(w), _ptr(hidden), d_h, _stream(stream)))


def lookme_inject_multiscale_gated(h, n, kept, count, scene, prim, w, hidden, d_h, stream=None):
    _check(load().lookme_inject_multiscale_gated(h, n, _ptr(kept), _ptr(count), _ptr(scene),
                                                 _ptr(prim), _ptr(w), _ptr(hidden), d_h,
                                                 _stream(stream)))


def lookme_inject_fused_gated(h, layers, n, kept, count, scene, prim, w, hidden, d_h,
                              stream=None):
    _check(load().lookme_inject_fused_gated(h, layers, n, _ptr(kept), _ptr(count), _ptr(scene),
                                            _ptr(prim), _ptr(w), _ptr(hidden), d_h,
                                            _stream(stream)))


def lookme_inject_propagated_gated(h, steps, n, kept, count, scene, prim, w, hidden, d_h,
                                   stream=None):
    _check(load().lookme_inject_propagated_gated(h, steps, n, _ptr(kept), _ptr(count),
                                                 _ptr(scene), _ptr(prim), _ptr(w), _ptr(hidden),
                                                 d_h, _stream(stream)))


def lookme_index_errors(stream=None):
    """Kept entries left out for an index out of range since the last call
    (read and reset; synchronises the stream)."""
    v = ctypes.c_uint64(0)
    _check(load().lookme_index_errors(_stream(stream), ctypes.byref(v)))
    return v.value


def lookme_scene_keys(desc, prim_keys, scene_keys, stream=None):
    _check(load().lookme_scene_keys(ctypes.byref(desc) if desc is not None else None,
                                    _ptr(prim_keys), _ptr(scene_keys), _stream(stream)))


def scene_keys(prim_keys, stream=None):
    """lookme_scene_keys on a torch tensor prim_keys [S, P, d_e]: returns the
    [S, d_e] scene keys of Eq. 4 (a new tensor of the same dtype)."""
    import torch
    S, P, d_e = prim_keys.shape
    out = torch.empty((S, d_e), dtype=prim_keys.dtype, device=prim_keys.device)
    desc = lookme_desc_t(S, P, d_e, d_e, 1, DTYPE_CODE[prim_keys.dtype], 0)
    lookme_scene_keys(desc, prim_keys, out, stream)
    return out


def lookme_inject_text(dtype, table, vocab, d_t, n_text, pos, ids, kept, count, hidden, n, d_h,
                       stream=None):
    _check(load().lookme_inject_text(dtype, _ptr(table), vocab, d_t, n_text, _ptr(pos),
                                     _ptr(ids), _ptr(kept), _ptr(count), _ptr(hidden), n, d_h,
                                     _stream(stream)))


def inject_text(table, pos, ids, hidden, kept=None, count=None, stream=None):
    """lookme_inject_text on torch tensors: table [V, d_t], pos and ids
    [n_text] int32, hidden [n, d_h] (updated in place)."""
    lookme_inject_text(DTYPE_CODE[table.dtype], table, table.shape[0], table.shape[1],
                       pos.numel(), pos, ids, kept, count, hidden, hidden.shape[0],
                       hidden.shape[1], stream)


def _int32(*sizes):
    """refuses a size that ctypes would cut to 32 bits"""
    for v in sizes:
        if not -INT32 <= v < INT32:
            _refuse(f"{v} does not fit 32 bits")


def lookme_residual_norm(dtype, n, d, hidden, parts, add, part_w, weight, eps, hidden_out, out,
                         out_quant, scale_out, stream=None):
    _int32(dtype, d, parts)
    _check(load().lookme_residual_norm(dtype, n, d, _ptr(hidden), parts, _ptr(add), _ptr(part_w),
                                       _ptr(weight), eps, _ptr(hidden_out), _ptr(out),
                                       _ptr(out_quant), _ptr(scale_out), _stream(stream)))


def lookme_group_rows(groups, n, pick, rows_out, offsets_out, stream=None):
    _int32(groups)
    _check(load().lookme_group_rows(groups, n, _ptr(pick), _ptr(rows_out), _ptr(offsets_out),
                                    _stream(stream)))


def lookme_grouped_product(dtype, groups, m, d_in, d_out, x, x_rows, rows, picks, offsets, w,
                           w_up, out, scatter, stream=None):
    _int32(dtype, groups, d_in, d_out, picks, scatter)
    _check(load().lookme_grouped_product(dtype, groups, m, d_in, d_out, _ptr(x), x_rows,
                                         _ptr(rows), picks, _ptr(offsets), _ptr(w), _ptr(w_up),
                                         _ptr(out), scatter, _stream(stream)))


def lookme_grouped_product_quant(groups, m, d_in, d_out, x, x_scale, x_rows, rows, picks,
                                 offsets, w, w_scale, w_up, up_scale, out, scatter, stream=None):
    _int32(groups, d_in, d_out, picks, scatter)
    _check(load().lookme_grouped_product_quant(groups, m, d_in, d_out, _ptr(x), _ptr(x_scale),
                                               x_rows, _ptr(rows), picks, _ptr(offsets), _ptr(w),
                                               _ptr(w_scale), _ptr(w_up), _ptr(up_scale),
                                               _ptr(out), scatter, _stream(stream)))


def lookme_quant_product(dtype, n, d_in, d_out, group, x, w, scale, zero, add, out, stream=None):
    _int32(dtype, d_in, d_out, group)
    _check(load().lookme_quant_product(dtype, n, d_in, d_out, group, _ptr(x), _ptr(w),
                                       _ptr(scale), _ptr(zero), _ptr(add), _ptr(out),
                                       _stream(stream)))


def lookme_quant_swiglu(dtype, n, d_in, d_ff, group, x, w_gate, scale_gate, zero_gate, w_up,
                        scale_up, zero_up, out, stream=None):
    _int32(dtype, d_in, d_ff, group)
    _check(load().lookme_quant_swiglu(dtype, n, d_in, d_ff, group, _ptr(x), _ptr(w_gate),
                                      _ptr(scale_gate), _ptr(zero_gate), _ptr(w_up),
                                      _ptr(scale_up), _ptr(zero_up), _ptr(out),
                                      _stream(stream)))


def lookme_head_norm_rotary(dtype, n, head_dim, q_heads, q, q_stride, q_out, q_out_stride, k_heads,
                            k, k_stride, k_out, k_out_stride, norm, q_weight, k_weight, eps, rot,
                            interleaved, axes, pos, axis, freq, factor, stream=None):
    _int32(dtype, head_dim, q_heads, k_heads, norm, rot, interleaved, axes)
    _check(load().lookme_head_norm_rotary(dtype, n, head_dim, q_heads, _ptr(q), q_stride,
                                          _ptr(q_out), q_out_stride, k_heads, _ptr(k), k_stride,
                                          _ptr(k_out), k_out_stride, norm, _ptr(q_weight),
                                          _ptr(k_weight), eps, rot, interleaved, axes, _ptr(pos),
                                          _ptr(axis), _ptr(freq), factor, _stream(stream)))


def lookme_cache_write(dtype, n, kv_heads, head_dim, k, k_stride, v, v_stride, slots, pages, page,
                       cache, stream=None):
    _int32(dtype, kv_heads, head_dim, page)
    _check(load().lookme_cache_write(dtype, n, kv_heads, head_dim, _ptr(k), k_stride, _ptr(v),
                                     v_stride, _ptr(slots), pages, page, _ptr(cache),
                                     _stream(stream)))


def lookme_cache_read(dtype, n, kv_heads, head_dim, slots, pages, page, cache, k_out, k_stride,
                      v_out, v_stride, stream=None):
    _int32(dtype, kv_heads, head_dim, page)
    _check(load().lookme_cache_read(dtype, n, kv_heads, head_dim, _ptr(slots), pages, page,
                                    _ptr(cache), _ptr(k_out), k_stride, _ptr(v_out), v_stride,
                                    _stream(stream)))


def lookme_cache_attention(dtype, n, batch, q_heads, kv_heads, head_dim, q, q_stride, q_offsets,
                           lengths, pages, max_pages, num_pages, page, cache, scale, causal, out,
                           out_stride, workspace, workspace_bytes, stream=None):
    _int32(dtype, batch, q_heads, kv_heads, head_dim, max_pages, page, causal)
    _check(load().lookme_cache_attention(dtype, n, batch, q_heads, kv_heads, head_dim, _ptr(q),
                                         q_stride, _ptr(q_offsets), _ptr(lengths), _ptr(pages),
                                         max_pages, num_pages, page, _ptr(cache), scale, causal,
                                         _ptr(out), out_stride, _ptr(workspace), workspace_bytes,
                                         _stream(stream)))


def lookme_cache_attention_workspace(dtype, n, batch, q_heads, kv_heads, head_dim, max_pages,
                                     page) -> int:
    _int32(dtype, batch, q_heads, kv_heads, head_dim, max_pages, page)
    out = ctypes.c_size_t()
    _check(load().lookme_cache_attention_workspace(dtype, n, batch, q_heads, kv_heads, head_dim,
                                                   max_pages, page, ctypes.byref(out)))
    return out.value


# The same on torch tensors: sizes come from the shapes, which are checked (the
# C side sees pointers only), and the call runs on the tensors' device.  These
# are called once a layer and token, so they keep their own time short.

def _refuse(msg):
    raise LookmeError(LOOKME_ERR_INVALID, msg)


# The helpers below check their tensors in place, and call this for what it says
# where one is not as it must be: a call a tensor is 0.1 us of the 6 that a whole
# call takes on the host, 2.6 of them the launch.
def _wrong(name, t, dtype, shape, device):
    """refuses tensor t for its type, shape, device (an index, as of
    Tensor.get_device) or strides"""
    if t.dtype is not dtype:
        _refuse(f"{name} is {t.dtype}, not {dtype}")
    if t.shape != shape:
        _refuse(f"{name} has the shape {tuple(t.shape)}, not {tuple(shape)}")
    if t.get_device() != device:
        _refuse(f"{name} is on {t.device}, other tensors are elsewhere")
    _refuse(f"{name} is not contiguous")


def _tensor(name, t, dtype, shape, device):
    """t's address, for the rarer tensors"""
    if (t.dtype is not dtype or t.shape != shape or t.get_device() != device
            or not t.is_contiguous()):
        _wrong(name, t, dtype, shape, device)
    return t.data_ptr()


def _dtype_code(name, dtype):
    code = DTYPE_CODE.get(dtype)
    if code is None:
        _refuse(f"{name} is {dtype}: float32 or bfloat16")
    return code


def _call(name, device, stream, *args):
    """The entry point on `stream` (None: the current one) of the tensors'
    device, which is a GPU.  A stream of another device is refused: the kernel
    would run there, on memory that it may not reach."""
    if device < 0:
        _refuse("tensors that are not in device memory")
    if stream is not None and getattr(stream, "device_index", device) != device:
        _refuse(f"the stream is of device {stream.device_index}, the tensors are on {device}")
    if device != torch._C._cuda_getDevice():
        with torch.cuda.device(device):
            return _call(name, device, stream, *args)
    raw = torch._C._cuda_getCurrentRawStream(device) if stream is None else _stream(stream)
    status = getattr(_lib or load(), name)(*args, raw)
    if status != LOOKME_OK:
        _check(status)


def residual_norm(hidden, weight=None, eps=1e-6, add=None, part_w=None, hidden_out=None,
                  out=None, out_quant=None, scale_out=None, stream=None):
    """lookme_residual_norm on torch tensors: hidden [n, d]; add [n, d] or
    [n, parts, d]; part_w [n, parts] float32; weight [d]; the outputs
    hidden_out (may be hidden), out [n, d], out_quant [n, d] float8_e4m3fn
    with scale_out [n] float32."""
    dev, dt, rows = hidden.get_device(), hidden.dtype, hidden.shape
    code = _dtype_code("hidden", dt)
    if len(rows) != 2:
        _refuse(f"hidden has {len(rows)} dimensions, not 2")
    n, d = rows
    if d >= INT32:
        _int32(d)
    if not hidden.is_contiguous():
        _wrong("hidden", hidden, dt, rows, dev)
    parts = 0
    p_add = p_part = p_weight = p_sum = p_out = p_quant = p_scale = None
    if add is not None:
        if add.dim() == 2:
            parts, shape = 1, rows
        else:
            parts = add.shape[1] if add.dim() == 3 else 0
            shape = (n, parts, d)
            if parts >= INT32:
                _int32(parts)
        if (add.dtype is not dt or add.shape != shape or add.get_device() != dev
                or not add.is_contiguous()):
            _wrong("add", add, dt, shape, dev)
        if parts != 0:
            p_add = add.data_ptr()
    if part_w is not None:
        p_part = _tensor("part_w", part_w, torch.float32, (n, parts), dev)
        if parts == 0:
            p_part = None
    if weight is not None:
        if (weight.dtype is not dt or weight.shape != (d,) or weight.get_device() != dev
                or not weight.is_contiguous()):
            _wrong("weight", weight, dt, (d,), dev)
        p_weight = weight.data_ptr()
    if hidden_out is not None:
        if (hidden_out.dtype is not dt or hidden_out.shape != rows
                or hidden_out.get_device() != dev or not hidden_out.is_contiguous()):
            _wrong("hidden_out", hidden_out, dt, rows, dev)
        p_sum = hidden_out.data_ptr()
    if out is not None:
        if (out.dtype is not dt or out.shape != rows or out.get_device() != dev
                or not out.is_contiguous()):
            _wrong("out", out, dt, rows, dev)
        p_out = out.data_ptr()
    if out_quant is not None:
        p_quant = _tensor("out_quant", out_quant, torch.float8_e4m3fn, rows, dev)
    if scale_out is not None:
        p_scale = _tensor("scale_out", scale_out, torch.float32, (n,), dev)
    _call("lookme_residual_norm", dev, stream, code, n, d, hidden.data_ptr(), parts, p_add, p_part,
          p_weight, eps, p_sum, p_out, p_quant, p_scale)


def group_rows(pick, groups, rows_out, offsets_out, stream=None):
    """lookme_group_rows on torch tensors: pick (any shape, n entries) and
    rows_out (as many) int32, offsets_out [groups + 1] int32."""
    dev, n, i32 = pick.get_device(), pick.numel(), torch.int32
    if rows_out.numel() != n:
        _refuse(f"rows_out has {rows_out.numel()} entries, not {n}")
    if groups >= INT32:
        _int32(groups)
    if pick.dtype is not i32 or not pick.is_contiguous():
        _wrong("pick", pick, i32, pick.shape, dev)
    if rows_out.dtype is not i32 or rows_out.get_device() != dev or not rows_out.is_contiguous():
        _wrong("rows_out", rows_out, i32, rows_out.shape, dev)
    if (offsets_out.dtype is not i32 or offsets_out.shape != (groups + 1,)
            or offsets_out.get_device() != dev or not offsets_out.is_contiguous()):
        _wrong("offsets_out", offsets_out, i32, (groups + 1,), dev)
    _call("lookme_group_rows", dev, stream, groups, n, pick.data_ptr(), rows_out.data_ptr(),
          offsets_out.data_ptr())


def grouped_product(x, w, offsets, out, rows=None, picks=1, w_up=None, scatter=False,
                    x_scale=None, w_scale=None, w_up_scale=None, stream=None):
    """lookme_grouped_product on torch tensors, or lookme_grouped_product_quant
    for float8_e4m3fn: x [x_rows, d_in], w and w_up [groups, d_out, d_in],
    offsets [groups + 1] int32, out [m, d_out], rows [m] int32.  With rows,
    entry i reads x[rows[i] // picks] (picks = 0: x[i]); without, x[i]."""
    dev, dt, i32 = x.get_device(), x.dtype, torch.int32
    quant = dt is torch.float8_e4m3fn
    code = 0 if quant else _dtype_code("x", dt)
    x_shape, shape, out_shape = x.shape, w.shape, out.shape
    if len(x_shape) != 2 or len(shape) != 3 or len(out_shape) != 2:
        _refuse("x and out have 2 dimensions, w has 3")
    x_rows, d_in = x_shape
    groups, d_out, _ = shape
    m = out_shape[0]
    if d_in >= INT32 or d_out >= INT32 or groups >= INT32 or not -INT32 <= picks < INT32:
        _int32(d_in, d_out, groups, picks)
    if not x.is_contiguous():
        _wrong("x", x, dt, x_shape, dev)
    if w.dtype is not dt or shape[2] != d_in or w.get_device() != dev or not w.is_contiguous():
        _wrong("w", w, dt, (groups, d_out, d_in), dev)
    if (offsets.dtype is not i32 or offsets.shape != (groups + 1,)
            or offsets.get_device() != dev or not offsets.is_contiguous()):
        _wrong("offsets", offsets, i32, (groups + 1,), dev)
    out_dt = torch.bfloat16 if quant else dt
    if (out.dtype is not out_dt or out_shape[1] != d_out or out.get_device() != dev
            or not out.is_contiguous()):
        _wrong("out", out, out_dt, (m, d_out), dev)
    p_up = p_rows = None
    if w_up is not None:
        if (w_up.dtype is not dt or w_up.shape != shape or w_up.get_device() != dev
                or not w_up.is_contiguous()):
            _wrong("w_up", w_up, dt, shape, dev)
        p_up = w_up.data_ptr()
    if rows is None:
        picks = 0
    else:
        if (rows.dtype is not i32 or rows.shape != (m,) or rows.get_device() != dev
                or not rows.is_contiguous()):
            _wrong("rows", rows, i32, (m,), dev)
        p_rows = rows.data_ptr()
    if not quant:
        if x_scale is not None or w_scale is not None or w_up_scale is not None:
            _refuse(f"scales given for {dt}")
        return _call("lookme_grouped_product", dev, stream, code, groups, m, d_in, d_out,
                     x.data_ptr(), x_rows, p_rows, picks, offsets.data_ptr(), w.data_ptr(), p_up,
                     out.data_ptr(), int(scatter))
    if x_scale is None or w_scale is None:
        _refuse("float8_e4m3fn needs x_scale and w_scale")
    f32 = torch.float32
    p_xs = _tensor("x_scale", x_scale, f32, (x_rows,), dev)
    p_ws = _tensor("w_scale", w_scale, f32, (groups, d_out), dev)
    p_us = None if w_up_scale is None else _tensor("w_up_scale", w_up_scale, f32, (groups, d_out),
                                                   dev)
    _call("lookme_grouped_product_quant", dev, stream, groups, m, d_in, d_out, x.data_ptr(), p_xs,
          x_rows, p_rows, picks, offsets.data_ptr(), w.data_ptr(), p_ws, p_up, p_us,
          out.data_ptr(), int(scatter))


def _quant_matrix(name, dev, dt, d_in, w, scale, zero):
    """(d_out, group, addresses of w, scale and zero)"""
    shape, u8 = scale.shape, torch.uint8
    d_out, groups = shape
    if d_in >= INT32 or d_out >= INT32:
        _int32(d_in, d_out)
    if groups < 1 or d_in % groups != 0:
        _refuse(f"scale has {groups} groups for {d_in} columns")
    if (w.dtype is not u8 or w.shape != (d_out, d_in // 2) or w.get_device() != dev
            or not w.is_contiguous()):
        _wrong(name, w, u8, (d_out, d_in // 2), dev)
    if scale.dtype is not dt or scale.get_device() != dev or not scale.is_contiguous():
        _wrong("its scale", scale, dt, shape, dev)
    return (d_out, d_in // groups, w.data_ptr(), scale.data_ptr(),
            None if zero is None else _tensor("its zero", zero, u8, shape, dev))


def quant_product(x, w, scale, out, zero=None, add=None, stream=None):
    """lookme_quant_product on torch tensors: x [n, d_in], w [d_out, d_in / 2]
    uint8, scale [d_out, groups], zero [d_out, groups] uint8, add and out
    [n, d_out] (out may be add)."""
    dev, dt, shape = x.get_device(), x.dtype, x.shape
    code = _dtype_code("x", dt)
    if len(shape) != 2 or scale.dim() != 2:
        _refuse("x and scale have 2 dimensions")
    n, d_in = shape
    if not x.is_contiguous():
        _wrong("x", x, dt, shape, dev)
    d_out, group, p_w, p_s, p_z = _quant_matrix("w", dev, dt, d_in, w, scale, zero)
    if (out.dtype is not dt or out.shape != (n, d_out) or out.get_device() != dev
            or not out.is_contiguous()):
        _wrong("out", out, dt, (n, d_out), dev)
    p_add = None if add is None else _tensor("add", add, dt, (n, d_out), dev)
    _call("lookme_quant_product", dev, stream, code, n, d_in, d_out, group, x.data_ptr(), p_w, p_s,
          p_z, p_add, out.data_ptr())


def quant_swiglu(x, w_gate, s_gate, w_up, s_up, out, z_gate=None, z_up=None, stream=None):
    """lookme_quant_swiglu on torch tensors, each matrix as for quant_product;
    out [n, d_ff]."""
    dev, dt, shape = x.get_device(), x.dtype, x.shape
    code = _dtype_code("x", dt)
    if len(shape) != 2 or s_gate.dim() != 2 or s_up.dim() != 2:
        _refuse("x and the scales have 2 dimensions")
    n, d_in = shape
    if not x.is_contiguous():
        _wrong("x", x, dt, shape, dev)
    d_ff, group, *gate = _quant_matrix("w_gate", dev, dt, d_in, w_gate, s_gate, z_gate)
    d_up, group_up, *up = _quant_matrix("w_up", dev, dt, d_in, w_up, s_up, z_up)
    if (d_up, group_up) != (d_ff, group):
        _refuse("w_gate and w_up differ in size or group")
    p_out = _tensor("out", out, dt, (n, d_ff), dev)
    _call("lookme_quant_swiglu", dev, stream, code, n, d_in, d_ff, group, x.data_ptr(), *gate, *up,
          p_out)


def _heads(name, t, dtype, shape, device):
    """(address, stride of a row) of t of the shape (n, heads, d), whose rows may lie
    apart"""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device:
        _wrong(name, t, dtype, shape, device)
    n, heads, d = shape
    if t.is_contiguous():
        return t.data_ptr(), heads * d
    row, head, one = t.stride()
    if (one != 1 and d > 1) or (head != d and heads > 1):
        _refuse(f"the heads of {name} do not lie side by side (strides {t.stride()})")
    if n < 2:
        row = heads * d
    elif row < heads * d:
        _refuse(f"the rows of {name} overlap (stride {row})")
    return t.data_ptr(), row


def head_norm_rotary(q, q_out, k=None, k_out=None, norm=True, q_weight=None, k_weight=None,
                     eps=1e-6, pos=None, freq=None, axis=None, factor=1.0, interleaved=False,
                     stream=None):
    """lookme_head_norm_rotary on torch tensors: q and q_out [n, q_heads, d], k and
    k_out [n, k_heads, d] (rows may lie apart, as in a product of q, k and v; outputs
    may be their inputs); q_weight and k_weight [d]; pos [n] or [axes, n] int32, freq
    [rot / 2] float32, axis [rot / 2] int32.  Without freq nothing is rotated."""
    dev, dt = q.get_device(), q.dtype
    code = _dtype_code("q", dt)
    if q.dim() != 3:
        _refuse(f"q has {q.dim()} dimensions, not 3")
    shape = q.shape
    n, q_heads, d = shape
    if d >= INT32 or q_heads >= INT32:
        _int32(d, q_heads)
    p_q, q_row = _heads("q", q, dt, shape, dev)
    p_qo, qo_row = _heads("q_out", q_out, dt, shape, dev)
    k_heads, p_k, k_row, p_ko, ko_row = 0, None, 0, None, 0
    if (k is None) != (k_out is None):
        _refuse("k and k_out go together")
    if k is not None:
        shape = k.shape
        k_heads = shape[1] if len(shape) == 3 else 0
        if k_heads >= INT32:
            _int32(k_heads)
        if len(shape) != 3 or shape[0] != n or shape[2] != d:
            _wrong("k", k, dt, (n, k_heads, d), dev)
        p_k, k_row = _heads("k", k, dt, shape, dev)
        p_ko, ko_row = _heads("k_out", k_out, dt, shape, dev)
    elif k_weight is not None:
        _refuse("k_weight given without k")
    p_qw = None if q_weight is None else _tensor("q_weight", q_weight, dt, (d,), dev)
    p_kw = None if k_weight is None else _tensor("k_weight", k_weight, dt, (d,), dev)
    rot, axes, p_pos, p_axis, p_freq = 0, 1, None, None, None
    if freq is not None:
        rot = 2 * freq.numel()
        if pos is None:
            _refuse("freq given without pos")
        two = pos.dim() == 2
        axes = pos.shape[0] if two else 1
        if rot >= INT32 or axes >= INT32:
            _int32(rot, axes)
        if (freq.dtype is not torch.float32 or freq.dim() != 1 or freq.get_device() != dev
                or not freq.is_contiguous()):
            _wrong("freq", freq, torch.float32, (rot // 2,), dev)
        p_freq = freq.data_ptr()
        if (pos.dtype is not torch.int32 or pos.shape != ((axes, n) if two else (n,))
                or pos.get_device() != dev or not pos.is_contiguous()):
            _wrong("pos", pos, torch.int32, (axes, n) if two else (n,), dev)
        p_pos = pos.data_ptr()
        if axis is not None:
            p_axis = _tensor("axis", axis, torch.int32, (rot // 2,), dev)
        elif axes > 1:
            _refuse(f"positions of {axes} axes need axis")
        if rot == 0:
            p_pos = p_axis = p_freq = None
    elif pos is not None or axis is not None:
        _refuse("positions given without freq")
    _call("lookme_head_norm_rotary", dev, stream, code, n, d, q_heads, p_q, q_row, p_qo, qo_row,
          k_heads, p_k, k_row, p_ko, ko_row, int(norm), p_qw, p_kw, eps, rot, int(interleaved),
          axes, p_pos, p_axis, p_freq, factor)


def cache_shape(pages, kv_heads, page, head_dim):
    """The shape of a 4-bit cache (a uint8 tensor) of `pages` pages of `page` tokens"""
    return (pages, kv_heads, page // 32, 34 * head_dim)


def _cache(cache, dev):
    """(pages, kv_heads, page, head_dim, address) of a 4-bit cache"""
    shape = cache.shape
    if len(shape) != 4 or shape[3] % 34 != 0:
        _refuse(f"cache has the shape {tuple(shape)}, not [pages, kv_heads, page / 32, 34 d]")
    if cache.dtype is not torch.uint8 or cache.get_device() != dev or not cache.is_contiguous():
        _wrong("cache", cache, torch.uint8, shape, dev)
    pages, heads, tiles, width = shape
    if heads >= INT32 or tiles >= INT32 // 32 or width >= INT32:
        _int32(heads, 32 * tiles, width)
    return pages, heads, 32 * tiles, width // 34, cache.data_ptr()


def cache_write(k, v, slots, cache, stream=None):
    """lookme_cache_write on torch tensors: k and v [n, kv_heads, d] (rows may lie
    apart), slots [n] int32, cache [pages, kv_heads, page / 32, 34 d] uint8."""
    dev, dt = k.get_device(), k.dtype
    code = _dtype_code("k", dt)
    pages, heads, page, d, p_c = _cache(cache, dev)
    shape = k.shape
    n = shape[0] if len(shape) == 3 else 0
    if len(shape) != 3 or shape[1] != heads or shape[2] != d:
        _wrong("k", k, dt, (n, heads, d), dev)
    p_k, k_row = _heads("k", k, dt, shape, dev)
    p_v, v_row = _heads("v", v, dt, shape, dev)
    p_s = _tensor("slots", slots, torch.int32, (n,), dev)
    _call("lookme_cache_write", dev, stream, code, n, heads, d, p_k, k_row, p_v, v_row, p_s, pages,
          page, p_c)


def cache_read(slots, cache, k_out=None, v_out=None, stream=None):
    """lookme_cache_read on torch tensors: slots [n] int32, cache as for
    cache_write, k_out and v_out [n, kv_heads, d] (rows may lie apart), one of them
    may be None."""
    one = v_out if k_out is None else k_out
    if one is None:
        _refuse("no output given")
    dev, dt, n = slots.get_device(), one.dtype, slots.numel()
    code = _dtype_code("the output", dt)
    pages, heads, page, d, p_c = _cache(cache, dev)
    p_s = _tensor("slots", slots, torch.int32, (n,), dev)
    shape = (n, heads, d)
    p_k, k_row = (None, 0) if k_out is None else _heads("k_out", k_out, dt, shape, dev)
    p_v, v_row = (None, 0) if v_out is None else _heads("v_out", v_out, dt, shape, dev)
    _call("lookme_cache_read", dev, stream, code, n, heads, d, p_s, pages, page, p_c, p_k, k_row,
          p_v, v_row)


def cache_attention(q, cache, pages, lengths, out, workspace=None, q_offsets=None, scale=None,
                    causal=True, stream=None):
    """lookme_cache_attention on torch tensors: q and out [n, q_heads, d] (rows may
    lie apart; out may be q), cache as for cache_write, pages [batch, max_pages],
    lengths [batch] and q_offsets [batch + 1] int32 (None: a row each), scale d ** -0.5
    if None, workspace uint8 (of LOOKME_ATTENTION_WORKSPACE bytes for every call, or
    what lookme_cache_attention_workspace gives for one)."""
    dev, dt, i32 = q.get_device(), q.dtype, torch.int32
    code = _dtype_code("q", dt)
    shape, p_shape = q.shape, pages.shape
    if len(shape) != 3 or len(p_shape) != 2:
        _refuse("q has 3 dimensions, pages has 2")
    n, q_heads, _ = shape
    num_pages, kv_heads, page, d, p_c = _cache(cache, dev)
    batch, max_pages = p_shape
    if batch >= INT32 or max_pages >= INT32 or q_heads >= INT32:
        _int32(batch, max_pages, q_heads)
    if shape[2] != d:
        _wrong("q", q, dt, (n, q_heads, d), dev)
    p_q, q_row = _heads("q", q, dt, shape, dev)
    p_o, o_row = _heads("out", out, dt, shape, dev)
    if pages.dtype is not i32 or pages.get_device() != dev or not pages.is_contiguous():
        _wrong("pages", pages, i32, p_shape, dev)
    if (lengths.dtype is not i32 or lengths.shape != (batch,) or lengths.get_device() != dev
            or not lengths.is_contiguous()):
        _wrong("lengths", lengths, i32, (batch,), dev)
    p_l = lengths.data_ptr()
    p_off = None if q_offsets is None else _tensor("q_offsets", q_offsets, i32, (batch + 1,), dev)
    p_w, w_bytes = None, 0
    if workspace is not None:
        w_bytes = workspace.numel()
        p_w = _tensor("workspace", workspace, torch.uint8, workspace.shape, dev)
    _call("lookme_cache_attention", dev, stream, code, n, batch, q_heads, kv_heads, d, p_q, q_row,
          p_off, p_l, pages.data_ptr(), max_pages, num_pages, page, p_c,
          d ** -0.5 if scale is None else scale, int(causal), p_o, o_row, p_w, w_bytes)


def lookme_destroy(h):
    if h:
        _check(load().lookme_destroy(h))


def lookme_profile_enable(h, enabled: bool):
    _check(load().lookme_profile_enable(h, 1 if enabled else 0))


def lookme_profile_read(h, group: int, reset: bool = False):
    """(number of timed launches, total milliseconds) of one kernel group."""
    c = ctypes.c_int64()
    ms = ctypes.c_double()
    _check(load().lookme_profile_read(h, group, ctypes.byref(c), ctypes.byref(ms),
                                      1 if reset else 0))
    return c.value, ms.value


def lookme_last_error() -> str:
    return load().lookme_last_error().decode()


class Table:
    """Convenience owner of a handle plus its workspace (torch device memory)."""

    def __init__(self, scene_keys, prim_keys, values, top_k, scene_bias=None,
                 score=LOOKME_SCORE_DOT):
        S, P, d_e = prim_keys.shape
        self.desc = lookme_desc_t(S, P, d_e, values.shape[1], top_k,
                                  DTYPE_CODE[prim_keys.dtype], score)
        self.tensors = (scene_keys, prim_keys, values, scene_bias)   # keep alive
        self.handle = lookme_create(self.desc, scene_keys, prim_keys, values, scene_bias)
        self.ws = None
        self.ws_rows = (0, 0)
        self.device = prim_keys.device

    def reserve(self, layers: int, n: int):
        need = lookme_workspace_size(self.handle, layers, n)
        if self.ws is None or self.ws.numel() < need:
            self.ws = torch.empty(need, dtype=torch.uint8, device=self.device)
            lookme_set_workspace(self.handle, self.ws, self.ws.numel())
        return need

    def route(self, x, w_proj, q_out, scene_out, layers=1, stream=None):
        n, d_in = x.shape
        self.reserve(layers, n)
        lookme_route(self.handle, layers, n, d_in, x, w_proj, q_out, scene_out, stream)

    def lookup(self, q, scene, prim_out, w_out, layers=1, stream=None):
        n = scene.numel() // layers
        self.reserve(layers, n)
        lookme_lookup(self.handle, layers, n, q, scene, prim_out, w_out, stream)

    def inject(self, crit, scene, prim, w, hidden, n_keep, kept_out=None, layers=1, stream=None):
        n = scene.numel() // layers
        self.reserve(layers, n)
        lookme_inject(self.handle, layers, n, n_keep, crit, crit.shape[-1], scene, prim, w,
                      hidden, hidden.shape[-1], kept_out, stream)

    def lookup_select(self, q, scene, prim_out, w_out, crit, kept_out, n_keep, layers=1,
                      stream=None):
        n = scene.numel() // layers
        self.reserve(layers, n)
        lookme_lookup_select(self.handle, layers, n, q, scene, prim_out, w_out, n_keep, crit,
                             crit.shape[-1], kept_out, stream)

    def lookup_gate(self, q, scene, prim_out, w_out, delta, w_g, kept_out, count_out, layers=1,
                    stream=None):
        n = scene.numel() // layers
        self.reserve(layers, n)
        lookme_lookup_gate(self.handle, layers, n, q, scene, prim_out, w_out, delta,
                           delta.shape[-1], w_g, kept_out, count_out, stream)

    def select(self, crit, kept_out, n_keep, layers=1, stream=None):
        n = crit.numel() // (layers * crit.shape[-1])
        self.reserve(layers, n)
        lookme_select(self.handle, layers, n, n_keep, crit, crit.shape[-1], kept_out, stream)

    def inject_kept(self, kept, scene, prim, w, hidden, n_keep, layers=1, stream=None):
        n = scene.numel() // layers
        lookme_inject_kept(self.handle, layers, n, n_keep, kept, scene, prim, w, hidden,
                           hidden.shape[-1], stream)

    def set_relevance(self, w1, b1, w2, b2):
        self.relevance = (w1, b1, w2, b2)      # keep alive
        lookme_set_relevance(self.handle, w1.shape[0], w1, b1, w2, b2)

    def lookup_relevance(self, q, scene, act_out, prim_out, w_out, layers=1, stream=None):
        n = scene.numel() // layers
        self.reserve(layers, n)
        lookme_lookup_relevance(self.handle, layers, n, q, scene, act_out, prim_out, w_out,
                                stream)

    def set_fusion(self, w_gate, w_up, w_down):
        self.fusion = (w_gate, w_up, w_down)     # keep alive
        L, d_ff, _ = w_gate.shape
        lookme_set_fusion(self.handle, L, d_ff, w_down.shape[1], w_gate, w_up, w_down)

    def inject_fused(self, kept, scene, prim, w, hidden, n_keep, layers=1, stream=None):
        n = scene.numel() // layers
        self.reserve(layers, n)
        lookme_inject_fused(self.handle, layers, n, n_keep, kept, scene, prim, w, hidden,
                            hidden.shape[-1], stream)

    def set_propagation(self, w_p_t):
        self.propagation = w_p_t                 # keep alive
        lookme_set_propagation(self.handle, w_p_t.shape[0], w_p_t)

    def inject_propagated(self, kept, scene, prim, w, hidden, n_keep, steps, stream=None):
        n = scene.numel()
        self.reserve(steps + 1, n)
        lookme_inject_propagated(self.handle, steps, n, n_keep, kept, scene, prim, w, hidden,
                                 hidden.shape[-1], stream)

    def scale_view(self, m: int, scales: int) -> "Table":
        """A table over scale m's partition (scenes [m S/M, (m+1) S/M)) of
        this table's tensors (views, no copies), for that scale's routing and
        lookup."""
        scene_keys, prim_keys, values, _ = self.tensors
        S, P = prim_keys.shape[0], prim_keys.shape[1]
        Sm = S // scales
        return Table(scene_keys[m * Sm:(m + 1) * Sm], prim_keys[m * Sm:(m + 1) * Sm],
                     values[m * Sm * P:(m + 1) * Sm * P], self.desc.top_k)

    def set_multiscale(self, scales, w_he_t):
        self.multiscale = w_he_t                 # keep alive
        lookme_set_multiscale(self.handle, scales, w_he_t.shape[1], w_he_t)

    def inject_multiscale(self, kept, scene, prim, w, hidden, n_keep, stream=None):
        n = hidden.shape[0]
        self.reserve(1, n)
        lookme_inject_multiscale(self.handle, n, n_keep, kept, scene, prim, w, hidden,
                                 hidden.shape[-1], stream)

    def inject_multiscale_gated(self, kept, count, scene, prim, w, hidden, stream=None):
        n = hidden.shape[0]
        self.reserve(1, n)
        lookme_inject_multiscale_gated(self.handle, n, kept, count, scene, prim, w, hidden,
                                       hidden.shape[-1], stream)

    def gate(self, delta, w_g, kept_out, count_out, pos=None, layers=1, stream=None):
        """lookme_gate: delta [layers, rows, d_c] (or [rows, d_c]); pos [n] or
        None (n = rows); w_g [layers, d_c]; kept_out [layers, n]; count_out
        [layers]."""
        rows = delta.numel() // (layers * delta.shape[-1])
        n = rows if pos is None else pos.numel()
        self.reserve(layers, n)
        lookme_gate(self.handle, layers, n, delta, rows, delta.shape[-1], pos, w_g, kept_out,
                    count_out, stream)

    def inject_gated(self, kept, count, scene, prim, w, hidden, layers=1, stream=None):
        n = scene.numel() // layers
        lookme_inject_gated(self.handle, layers, n, kept, count, scene, prim, w, hidden,
                            hidden.shape[-1], stream)

    def inject_fused_gated(self, kept, count, scene, prim, w, hidden, layers=1, stream=None):
        n = scene.numel() // layers
        self.reserve(layers, n)
        lookme_inject_fused_gated(self.handle, layers, n, kept, count, scene, prim, w, hidden,
                                  hidden.shape[-1], stream)

    def inject_propagated_gated(self, kept, count, scene, prim, w, hidden, steps, stream=None):
        n = scene.numel()
        self.reserve(steps + 1, n)
        lookme_inject_propagated_gated(self.handle, steps, n, kept, count, scene, prim, w, hidden,
                                       hidden.shape[-1], stream)

    def close(self):
        if self.handle:
            lookme_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
