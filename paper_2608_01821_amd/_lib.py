"""ctypes binding of libdavet.so (the C ABI declared in include/davet.h).

Argument marshalling only: tensors are passed as device pointers, host
arrays as ctypes arrays, and every non-zero status raises DavetError with the
library's own message.  There is no fallback: if the shared library is
missing the import of this module fails.
"""

import ctypes as C
import os
import struct

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdavet.so")

DAVET_F32 = 0
DAVET_BF16 = 1
DAVET_F16 = 2
MAX_SEQS = 64


class DavetError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__("davet status %d: %s" % (status, msg))
        self.status = status


class ViewGeom(C.Structure):
    _fields_ = [("n_crops", C.c_int32), ("grid", C.c_int32), ("d", C.c_int32),
                ("K", C.c_int32), ("dtype", C.c_int32),
                ("mixed_stride", C.c_int32), ("realizer", C.c_int32)]


DAVET_REALIZER_POOL = 0
DAVET_REALIZER_PRUNE = 1
DAVET_REALIZER_MERGE = 2
MAX_REALIZER_GRID = 64


class ModelCfg(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d", C.c_int32),
                ("n_heads", C.c_int32), ("head_dim", C.c_int32),
                ("ffn", C.c_int32), ("vocab", C.c_int32),
                ("mask_id", C.c_int32), ("rms_eps", C.c_float),
                ("rope_theta", C.c_float), ("dtype", C.c_int32)]


class LayerWeights(C.Structure):
    _fields_ = [("wqkv", C.c_void_p), ("wo", C.c_void_p), ("wg", C.c_void_p),
                ("wu", C.c_void_p), ("wd", C.c_void_p),
                ("attn_norm", C.c_void_p), ("ffn_norm", C.c_void_p)]


class WeightsT(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("head", C.c_void_p),
                ("final_norm", C.c_void_p),
                ("layers", C.POINTER(LayerWeights)),
                ("head_layout", C.c_int32)]


DAVET_HEAD_ROWS = 0
DAVET_HEAD_TILED = 1


class Policy(C.Structure):
    _fields_ = [("B", C.c_double), ("rho", C.c_double), ("alpha", C.c_double),
                ("demand", C.c_double), ("early", C.c_int32), ("K", C.c_int32)]


class KvCacheT(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p),
                ("page_table", C.c_void_p), ("max_pages", C.c_int32),
                ("n_pages", C.c_int32), ("page_size", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("dtype", C.c_int32)]


MAX_PAGE_SIZE = 256
MAX_TOP = 64
MAX_TREE = 256
MAX_BEAMS = 64
TREE_WORDS = MAX_TREE // 32
DAVET_ROTARY_HALVES = 0
DAVET_ROTARY_PAIRS = 1
DAVET_ROTARY_PLAIN = 0
DAVET_ROTARY_LINEAR = 1
DAVET_ROTARY_BASE = 2
DAVET_ROTARY_RAMP = 3


if not os.path.exists(LIB_PATH):
    raise ImportError("libdavet.so is not built (%s); run "
                      "`python paper_2608_01821_amd/build.py`" % LIB_PATH)
_L = C.CDLL(LIB_PATH)

_vp = C.c_void_p
_i32 = C.c_int32
_i64 = C.c_int64
_P_i32 = C.POINTER(C.c_int32)
_P_f64 = C.POINTER(C.c_double)
_P_i64 = C.POINTER(C.c_int64)
_P_vp = C.POINTER(C.c_void_p)

_SIGS = {
    "davet_last_error": (C.c_char_p, []),
    "davet_version": (C.c_char_p, []),
    "davet_view_sizes": (C.c_int, [C.POINTER(ViewGeom), _P_i32]),
    "davet_view_map_sizes": (C.c_int, [C.POINTER(ViewGeom), _P_i32]),
    "davet_build_views": (C.c_int, [C.POINTER(ViewGeom), _vp, _P_vp, _P_vp,
                                    _P_vp, _vp, C.c_size_t, _vp]),
    "davet_build_views_static": (C.c_int, [C.POINTER(ViewGeom), _vp, _P_vp,
                                           _P_vp, _P_vp, _vp]),
    "davet_views_scratch_bytes": (C.c_int, [C.POINTER(ViewGeom),
                                            C.POINTER(C.c_size_t)]),
    "davet_realizer_key_count": (C.c_int, [C.POINTER(ViewGeom), _P_i32]),
    "davet_realizer_keys": (C.c_int, [C.POINTER(ViewGeom), _vp, _vp, _vp]),
    "davet_realizer_maps": (C.c_int, [C.POINTER(ViewGeom), _vp, _P_vp, _P_vp,
                                      _vp]),
    "davet_convert": (C.c_int, [_vp, _i32, _vp, _i32, C.c_size_t, _vp]),
    "davet_head_tiled_elems": (C.c_size_t, [_i32, _i32]),
    "davet_pack_head": (C.c_int, [_vp, _vp, _i32, _i32, _i32, _vp]),
    "davet_workspace_bytes": (C.c_int, [C.POINTER(ModelCfg), _i32, _i32, _i32,
                                        C.POINTER(C.c_size_t)]),
    "davet_denoise_step": (C.c_int, [C.POINTER(ModelCfg), C.POINTER(WeightsT),
                                     _i32, _P_vp, _P_i32, _vp, _P_i32, _vp,
                                     _vp, _i32, _vp, _vp, _vp, _vp, C.c_size_t,
                                     _vp]),
    "davet_fp16_overflow_count": (C.c_int, [_vp, _P_i32, _vp]),
    "davet_set_attention_split": (C.c_int, [_i32]),
    "davet_unmask": (C.c_int, [_i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp,
                               _vp]),
    "davet_demand_prior": (C.c_double, [_i32]),
    "davet_parse_operation": (C.c_int, [C.c_char_p, _P_i32]),
    "davet_policy_envelope": (C.c_int, [C.POINTER(Policy), _i32, _P_f64,
                                        _P_f64]),
    "davet_policy_step": (C.c_int, [C.POINTER(Policy), _i32, _i32, _P_f64,
                                    _P_f64, C.c_double, C.c_double, _P_f64,
                                    _P_i32, _P_f64]),
    "davet_step_stats": (C.c_int, [_i32, C.POINTER(C.c_float), _P_i32, _P_i32,
                                   C.POINTER(C.c_uint8), _P_f64, _P_f64]),
    "davet_policy_step_device": (C.c_int, [_i32, _i32, _i32, _i32,
                                           C.POINTER(Policy), _P_f64, _P_f64,
                                           _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                           _vp]),
    "davet_run_schedule": (C.c_int, [C.POINTER(ModelCfg), C.POINTER(WeightsT),
                                     _i32, C.POINTER(ViewGeom), _P_vp, _P_vp,
                                     _vp, _P_i32, _i32, _i32, _i32,
                                     C.POINTER(Policy), _P_i32, _vp, _vp,
                                     _P_i32, _P_f64, _vp, _vp, _vp, _vp,
                                     C.c_size_t, _vp]),
    "davet_mailbox_create": (C.c_int, [_P_vp]),
    "davet_mailbox_destroy": (C.c_int, [_vp]),
    "davet_set_wait_limit": (C.c_int, [C.c_double]),
    "davet_cache_append": (C.c_int, [C.POINTER(KvCacheT), _i32, _P_i32, _P_i32,
                                     _vp, _i64, _i32, _vp, _i32, _vp, _vp,
                                     C.c_float, C.c_float, _vp, _i64, _vp]),
    "davet_cache_workspace_bytes": (C.c_int, [_i32, _i32, _i32,
                                              C.POINTER(C.c_size_t)]),
    "davet_cache_attention": (C.c_int, [C.POINTER(KvCacheT), _i32, _P_i32,
                                        _P_i32, _vp, _i64, _i32, C.c_float,
                                        _i32, _vp, _i64, _vp, _vp, C.c_size_t,
                                        _vp]),
    "davet_cache_weights": (C.c_int, [C.POINTER(KvCacheT), _i32, _P_i32, _P_i32,
                                      _vp, _i64, _i32, C.c_float, _i32, _vp,
                                      _vp, _vp, _i64, _vp, C.c_size_t, _vp]),
    "davet_tree_plan": (C.c_int, [_i32, _P_i32, _P_i32, _P_i32, _vp, _vp, _vp,
                                  _vp]),
    "davet_cache_tree_attention": (C.c_int, [C.POINTER(KvCacheT), _i32, _P_i32,
                                             _P_i32, _vp, _i64, _i32, C.c_float,
                                             _vp, _vp, _i64, _vp, _vp,
                                             C.c_size_t, _vp]),
    "davet_cache_page_bounds": (C.c_int, [C.POINTER(KvCacheT), _i32, _P_i32,
                                          _P_i32, _vp, _vp]),
    "davet_cache_page_select": (C.c_int, [C.POINTER(KvCacheT), _i32, _P_i32,
                                          _P_i32, _vp, _i64, _i32, _i32, _vp,
                                          _i32, _i32, _i32, _vp, _vp]),
    "davet_cache_page_attention": (C.c_int, [C.POINTER(KvCacheT), _i32, _P_i32,
                                             _P_i32, _vp, _i64, _i32, C.c_float,
                                             _i32, _vp, _i32, _vp, _i64, _vp,
                                             _vp, C.c_size_t, _vp]),
    "davet_beam_workspace_bytes": (C.c_int, [_i32, _i32, _i32, _i32,
                                             C.POINTER(C.c_size_t)]),
    "davet_beam_select": (C.c_int, [_i32, _i32, _i32, _vp, _i32, _i64, _i32, _vp,
                                    _vp, _i32, _i32, _vp, _vp, _vp, _vp,
                                    C.c_size_t, _vp]),
    "davet_cache_reorder": (C.c_int, [C.POINTER(KvCacheT), _i32, _P_i32, _vp, _vp,
                                      _vp, _i32, _vp]),
    "davet_rotary_turns": (C.c_int, [_i32, C.c_double, _i32, C.c_double,
                                     C.c_double, C.c_double, C.c_double,
                                     _P_f64]),
    "davet_rotary": (C.c_int, [_i32, _i32, _i32, _i32, _i32, _vp, _i64, _vp,
                               _i64, _i32, _vp, _vp, C.c_float, _i32, _vp]),
    "davet_evict_select": (C.c_int, [_i32, _P_i32, _P_i32, _vp, _i64, _i32,
                                     _i32, _vp, _i64, _vp, _i64, _vp]),
    "davet_cache_gather": (C.c_int, [C.POINTER(KvCacheT), _i32, _P_i32, _vp,
                                     _i64, _vp, _i32, _vp]),
    "davet_logprobs_workspace_bytes": (C.c_int, [_i32, _i32, _i32,
                                                 C.POINTER(C.c_size_t)]),
    "davet_token_logprobs": (C.c_int, [_i32, _i32, _vp, _i32, _i64, _i32, _vp,
                                       _vp, _vp, _i32, _vp, _vp, _vp,
                                       C.c_size_t, _vp]),
    "davet_prof_enable": (C.c_int, [_i32]),
    "davet_prof_reset": (C.c_int, []),
    "davet_prof_only": (C.c_int, [_i32]),
    "davet_prof_read": (C.c_int, [_i32, _P_i64, _P_f64]),
    "davet_prof_class_name": (C.c_char_p, [_i32]),
}

for _name, (_res, _args) in _SIGS.items():
    _f = getattr(_L, _name)
    _f.restype = _res
    _f.argtypes = _args

EXPORTED = tuple(_SIGS)


class _ByBytes:
    """The calls that take host lists as _words gives them: functions of their own, so
    that raw()'s take int32 arrays and nothing else."""


for _name in ("davet_cache_append", "davet_cache_attention", "davet_cache_weights",
              "davet_tree_plan", "davet_cache_tree_attention",
              "davet_cache_page_bounds", "davet_cache_page_select",
              "davet_cache_page_attention", "davet_cache_reorder"):
    _f = _L[_name]
    _f.restype, _args = _SIGS[_name]
    _f.argtypes = [C.c_char_p if _a is _P_i32 else _a for _a in _args]
    setattr(_ByBytes, _name, _f)


def raw():
    """The loaded ctypes library."""
    return _L


def _check(status):
    if status != 0:
        raise DavetError(status, _L.davet_last_error().decode())
    return status


def _ptr(t):
    """Device (or host) address of a tensor, or None.  The library reads
    every buffer as dense, so a strided view is refused."""
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("davet: tensor arguments must be contiguous")
    return C.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:
        import torch
        return C.c_void_p(torch.cuda.current_stream().cuda_stream)
    if isinstance(stream, int):
        return C.c_void_p(stream)
    return C.c_void_p(stream.cuda_stream)


def _addr(t):
    """Integer address of a dense tensor, or None."""
    p = _ptr(t)
    return None if p is None else p.value


def _ptr_array(items):
    arr = (C.c_void_p * max(1, len(items)))()
    for i, t in enumerate(items):
        if t is None or isinstance(t, int):
            arr[i] = t
        else:
            if not t.is_contiguous():
                raise ValueError("davet: tensor arguments must be contiguous")
            arr[i] = t.data_ptr()
    return arr


def _i32_array(vals):
    arr = (C.c_int32 * max(1, len(vals)))()
    for i, v in enumerate(vals):
        arr[i] = int(v)
    return arr


class Weights:
    """Holds the davet_weights struct and keeps the tensors it points to
    alive.  ``layers`` is a list of dicts with tensors wqkv, wo, wg, wu, wd
    and optional attn_norm / ffn_norm (float32).  ``head`` is row-major
    [vocab, d], or the output of davet_pack_head with
    head_layout=DAVET_HEAD_TILED."""

    def __init__(self, embed, head, layers, final_norm=None,
                 head_layout=DAVET_HEAD_ROWS):
        self._keep = [embed, head, final_norm, layers]
        self._layers = (LayerWeights * max(1, len(layers)))()
        for i, lw in enumerate(layers):
            self._layers[i] = LayerWeights(
                _addr(lw["wqkv"]), _addr(lw["wo"]), _addr(lw["wg"]),
                _addr(lw["wu"]), _addr(lw["wd"]), _addr(lw.get("attn_norm")),
                _addr(lw.get("ffn_norm")))
        self.struct = WeightsT(_addr(embed), _addr(head), _addr(final_norm),
                               self._layers, int(head_layout))


def davet_version():
    return _L.davet_version().decode()


def davet_view_sizes(geom: ViewGeom):
    out = (C.c_int32 * geom.K)()
    _check(_L.davet_view_sizes(C.byref(geom), out))
    return list(out)


def davet_view_map_sizes(geom: ViewGeom):
    out = (C.c_int32 * geom.K)()
    _check(_L.davet_view_map_sizes(C.byref(geom), out))
    return list(out)


def davet_views_scratch_bytes(geom):
    out = C.c_size_t(0)
    _check(_L.davet_views_scratch_bytes(C.byref(geom), C.byref(out)))
    return int(out.value)


def davet_build_views(geom, v, levels, offsets=None, members=None,
                      scratch=None, stream=None):
    """``scratch``: a device tensor of davet_views_scratch_bytes bytes; when
    None and the realizer needs one, a torch buffer on v's device."""
    K = geom.K
    lv = _ptr_array(list(levels) + [None] * (K - len(levels)))
    off = _ptr_array(offsets) if offsets is not None else None
    mem = _ptr_array(members) if members is not None else None
    if scratch is None:
        nb = davet_views_scratch_bytes(geom)
        if nb:
            import torch
            scratch = torch.empty(nb, dtype=torch.uint8, device=v.device)
    nbytes = 0 if scratch is None else scratch.numel() * scratch.element_size()
    _check(_L.davet_build_views(C.byref(geom), _ptr(v), lv, off, mem,
                                _ptr(scratch), nbytes, _stream(stream)))


STATIC_SCRATCH_BYTES = 4 << 20


def davet_build_views_static(geom, v, levels, offsets=None, members=None,
                             stream=None):
    """davet_build_views with the library's own device scratch (no
    allocation by the library or by this binding)."""
    K = geom.K
    lv = _ptr_array(list(levels) + [None] * (K - len(levels)))
    off = _ptr_array(offsets) if offsets is not None else None
    mem = _ptr_array(members) if members is not None else None
    _check(_L.davet_build_views_static(C.byref(geom), _ptr(v), lv, off, mem,
                                       _stream(stream)))


def davet_realizer_key_count(geom):
    out = C.c_int32(0)
    _check(_L.davet_realizer_key_count(C.byref(geom), C.byref(out)))
    return int(out.value)


def davet_realizer_keys(geom, v, keys, stream=None):
    _check(_L.davet_realizer_keys(C.byref(geom), _ptr(v), _ptr(keys),
                                  _stream(stream)))


def davet_realizer_maps(geom, keys, offsets=None, members=None, stream=None):
    K = geom.K
    off = _ptr_array(list(offsets) + [None] * (K - len(offsets))) \
        if offsets is not None else None
    mem = _ptr_array(list(members) + [None] * (K - len(members))) \
        if members is not None else None
    _check(_L.davet_realizer_maps(C.byref(geom), _ptr(keys), off, mem,
                                  _stream(stream)))


def davet_convert(src, src_dtype, dst, dst_dtype, n=None, stream=None):
    n = src.numel() if n is None else n
    _check(_L.davet_convert(_ptr(src), int(src_dtype), _ptr(dst),
                            int(dst_dtype), int(n), _stream(stream)))


def davet_head_tiled_elems(vocab, d):
    return int(_L.davet_head_tiled_elems(int(vocab), int(d)))


def davet_pack_head(src, dst, vocab, d, dtype, stream=None):
    _check(_L.davet_pack_head(_ptr(src), _ptr(dst), int(vocab), int(d),
                              int(dtype), _stream(stream)))


def davet_workspace_bytes(cfg, max_tokens, max_seqs, L):
    out = C.c_size_t(0)
    _check(_L.davet_workspace_bytes(C.byref(cfg), int(max_tokens),
                                    int(max_seqs), int(L), C.byref(out)))
    return out.value


def davet_denoise_step(cfg, weights: Weights, views, n_view, prompt_ids,
                       cu_prompt, resp_ids, resp_masked, L, conf_out,
                       argmax_out, logits_out, workspace, stream=None):
    n = len(views)
    _check(_L.davet_denoise_step(
        C.byref(cfg), C.byref(weights.struct), n, _ptr_array(views),
        _i32_array(n_view), _ptr(prompt_ids), _i32_array(cu_prompt),
        _ptr(resp_ids), _ptr(resp_masked), int(L), _ptr(conf_out),
        _ptr(argmax_out), _ptr(logits_out), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream)))


def davet_fp16_overflow_count(workspace, stream=None) -> int:
    """Non-finite 16-bit projection outputs stored by the last step (or
    schedule) that ran on `workspace`; waits for `stream`."""
    out = C.c_int32(0)
    _check(_L.davet_fp16_overflow_count(_ptr(workspace), C.byref(out),
                                        _stream(stream)))
    return out.value


def davet_set_attention_split(mode):
    """Attention key-range split: 0 automatic, 1 off, 2..8 forced."""
    _check(_L.davet_set_attention_split(int(mode)))


def davet_unmask(n_seqs, L, k, conf, argmax, resp_ids, resp_masked,
                 selected=None, stream=None):
    _check(_L.davet_unmask(int(n_seqs), int(L), int(k), _ptr(conf),
                           _ptr(argmax), _ptr(resp_ids), _ptr(resp_masked),
                           _ptr(selected), _stream(stream)))


def davet_demand_prior(category):
    return _L.davet_demand_prior(int(category))


def davet_parse_operation(query: str) -> int:
    out = C.c_int32(-1)
    _check(_L.davet_parse_operation(query.encode("utf-8"), C.byref(out)))
    return out.value


def davet_policy_envelope(pol: Policy, T):
    lo = (C.c_double * T)()
    up = (C.c_double * T)()
    _check(_L.davet_policy_envelope(C.byref(pol), int(T), lo, up))
    return list(lo), list(up)


def davet_policy_step(pol: Policy, t, T, lower, upper, cbar_prev, churn_prev):
    lo = (C.c_double * T)(*lower)
    up = (C.c_double * T)(*upper)
    b = C.c_double(0)
    lv = C.c_int32(0)
    r = C.c_double(0)
    _check(_L.davet_policy_step(C.byref(pol), int(t), int(T), lo, up,
                                float(cbar_prev), float(churn_prev),
                                C.byref(b), C.byref(lv), C.byref(r)))
    return b.value, lv.value, r.value


def davet_step_stats(conf, argmax, argmax_prev, masked_after):
    conf = np.ascontiguousarray(conf, dtype=np.float32)
    am = np.ascontiguousarray(argmax, dtype=np.int32)
    m = np.ascontiguousarray(masked_after, dtype=np.uint8)
    prev = None if argmax_prev is None else \
        np.ascontiguousarray(argmax_prev, dtype=np.int32)
    cb = C.c_double(0)
    ch = C.c_double(0)
    _check(_L.davet_step_stats(
        len(conf), conf.ctypes.data_as(C.POINTER(C.c_float)),
        am.ctypes.data_as(_P_i32),
        None if prev is None else prev.ctypes.data_as(_P_i32),
        m.ctypes.data_as(C.POINTER(C.c_uint8)), C.byref(cb), C.byref(ch)))
    return cb.value, ch.value


def davet_policy_step_device(pols, t, T, lower, upper, conf, argmax,
                             argmax_prev, masked_after, level_out, budget_out,
                             r_out=None, stream=None):
    """lower/upper: host float64 [n_seqs * T]; the other arrays are device
    tensors ([n_seqs * L] inputs, [n_seqs] outputs)."""
    n = len(pols)
    L = conf.numel() // n
    p = (Policy * n)(*pols)
    lo = np.ascontiguousarray(lower, dtype=np.float64)
    up = np.ascontiguousarray(upper, dtype=np.float64)
    _check(_L.davet_policy_step_device(
        n, L, int(t), int(T), p, lo.ctypes.data_as(_P_f64),
        up.ctypes.data_as(_P_f64), _ptr(conf), _ptr(argmax), _ptr(argmax_prev),
        _ptr(masked_after), _ptr(level_out), _ptr(budget_out), _ptr(r_out),
        _stream(stream)))


class Mailbox:
    """A davet_mailbox (pinned host memory the policy-mode loop writes the
    next levels into), made once and freed by close() or at exit."""

    def __init__(self):
        h = C.c_void_p()
        _check(_L.davet_mailbox_create(C.byref(h)))
        self.handle = h

    def close(self):
        if self.handle is not None and self.handle.value:
            h, self.handle = self.handle, None
            _check(_L.davet_mailbox_destroy(h))

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


_MAILBOX = None


def default_mailbox():
    """The process's mailbox, made on first use (a set-up step, not part of
    a loop's steady state)."""
    global _MAILBOX
    if _MAILBOX is None:
        _MAILBOX = Mailbox()
    return _MAILBOX


def davet_set_wait_limit(seconds):
    _check(_L.davet_set_wait_limit(float(seconds)))


def davet_run_schedule(cfg, weights: Weights, geoms, visual, view_bufs,
                       prompt_ids, cu_prompt, L, T, k, pols, fixed_levels,
                       resp_ids, resp_masked, workspace, conf_trace=None,
                       argmax_trace=None, stream=None, mailbox=None):
    """Returns (levels [n_seqs*T], budgets [n_seqs*T]) as host lists.
    ``mailbox``: a Mailbox; in policy mode the process's default one when
    None."""
    n = len(visual)
    g = (ViewGeom * n)(*geoms)
    p = (Policy * n)(*pols) if pols is not None else None
    fl = _i32_array(np.asarray(fixed_levels).reshape(-1)) \
        if fixed_levels is not None else None
    lv = (C.c_int32 * (n * T))()
    bu = (C.c_double * (n * T))()
    if mailbox is None and pols is not None:
        mailbox = default_mailbox()
    mb = None if mailbox is None else mailbox.handle
    _check(_L.davet_run_schedule(
        C.byref(cfg), C.byref(weights.struct), n, g, _ptr_array(visual),
        _ptr_array(view_bufs), _ptr(prompt_ids), _i32_array(cu_prompt),
        int(L), int(T), int(k), p, fl, _ptr(resp_ids), _ptr(resp_masked),
        lv, bu, _ptr(conf_trace), _ptr(argmax_trace), mb, _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream)))
    return list(lv), list(bu)


# ---- paged cache and token log probabilities.  These take row-strided tensors
# (last dimension dense) and check that each is of the type that the call takes
# and holds what it reads or writes; without `stream` they run on the current
# stream of their tensors' device, whichever device is current.

_torch = None
_FLOAT = _INT = _DOUBLE = ()    # torch types of float32, int32, float64 arguments
_BITS = ()                  # and of 32-bit masks
_KINDS = {}                 # of a davet_dtype's: 16 bits also as bit patterns
_device = _raw_stream = None    # the current device; a device's current stream


def _load_torch():
    global _torch, _FLOAT, _INT, _DOUBLE, _BITS, _device, _raw_stream
    import torch
    # torch's own short cuts where it has them: torch.cuda.current_stream() builds
    # an object, 2 us
    _device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                          lambda dev: torch.cuda.current_stream(dev).cuda_stream)
    _FLOAT, _INT, _DOUBLE = (torch.float32,), (torch.int32,), (torch.float64,)
    _BITS = _INT + ((torch.uint32,) if hasattr(torch, "uint32") else ())
    bits = (torch.int16,) + ((torch.uint16,) if hasattr(torch, "uint16") else ())
    _KINDS.update({DAVET_F32: _FLOAT, DAVET_BF16: (torch.bfloat16,) + bits,
                   DAVET_F16: (torch.float16,) + bits})
    _torch = torch


def _kinds(dtype):
    """The torch types that hold a davet_dtype."""
    if _torch is None:
        _load_torch()
    if dtype not in _KINDS:
        raise DavetError(-3, "dtype must be DAVET_F32, DAVET_BF16 or DAVET_F16")
    return _KINDS[dtype]


def _wrong_type(t, kinds, name):
    return ValueError("davet: %s is of %s, not of %s"
                      % (name, t.dtype, " or ".join(str(k) for k in kinds)))


def _rows(t, width, n_rows, kinds, name):
    """(address, row stride in elements) of a 2-D tensor of a type in `kinds` whose
    rows are dense and hold `width` elements."""
    if t.dtype not in kinds:
        raise _wrong_type(t, kinds, name)
    shape = t.shape
    if len(shape) != 2:
        raise ValueError("davet: %s must be 2-D" % name)
    n, w = shape
    if n < n_rows or w < width:
        raise ValueError("davet: %s must hold [%d, %d]" % (name, n_rows, width))
    ld, one = t.stride()
    if one != 1 and w > 1:
        raise ValueError("davet: the rows of %s must be dense" % name)
    if n < 2:
        ld = width              # one row: whatever its tensor's stride
    elif ld < width:
        raise ValueError("davet: the rows of %s overlap" % name)
    return t.data_ptr(), ld


def _dense(t, n, kinds, name):
    """Address of a dense tensor of at least `n` elements of a type in `kinds`, or
    None."""
    if t is None:
        return None
    if t.dtype not in kinds:
        raise _wrong_type(t, kinds, name)
    if t.numel() < n or not t.is_contiguous():
        raise ValueError("davet: %s must be dense, with %d elements" % (name, n))
    return t.data_ptr()


def _space(t):
    """(address, bytes) of a workspace."""
    if t is None:
        return None, 0
    if not t.is_contiguous():
        raise ValueError("davet: the workspace must be dense")
    return t.data_ptr(), t.nbytes


_PACK = [(struct.Struct("%di" % n).pack, (C.c_int32 * n).from_buffer_copy)
         for n in range(MAX_SEQS + 2)]


def _ints(vals):
    """A host list as an array of int32."""
    if isinstance(vals, C.Array):
        return vals
    n = len(vals)
    # (filled element by element a ctypes array takes 2^32 + 3 for 3, and 4 us for
    # 65 of them; so 0.6)
    pack, make = _PACK[n] if n < len(_PACK) else \
        (struct.Struct("%di" % n).pack, (C.c_int32 * n).from_buffer_copy)
    try:
        return make(pack(*vals))
    except struct.error as e:
        raise ValueError("davet: host lists must hold 32-bit integers (%s)" % e)


_WORDS = [struct.Struct("%di" % n).pack for n in range(MAX_SEQS + 2)]


def _words(vals):
    """The same as bytes, for calls that take no copy of it: with its conversion to an
    argument 0.3 us a list less."""
    n = len(vals)
    try:
        return (_WORDS[n] if n < len(_WORDS) else struct.Struct("%di" % n).pack)(*vals)
    except struct.error as e:
        raise ValueError("davet: host lists must hold 32-bit integers (%s)" % e)


def _small(v, name):
    """A host integer that fits int32 (ctypes would keep its low 32 bits)."""
    if not -0x80000000 <= v <= 0x7fffffff:
        raise ValueError("davet: %s must be a 32-bit integer" % name)
    return v


def _too_large():
    raise ValueError("davet: a tensor's sizes must be 32-bit integers")


def _gpu(first, *tensors):
    """Index of the GPU that holds all tensors (None entries aside)."""
    dev = first.get_device()
    if dev < 0:
        raise ValueError("davet: tensor arguments must be on a GPU")
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError("davet: tensor arguments must be on one GPU")
    return dev


def _launch(dev, stream, fn, *args):
    """fn(*args, stream handle) with GPU `dev` current; without `stream`, on its
    current one."""
    if dev != _device():                # (a tensor is there: initialised)
        with _torch.cuda.device(dev):
            return _launch(dev, stream, fn, *args)
    if stream is None:
        stream = _raw_stream(dev)
    elif not isinstance(stream, int):
        stream = stream.cuda_stream
    status = fn(*args, stream)
    if status:
        _check(status)


class KvCache:
    """A davet_kv_cache: ``k`` and ``v`` [n_pages, n_kv_heads, page_size,
    head_dim] (``v`` may be None for davet_cache_weights) and ``page_table``
    int32 [n_seqs, max_pages], dense device tensors, which it keeps alive."""

    def __init__(self, k, v, page_table, dtype):
        kinds = _kinds(dtype)
        if k.dim() != 4 or (v is not None and v.shape != k.shape) or \
                page_table.dim() != 2:
            raise ValueError("davet: k and v must be [n_pages, n_kv_heads, "
                             "page_size, head_dim] alike, page_table [n_seqs, "
                             "max_pages]")
        if max(*k.shape, page_table.shape[1]) >> 31:
            _too_large()
        addr = (_dense(k, 0, kinds, "k"), _dense(v, 0, kinds, "v"),
                _dense(page_table, 0, _INT, "page_table"))
        self.k, self.v, self.page_table = k, v, page_table
        self.n_seqs, self.head_dim, self.kinds = len(page_table), k.shape[3], kinds
        self.n_kv_heads, self.page_size = k.shape[1], k.shape[2]
        self.struct = KvCacheT(*addr, page_table.shape[1], k.shape[0], k.shape[2],
                               k.shape[1], k.shape[3], int(dtype))
        self._ref = C.byref(self.struct)
        devs = {x.get_device() for x in (k, v, page_table) if x is not None}
        self._dev = devs.pop() if len(devs) == 1 else -1     # its tensors' GPU, or -1

    def _chunk(self, cu_q, kv_len):
        n = len(kv_len)
        if len(cu_q) != n + 1 or n > self.n_seqs:
            raise ValueError("davet: cu_q needs an entry more than kv_len, and "
                             "page_table a row for each of those")
        return n, _words(cu_q), _words(kv_len), max(0, cu_q[n])

    def _gpu(self, *tensors):
        dev = self._dev
        if dev < 0:
            return _gpu(self.k, self.v, self.page_table, *tensors)
        for t in tensors:
            if t is not None and t.get_device() != dev:
                raise ValueError("davet: tensor arguments must be on one GPU")
        return dev


def davet_cache_append(cache: KvCache, cu_q, kv_len, qkv, n_heads, q_out,
                       pos=None, norm=False, q_gain=None, k_gain=None, eps=1e-6,
                       theta=10000.0, stream=None):
    n, cu, kv, rows = cache._chunk(cu_q, kv_len)
    n_heads, D, kinds = _small(n_heads, "n_heads"), cache.head_dim, cache.kinds
    x, ldx = _rows(qkv, (n_heads + 2 * cache.n_kv_heads) * D, rows, kinds, "qkv")
    q, ldq = _rows(q_out, n_heads * D, rows, kinds, "q_out")
    p = _dense(pos, rows, _INT, "pos")
    gq, gk = _dense(q_gain, D, _FLOAT, "q_gain"), _dense(k_gain, D, _FLOAT, "k_gain")
    _launch(cache._gpu(qkv, q_out, pos, q_gain, k_gain), stream,
            _ByBytes.davet_cache_append, cache._ref, n, cu, kv, x, ldx, n_heads, p,
            1 if norm else 0, gq, gk, eps, theta, q, ldq)


def davet_cache_workspace_bytes(n_heads, head_dim, max_q):
    out = C.c_size_t(0)
    _check(_L.davet_cache_workspace_bytes(
        _small(int(n_heads), "n_heads"), _small(int(head_dim), "head_dim"),
        _small(int(max_q), "max_q"), C.byref(out)))
    return out.value


def davet_cache_attention(cache: KvCache, cu_q, kv_len, q, n_heads, out,
                          lse=None, scale=0.0, block=0, workspace=None,
                          stream=None):
    n, cu, kv, rows = cache._chunk(cu_q, kv_len)
    n_heads, block = _small(n_heads, "n_heads"), _small(block, "block")
    width = n_heads * cache.head_dim
    x, ldx = _rows(q, width, rows, cache.kinds, "q")
    o, ldo = _rows(out, width, rows, cache.kinds, "out")
    e, (ws, nb) = _dense(lse, rows * n_heads, _FLOAT, "lse"), _space(workspace)
    _launch(cache._gpu(q, out, lse, workspace), stream, _ByBytes.davet_cache_attention,
            cache._ref, n, cu, kv, x, ldx, n_heads, scale, block, o, ldo, e, ws, nb)


def davet_cache_weights(cache: KvCache, cu_q, kv_len, q, n_heads, lse, weights,
                        prev=None, scale=0.0, block=0, workspace=None,
                        stream=None):
    n, cu, kv, rows = cache._chunk(cu_q, kv_len)
    n_heads, block = _small(n_heads, "n_heads"), _small(block, "block")
    most = max(kv_len)
    x, ldx = _rows(q, n_heads * cache.head_dim, rows, cache.kinds, "q")
    w, ldw = _rows(weights, most, n, _FLOAT, "weights")
    p = None
    if prev is not None:
        p, ldp = _rows(prev, most, n, _FLOAT, "prev")
        if ldp != ldw and n > 1:
            raise ValueError("davet: prev and weights need one row stride")
    e, (ws, nb) = _dense(lse, rows * n_heads, _FLOAT, "lse"), _space(workspace)
    _launch(cache._gpu(q, lse, weights, prev, workspace), stream,
            _ByBytes.davet_cache_weights, cache._ref, n, cu, kv, x, ldx, n_heads, scale,
            block, e, p, w, ldw, ws, nb)


def davet_evict_select(n, keep, weights, kept, first=0, last=0,
                       weights_out=None, stream=None):
    """``n`` and ``keep``: host lists, one entry a sequence."""
    seqs = len(n)
    if seqs != len(keep) or seqs == 0:
        raise ValueError("davet: n and keep need one entry a sequence")
    most = max(keep)
    if _torch is None:
        _load_torch()
    w, ldw = _rows(weights, max(n), seqs, _FLOAT, "weights")
    k, ldk = _rows(kept, most, seqs, _INT, "kept")
    o, ldo = (None, 0) if weights_out is None else \
        _rows(weights_out, most, seqs, _FLOAT, "weights_out")
    first, last = _small(first, "first"), _small(last, "last")
    _launch(_gpu(weights, kept, weights_out), stream, _L.davet_evict_select, seqs,
            _ints(n), _ints(keep), w, ldw, first, last, k, ldk, o, ldo)


def davet_cache_gather(cache: KvCache, kept, keep, dst_table, stream=None):
    """``keep``: host list; ``dst_table``: dense int32 [n_seqs, pages]."""
    n = len(keep)
    if n == 0 or n > cache.n_seqs or dst_table.dim() != 2 or len(dst_table) < n:
        raise ValueError("davet: the page tables need a row a sequence")
    if dst_table.shape[1] >> 31:
        _too_large()
    k, ldk = _rows(kept, max(keep), n, _INT, "kept")
    dst = _dense(dst_table, 0, _INT, "dst_table")
    _launch(cache._gpu(kept, dst_table), stream, _L.davet_cache_gather, cache._ref,
            n, _ints(keep), k, ldk, dst, dst_table.shape[1])


def davet_logprobs_workspace_bytes(rows, vocab, top):
    out = C.c_size_t(0)
    _check(_L.davet_logprobs_workspace_bytes(
        _small(int(rows), "rows"), _small(int(vocab), "vocab"),
        _small(int(top), "top"), C.byref(out)))
    return out.value


def davet_token_logprobs(logits, dtype, targets=None, logp=None, entropy=None,
                         top_logp=None, top_ids=None, exclude=-1,
                         workspace=None, stream=None):
    """``logits`` [rows, vocab]; ``top_logp`` and ``top_ids`` [rows, top], dense
    (both or neither)."""
    rows, vocab = logits.shape
    if (rows | vocab) >> 31:
        _too_large()
    x, ld = _rows(logits, vocab, rows, _kinds(dtype), "logits")
    g, lp = _dense(targets, rows, _INT, "targets"), _dense(logp, rows, _FLOAT, "logp")
    en = _dense(entropy, rows, _FLOAT, "entropy")
    top, tl, ti = 0, None, None
    if top_ids is not None or top_logp is not None:
        if top_ids is None or top_logp is None or top_ids.dim() != 2 or \
                top_ids.shape != top_logp.shape:
            raise ValueError("davet: top_logp and top_ids must be [rows, top]")
        top = top_ids.shape[1]
        if top >> 31:
            _too_large()
        tl = _dense(top_logp, rows * top, _FLOAT, "top_logp")
        ti = _dense(top_ids, rows * top, _INT, "top_ids")
    exclude, (ws, nb) = _small(exclude, "exclude"), _space(workspace)
    _launch(_gpu(logits, targets, logp, entropy, top_logp, top_ids, workspace),
            stream, _L.davet_token_logprobs, rows, vocab, x, int(dtype), ld,
            exclude, g, lp, en, top, tl, ti, ws, nb)


# ---- a tree of drafted tokens

def davet_tree_plan(cu_q, kv_len, parent, pos=None, mask=None, first_pos=None,
                    stream=None):
    """``cu_q``, ``kv_len`` and ``first_pos``: host lists; ``parent`` and ``pos``
    dense int32 [rows], ``mask`` dense int32 (or uint32) [rows, TREE_WORDS]."""
    n = len(cu_q) - 1
    if n < 1 or (kv_len is None and first_pos is None) or \
            (kv_len is not None and len(kv_len) != n) or \
            (first_pos is not None and len(first_pos) != n):
        raise ValueError("davet: cu_q needs an entry more than kv_len and first_pos")
    if _torch is None:
        _load_torch()
    rows = max(0, cu_q[n])
    up, p = _dense(parent, rows, _INT, "parent"), _dense(pos, rows, _INT, "pos")
    m = _dense(mask, rows * TREE_WORDS, _BITS, "mask")
    cu, kv = _words(cu_q), None if kv_len is None else _words(kv_len)
    first = None if first_pos is None else _words(first_pos)
    _launch(_gpu(parent, pos, mask), stream, _ByBytes.davet_tree_plan, n, cu, kv,
            first, up, p, m)


def davet_cache_tree_attention(cache: KvCache, cu_q, kv_len, q, n_heads, mask, out,
                               lse=None, scale=0.0, workspace=None, stream=None):
    n, cu, kv, rows = cache._chunk(cu_q, kv_len)
    n_heads, width = _small(n_heads, "n_heads"), n_heads * cache.head_dim
    x, ldx = _rows(q, width, rows, cache.kinds, "q")
    o, ldo = _rows(out, width, rows, cache.kinds, "out")
    m = _dense(mask, rows * TREE_WORDS, _BITS, "mask")
    e, (ws, nb) = _dense(lse, rows * n_heads, _FLOAT, "lse"), _space(workspace)
    _launch(cache._gpu(q, mask, out, lse, workspace), stream,
            _ByBytes.davet_cache_tree_attention, cache._ref, n, cu, kv, x, ldx, n_heads,
            scale, m, o, ldo, e, ws, nb)


# ---- attention over selected pages

def _page_bounds(cache, bounds):
    """Address of a cache's bounds [n_pages, n_kv_heads, 2, head_dim]."""
    s = cache.struct
    return _dense(bounds, s.n_pages * s.n_kv_heads * 2 * s.head_dim, cache.kinds,
                  "bounds")


def _page_list(cache, pages, rows):
    """(address, top) of pages [rows, n_kv_heads, top]."""
    shape = pages.shape
    if len(shape) != 3 or shape[0] < rows or shape[1] != cache.n_kv_heads:
        raise ValueError("davet: pages must be [rows, n_kv_heads, top]")
    if shape[2] >> 31:
        _too_large()
    return _dense(pages, 0, _INT, "pages"), shape[2]


def davet_cache_page_bounds(cache: KvCache, cu_q, kv_len, bounds, stream=None):
    """``bounds``: dense [n_pages, n_kv_heads, 2, head_dim] of the cache's type."""
    n, cu, kv, _ = cache._chunk(cu_q, kv_len)
    b = _page_bounds(cache, bounds)
    _launch(cache._gpu(bounds), stream, _ByBytes.davet_cache_page_bounds, cache._ref,
            n, cu, kv, b)


def davet_cache_page_select(cache: KvCache, cu_q, kv_len, q, n_heads, bounds, pages,
                            first=0, last=0, block=0, stream=None):
    """``pages``: dense int32 [rows, n_kv_heads, top]."""
    n, cu, kv, rows = cache._chunk(cu_q, kv_len)
    n_heads, block = _small(n_heads, "n_heads"), _small(block, "block")
    first, last = _small(first, "first"), _small(last, "last")
    x, ldx = _rows(q, n_heads * cache.head_dim, rows, cache.kinds, "q")
    b, (p, top) = _page_bounds(cache, bounds), _page_list(cache, pages, rows)
    _launch(cache._gpu(q, bounds, pages), stream, _ByBytes.davet_cache_page_select,
            cache._ref, n, cu, kv, x, ldx, n_heads, block, b, first, last, top, p)


def davet_cache_page_attention(cache: KvCache, cu_q, kv_len, q, n_heads, pages, out,
                               lse=None, scale=0.0, block=0, workspace=None,
                               stream=None):
    n, cu, kv, rows = cache._chunk(cu_q, kv_len)
    n_heads, block = _small(n_heads, "n_heads"), _small(block, "block")
    width = n_heads * cache.head_dim
    x, ldx = _rows(q, width, rows, cache.kinds, "q")
    o, ldo = _rows(out, width, rows, cache.kinds, "out")
    p, top = _page_list(cache, pages, rows)
    e, (ws, nb) = _dense(lse, rows * n_heads, _FLOAT, "lse"), _space(workspace)
    _launch(cache._gpu(q, pages, out, lse, workspace), stream,
            _ByBytes.davet_cache_page_attention, cache._ref, n, cu, kv, x, ldx, n_heads,
            scale, block, p, top, o, ldo, e, ws, nb)


# ---- beams

def davet_beam_workspace_bytes(groups, beams, vocab, top):
    out = C.c_size_t(0)
    _check(_L.davet_beam_workspace_bytes(
        _small(int(groups), "groups"), _small(int(beams), "beams"),
        _small(int(vocab), "vocab"), _small(int(top), "top"), C.byref(out)))
    return out.value


def davet_beam_select(logits, dtype, scores, beams, out_scores, out_rows, out_tokens,
                      exclude=-1, done=None, pad=0, workspace=None, stream=None):
    """``logits`` [groups * beams, vocab]; ``out_scores``, ``out_rows`` and
    ``out_tokens`` [groups, top], dense."""
    rows, vocab = logits.shape
    beams = _small(beams, "beams")
    if beams < 1 or rows % beams:
        raise ValueError("davet: logits needs a row a beam of every request")
    groups = rows // beams
    x, ld = _rows(logits, vocab, rows, _kinds(dtype), "logits")
    sc, dn = _dense(scores, rows, _FLOAT, "scores"), _dense(done, rows, _INT, "done")
    shape = out_scores.shape
    if len(shape) != 2 or shape[0] < groups or out_rows.shape != shape or \
            out_tokens.shape != shape:
        raise ValueError("davet: out_scores, out_rows and out_tokens must be "
                         "[groups, top]")
    if (rows | vocab | shape[1]) >> 31:
        _too_large()
    o = _dense(out_scores, 0, _FLOAT, "out_scores")
    r, t = _dense(out_rows, 0, _INT, "out_rows"), _dense(out_tokens, 0, _INT,
                                                         "out_tokens")
    exclude, pad = _small(exclude, "exclude"), _small(pad, "pad")
    ws, nb = _space(workspace)
    _launch(_gpu(logits, scores, done, out_scores, out_rows, out_tokens, workspace),
            stream, _L.davet_beam_select, groups, beams, vocab, x, int(dtype), ld,
            exclude, sc, dn, pad, shape[1], o, r, t, ws, nb)


def davet_cache_reorder(cache: KvCache, kv_len, parent, fresh, dst_table,
                        stream=None):
    """``kv_len``: host list, one entry a row of the cache's page table; ``parent`` and
    ``fresh``: dense int32; ``dst_table``: dense int32 [n_seqs, pages]."""
    n = len(kv_len)
    if n == 0 or n != cache.n_seqs or dst_table.dim() != 2 or len(dst_table) < n:
        raise ValueError("davet: kv_len needs an entry, and dst_table a row, for each "
                         "of page_table's")
    if dst_table.shape[1] >> 31:
        _too_large()
    p, f = _dense(parent, n, _INT, "parent"), _dense(fresh, n, _INT, "fresh")
    dst = _dense(dst_table, 0, _INT, "dst_table")
    _launch(cache._gpu(parent, fresh, dst_table), stream, _ByBytes.davet_cache_reorder,
            cache._ref, n, _words(kv_len), p, f, dst, dst_table.shape[1])


# ---- rotary positions

def davet_rotary_turns(dim, theta, scaling=DAVET_ROTARY_PLAIN, factor=1.0,
                       trained=0.0, fast=0.0, slow=0.0):
    """The turns a position of each pair, a list of dim / 2 floats."""
    dim, scaling = _small(int(dim), "dim"), _small(scaling, "scaling")
    out = (C.c_double * max(1, min(dim, 512) // 2))()
    _check(_L.davet_rotary_turns(dim, theta, scaling, factor, trained, fast, slow,
                                 out))
    return list(out)


def davet_rotary(x, n_heads, head_dim, turns, out, dtype, pos=None,
                 layout=DAVET_ROTARY_HALVES, gain=1.0, inverse=False, stream=None):
    """``x`` and ``out`` [rows, n_heads * head_dim] or wider; ``turns`` a dense
    float64 device tensor: twice its length is the part of a head that turns."""
    kinds, rows, dim = _kinds(dtype), x.shape[0], 2 * turns.numel()
    if (rows | dim) >> 31:
        _too_large()
    n_heads, head_dim = _small(n_heads, "n_heads"), _small(head_dim, "head_dim")
    width = _small(n_heads * head_dim, "n_heads * head_dim")
    a, lda = _rows(x, width, rows, kinds, "x")
    o, ldo = _rows(out, width, rows, kinds, "out")
    t, p = _dense(turns, 1, _DOUBLE, "turns"), _dense(pos, rows, _INT, "pos")
    layout = _small(layout, "layout")
    _launch(_gpu(x, out, turns, pos), stream, _L.davet_rotary, rows, n_heads,
            head_dim, dim, layout, a, lda, o, ldo, int(dtype), p, t,
            gain, 1 if inverse else 0)


def prof_enable(max_launches):
    _check(_L.davet_prof_enable(int(max_launches)))


def prof_reset():
    _check(_L.davet_prof_reset())


def prof_only(cls_name=None):
    """Record only launches of the named kernel class (None: every class)."""
    idx = -1
    if cls_name is not None:
        i = 0
        while True:
            n = _L.davet_prof_class_name(i)
            if not n:
                raise DavetError(-1, "unknown kernel class %r" % cls_name)
            if n.decode() == cls_name:
                idx = i
                break
            i += 1
    _check(_L.davet_prof_only(idx))


def prof_read():
    """{kernel class name: (launches, total ms)}"""
    n = 32
    cnt = (C.c_int64 * n)()
    ms = (C.c_double * n)()
    k = _L.davet_prof_read(n, cnt, ms)
    if k < 0:
        _check(k)
    return {_L.davet_prof_class_name(i).decode(): (cnt[i], ms[i])
            for i in range(k)}
