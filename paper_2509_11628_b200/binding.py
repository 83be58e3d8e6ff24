"""ctypes binding of ``libspeca.so``: the same entry points as ``include/speca.h``.

Argument marshalling only -- every arithmetic step runs in the CUDA kernels behind the C ABI.
Device buffers are torch tensors (or raw integer addresses); host arrays are Python sequences.
There is no fallback: if the library is missing or cannot be loaded, importing the entry points
raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libspeca.so")

SPECA_OK = 0
SPECA_ERR_INVALID_ARG, SPECA_ERR_SHAPE, SPECA_ERR_ALIGNMENT, SPECA_ERR_STATE = 1, 2, 3, 4
SPECA_ERR_ZERO_GAP, SPECA_ERR_NOMEM, SPECA_ERR_CUDA, SPECA_ERR_UNSUPPORTED = 5, 6, 7, 8
SPECA_F32, SPECA_BF16 = 0, 1
SPECA_BASIS_TAYLOR, SPECA_BASIS_NEWTON, SPECA_BASIS_ADAMS_BASHFORTH = 0, 1, 2
SPECA_METRIC_L2, SPECA_METRIC_L1, SPECA_METRIC_LINF, SPECA_METRIC_COSINE = 0, 1, 2, 3
SPECA_PATH_AUTO, SPECA_PATH_DIRECT, SPECA_PATH_BULK, SPECA_PATH_WIDE = 0, 1, 2, 3
SPECA_LAYOUT_TABLES, SPECA_LAYOUT_HISTORY = 0, 1
SPECA_FEATURE_IN_PLACE = 1   # as feats[entry]: the features already sit in the planes speca_cache_next_slot names
SPECA_MAX_ORDER, SPECA_MAX_BATCH, SPECA_MAX_ENTRIES, SPECA_MAX_HORIZON = 4, 64, 512, 8
SPECA_ROPE_INTERLEAVED, SPECA_ROPE_HALVES = 0, 1
SPECA_NORM_LAYER, SPECA_NORM_RMS = 0, 1
SPECA_ACT_NONE, SPECA_ACT_GELU, SPECA_ACT_SILU = 0, 1, 2
SPECA_BLOCK8, SPECA_MAX_K8 = 128, 262144
SPECA_MAX_SEQS, SPECA_MAX_ROWS, SPECA_MAX_HEAD_DIM, SPECA_MAX_GROUP, SPECA_MAX_AXES = 512, (1 << 31) - (1 << 16), 128, 128, 4

EXPORTS = [
    "speca_cache_arena_bytes", "speca_cache_create", "speca_cache_destroy", "speca_cache_reset",
    "speca_cache_update", "speca_cache_update_activate", "speca_cache_update_forecast", "speca_cache_update_forecast_multi", "speca_cache_commit_step", "speca_forecast", "speca_verify",
    "speca_select_adaptive", "speca_activate", "speca_tau", "speca_cache_state", "speca_cache_plane",
    "speca_cache_launch_count", "speca_cache_stats", "speca_cache_check", "speca_cache_next_slot", "speca_forecast_weights", "speca_status_string", "speca_last_error", "speca_version",
    "speca_verify_pred_static", "speca_forecast_multi", "speca_verify_metric",
    "speca_verify_partial", "speca_verify_decide", "speca_cache_get_history", "speca_cache_set_history",
    "speca_forecast_sum", "speca_verify_select",
    "speca_layer_workspace_bytes", "speca_layer_create", "speca_layer_destroy", "speca_layer_modulate", "speca_layer_rope",
    "speca_layer_attention", "speca_layer_check", "speca_layer_last_error",
    "speca_quantize8", "speca_layer_quantize8", "speca_layer_norm8", "speca_layer_matmul8",
]


class SpecaError(RuntimeError):
    def __init__(self, status: int, detail: str = ""):
        self.status = status
        name = _lib().speca_status_string(status).decode()
        super().__init__("speca status %d (%s)%s" % (status, name, (": " + detail) if detail else ""))


class EntryDesc(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("dim", ctypes.c_int32)]


class CacheStats(ctypes.Structure):
    _fields_ = [(name, ctypes.c_uint64) for name in (
        "update_launches", "forecast_launches", "forecast_multi_launches", "forecast_sum_launches",
        "verify_launches", "select_launches", "activate_launches", "update_forecast_launches")] + [
        ("reference_steps", ctypes.c_uint64 * 64), ("resets", ctypes.c_uint64 * 64)]


class CacheConfig(ctypes.Structure):
    _fields_ = [
        ("n_entries", ctypes.c_int32), ("entries", ctypes.POINTER(EntryDesc)), ("batch", ctypes.c_int32),
        ("max_order", ctypes.c_int32), ("dtype", ctypes.c_int32), ("basis", ctypes.c_int32),
        ("verify_entry", ctypes.c_int32), ("eps", ctypes.c_float), ("arena", ctypes.c_void_p),
        ("arena_bytes", ctypes.c_size_t), ("device", ctypes.c_int32), ("path", ctypes.c_int32),
        ("layout", ctypes.c_int32),
    ]


class LayerConfig(ctypes.Structure):
    _fields_ = [
        ("n_seqs", ctypes.c_int32), ("host_q_start", ctypes.POINTER(ctypes.c_int64)),
        ("host_kv_start", ctypes.POINTER(ctypes.c_int64)), ("dtype", ctypes.c_int32), ("n_heads", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("causal", ctypes.c_int32), ("scale", ctypes.c_float),
        ("norm_eps", ctypes.c_float), ("n_axes", ctypes.c_int32), ("axis_dims", ctypes.c_int32 * SPECA_MAX_AXES),
        ("theta", ctypes.c_double), ("pairing", ctypes.c_int32), ("workspace", ctypes.c_void_p),
        ("workspace_bytes", ctypes.c_size_t), ("device", ctypes.c_int32),
    ]


class Matrix8Desc(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("code_stride", ctypes.c_int64), ("scales", ctypes.c_void_p), ("scale_stride", ctypes.c_int64)]


_LIB = None


def _lib() -> ctypes.CDLL:
    global _LIB
    if _LIB is not None:
        return _LIB
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            "libspeca.so is not built (%s). Run `python -m paper_2509_11628_b200.build`; "
            "there is no CPU fallback." % LIB_PATH)
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, dbl = ctypes.c_void_p, ctypes.c_int32, ctypes.c_double
    cfgp = ctypes.POINTER(CacheConfig)
    L.speca_cache_arena_bytes.argtypes = [cfgp, ctypes.POINTER(ctypes.c_size_t)]
    L.speca_cache_create.argtypes = [cfgp, ctypes.POINTER(vp)]
    L.speca_cache_destroy.argtypes = [vp]
    L.speca_cache_reset.argtypes = [vp, vp]
    L.speca_cache_update.argtypes = [vp, vp, vp, vp, vp]
    L.speca_cache_update_activate.argtypes = [vp, vp, vp, vp, vp, vp, vp]
    L.speca_cache_update_forecast.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    L.speca_cache_update_forecast_multi.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp]
    L.speca_cache_commit_step.argtypes = [vp]
    L.speca_forecast.argtypes = [vp, vp, vp, vp, vp]
    L.speca_forecast_sum.argtypes = [vp, vp, i32, vp, vp, vp, vp, vp]
    L.speca_forecast_multi.argtypes = [vp, i32, vp, vp, vp, vp]
    L.speca_verify.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp]
    L.speca_verify_metric.argtypes = [vp, i32, vp, vp, vp, vp, vp, vp, vp, vp]
    L.speca_verify_select.argtypes = [vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, vp, vp, vp, vp]
    L.speca_verify_partial.argtypes = [vp, i32, vp, vp, vp, vp, vp, vp]
    L.speca_verify_decide.argtypes = [i32, vp, i32, vp, ctypes.c_float, vp, vp, vp, vp]
    L.speca_select_adaptive.argtypes = [vp, vp, i32, i32, vp, vp, vp, vp, vp]
    L.speca_activate.argtypes = [vp, vp, vp, vp, vp]
    L.speca_verify_pred_static.argtypes = [vp, vp, ctypes.c_int64, i32, i32, vp, ctypes.c_float, vp, vp, vp, i32, vp]
    L.speca_tau.argtypes = [dbl, dbl, dbl, dbl]
    L.speca_tau.restype = dbl
    L.speca_cache_state.argtypes = [vp, vp, vp]
    L.speca_cache_get_history.argtypes = [vp, vp, vp]
    L.speca_cache_set_history.argtypes = [vp, vp, vp]
    L.speca_cache_plane.argtypes = [vp, i32, i32, ctypes.POINTER(vp), ctypes.POINTER(ctypes.c_size_t)]
    L.speca_cache_launch_count.argtypes = [vp, ctypes.POINTER(ctypes.c_uint64)]
    L.speca_cache_stats.argtypes = [vp, ctypes.POINTER(CacheStats)]
    L.speca_cache_check.argtypes = [vp, vp]
    L.speca_cache_next_slot.argtypes = [vp, i32, i32, ctypes.POINTER(vp)]
    L.speca_forecast_weights.argtypes = [i32, i32, i32, i32, vp, dbl, ctypes.POINTER(i32), vp]
    i64 = ctypes.c_int64
    layerp = ctypes.POINTER(LayerConfig)
    L.speca_layer_workspace_bytes.argtypes = [layerp, ctypes.POINTER(ctypes.c_size_t)]
    L.speca_layer_create.argtypes = [layerp, ctypes.POINTER(vp)]
    L.speca_layer_destroy.argtypes = [vp]
    L.speca_layer_modulate.argtypes = [vp, i32, vp, i64, vp, i64, vp, vp, vp, i64, vp, vp, i64, vp, i64, vp]
    L.speca_layer_rope.argtypes = [vp] + [vp, i64, i64] * 4 + [vp] * 5
    L.speca_layer_attention.argtypes = [vp] + [vp, i64, i64] * 4 + [vp] * 4
    m8 = ctypes.POINTER(Matrix8Desc)
    L.speca_quantize8.argtypes = [i64, i32, vp, i64, i32, m8, i32, vp]
    L.speca_layer_quantize8.argtypes = [vp, i32, vp, i64, vp, m8, vp]
    L.speca_layer_norm8.argtypes = [vp, i32, i32, vp, i64, vp, i64, vp, vp, vp, i64, vp, vp, vp, i64, m8, vp]
    L.speca_layer_matmul8.argtypes = [vp, i32, i32, m8, m8, vp, i32, vp, i64, vp, i64, vp, vp, i64, m8, vp]
    L.speca_layer_check.argtypes = [vp, vp]
    L.speca_layer_last_error.argtypes = [vp]
    L.speca_layer_last_error.restype = ctypes.c_char_p
    L.speca_status_string.argtypes = [i32]
    L.speca_status_string.restype = ctypes.c_char_p
    L.speca_last_error.argtypes = [vp]
    L.speca_last_error.restype = ctypes.c_char_p
    L.speca_version.restype = ctypes.c_char_p
    for name in EXPORTS:
        if getattr(L, name).restype is ctypes.c_int:  # default restype: status codes
            getattr(L, name).restype = i32
    _LIB = L
    return L


# ---- marshalling helpers -------------------------------------------------------------------------

def _dev_ptr(x) -> Optional[int]:
    """torch CUDA tensor / int address / None -> integer address or None."""
    if x is None:
        return None
    if isinstance(x, torch.Tensor):
        if not x.is_cuda:
            raise TypeError("device buffer expected, got a CPU tensor")
        if not x.is_contiguous():
            raise TypeError("device buffers must be contiguous")
        return x.data_ptr()
    return int(x)


def _indexed(device) -> torch.device:
    """The device with its index: ``"cuda"`` alone means the current one, as it does where its memory is allocated."""
    device = torch.device(device)
    if device.type == "cuda" and device.index is None:
        device = torch.device("cuda", torch.cuda.current_device())
    return device


def _stream_ptr(stream) -> Optional[int]:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream or None
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream or None
    return int(stream) or None


def _stream_object(stream, device) -> Optional[torch.cuda.Stream]:
    """The stream as an object of torch's; None for the current one."""
    if stream is None or isinstance(stream, torch.cuda.Stream):
        return stream
    return torch.cuda.ExternalStream(int(stream), device) if int(stream) else torch.cuda.default_stream(device)


def _doubles(xs: Sequence[float]):
    return (ctypes.c_double * len(xs))(*[float(x) for x in xs])


def _floats(xs: Sequence[float]):
    return (ctypes.c_float * len(xs))(*[float(x) for x in xs])


def _bytes(xs: Optional[Sequence[int]]):
    if xs is None:
        return None
    return (ctypes.c_uint8 * len(xs))(*[1 if x else 0 for x in xs])


def _ptr_array(xs: Sequence):
    return (ctypes.c_void_p * len(xs))(*[_dev_ptr(x) for x in xs])


def _check(status: int, handle=None):
    if status != SPECA_OK:
        detail = _lib().speca_last_error(handle).decode() if handle else ""
        raise SpecaError(status, detail)


def _config(entries, batch, max_order, dtype, basis, verify_entry, eps, arena, arena_bytes, device, path,
            layout=SPECA_LAYOUT_TABLES):
    arr = (EntryDesc * len(entries))(*[EntryDesc(int(n), int(d)) for n, d in entries])
    cfg = CacheConfig(len(entries), arr, batch, max_order, dtype, basis, verify_entry, eps,
                      _dev_ptr(arena), arena_bytes, device, path, layout)
    cfg._keep = arr
    return cfg


# ---- the entry points, same names as the header ----------------------------------------------------

def speca_cache_arena_bytes(entries, batch, max_order, dtype, basis=SPECA_BASIS_TAYLOR, verify_entry=-1,
                            path=SPECA_PATH_AUTO, layout=SPECA_LAYOUT_TABLES) -> int:
    cfg = _config(entries, batch, max_order, dtype, basis, verify_entry, 0.0, None, 0, 0, path, layout)
    out = ctypes.c_size_t(0)
    _check(_lib().speca_cache_arena_bytes(ctypes.byref(cfg), ctypes.byref(out)))
    return out.value


def speca_cache_create(entries, batch, max_order, dtype, arena, basis=SPECA_BASIS_TAYLOR, verify_entry=-1,
                       eps=0.0, device=None, path=SPECA_PATH_AUTO, arena_bytes=None, layout=SPECA_LAYOUT_TABLES) -> int:
    """Returns the opaque handle (an integer address). ``arena`` is a CUDA uint8 tensor the caller
    keeps alive, or a raw device address together with ``arena_bytes``."""
    if isinstance(arena, torch.Tensor):
        if device is None:
            device = arena.device.index
        if arena_bytes is None:
            arena_bytes = arena.numel() * arena.element_size()
    cfg = _config(entries, batch, max_order, dtype, basis, verify_entry, eps, arena, arena_bytes or 0,
                  device or 0, path, layout)
    out = ctypes.c_void_p(None)
    _check(_lib().speca_cache_create(ctypes.byref(cfg), ctypes.byref(out)))
    return out.value


def speca_cache_destroy(cache) -> None:
    _check(_lib().speca_cache_destroy(cache))


def speca_cache_reset(cache, host_sample_mask=None) -> None:
    _check(_lib().speca_cache_reset(cache, _bytes(host_sample_mask)), cache)


def speca_cache_update(cache, feats, t_ref, host_sample_mask=None, stream=None) -> None:
    _check(_lib().speca_cache_update(cache, _ptr_array(feats), _doubles(t_ref), _bytes(host_sample_mask),
                                     _stream_ptr(stream)), cache)


def speca_cache_update_activate(cache, feats, t_ref, host_sample_mask, dev_spec_count, dev_active_mask, stream=None) -> None:
    """speca_cache_update + speca_activate for the masked samples in one launch."""
    _check(_lib().speca_cache_update_activate(cache, _ptr_array(feats), _doubles(t_ref), _bytes(host_sample_mask),
                                              _dev_ptr(dev_spec_count), _dev_ptr(dev_active_mask), _stream_ptr(stream)), cache)


def speca_cache_update_forecast(cache, feats, t_ref, host_sample_mask, t_target, dev_active_mask, outs, dev_spec_count=None,
                                dev_rearm_mask=None, stream=None) -> None:
    """A whole reference step (update + commit) and the forecast at t_target in one launch."""
    _check(_lib().speca_cache_update_forecast(cache, _ptr_array(feats), _doubles(t_ref), _bytes(host_sample_mask),
                                              _doubles(t_target), _dev_ptr(dev_active_mask), _ptr_array(outs),
                                              _dev_ptr(dev_spec_count), _dev_ptr(dev_rearm_mask), _stream_ptr(stream)), cache)


def speca_cache_update_forecast_multi(cache, feats, t_ref, host_sample_mask, t_targets, dev_active_mask, outs,
                                      dev_spec_count=None, dev_rearm_mask=None, stream=None) -> None:
    """The same with K speculative times: t_targets is K lists of B times, outs[e] a [K, B, N_e, D] tensor."""
    flat = [t for row in t_targets for t in row]
    _check(_lib().speca_cache_update_forecast_multi(cache, _ptr_array(feats), _doubles(t_ref), _bytes(host_sample_mask),
                                                    len(t_targets), _doubles(flat), _dev_ptr(dev_active_mask), _ptr_array(outs),
                                                    _dev_ptr(dev_spec_count), _dev_ptr(dev_rearm_mask), _stream_ptr(stream)), cache)


def speca_cache_commit_step(cache) -> None:
    _check(_lib().speca_cache_commit_step(cache), cache)


def speca_forecast(cache, t_target, dev_active_mask, outs, stream=None) -> None:
    _check(_lib().speca_forecast(cache, _doubles(t_target), _dev_ptr(dev_active_mask), _ptr_array(outs),
                                 _stream_ptr(stream)), cache)


def speca_forecast_sum(cache, entry_ids, t_target, dev_active_mask, base, out, stream=None) -> None:
    """out = base + sum of the forecasts of the listed (equally shaped) entries; base may be None."""
    ids = (ctypes.c_int32 * len(entry_ids))(*[int(e) for e in entry_ids])
    _check(_lib().speca_forecast_sum(cache, ids, len(entry_ids), _doubles(t_target), _dev_ptr(dev_active_mask),
                                     _dev_ptr(base), _dev_ptr(out), _stream_ptr(stream)), cache)


def speca_forecast_multi(cache, t_targets, dev_active_mask, outs, stream=None) -> None:
    """``t_targets``: K lists of B times; ``outs[e]``: device tensor [K, B, N_e, D] (None = skip)."""
    flat = [float(t) for row in t_targets for t in row]
    _check(_lib().speca_forecast_multi(cache, len(t_targets), _doubles(flat), _dev_ptr(dev_active_mask),
                                       _ptr_array(outs), _stream_ptr(stream)), cache)


def speca_verify(cache, fresh, t_target, tau, dev_active_mask, out_pred, dev_err, dev_accept, stream=None) -> None:
    _check(_lib().speca_verify(cache, _dev_ptr(fresh), _doubles(t_target), _floats(tau), _dev_ptr(dev_active_mask),
                               _dev_ptr(out_pred), _dev_ptr(dev_err), _dev_ptr(dev_accept), _stream_ptr(stream)),
           cache)


def speca_verify_metric(cache, metric, fresh, t_target, tau, dev_active_mask, out_pred, dev_err, dev_accept,
                        stream=None) -> None:
    _check(_lib().speca_verify_metric(cache, int(metric), _dev_ptr(fresh), _doubles(t_target), _floats(tau),
                                      _dev_ptr(dev_active_mask), _dev_ptr(out_pred), _dev_ptr(dev_err),
                                      _dev_ptr(dev_accept), _stream_ptr(stream)), cache)


def speca_verify_select(cache, metric, fresh, t_target, tau, dev_active_mask, dev_next_active_mask, out_pred, dev_err,
                        dev_accept, k_max, group, dev_spec_count, dev_active_idx=None, dev_n_active=None, stream=None) -> None:
    """speca_verify_metric + speca_select_adaptive in one launch; the next mask goes to its own buffer."""
    _check(_lib().speca_verify_select(cache, int(metric), _dev_ptr(fresh), _doubles(t_target), _floats(tau),
                                      _dev_ptr(dev_active_mask), _dev_ptr(dev_next_active_mask), _dev_ptr(out_pred),
                                      _dev_ptr(dev_err), _dev_ptr(dev_accept), int(k_max), int(group),
                                      _dev_ptr(dev_spec_count), _dev_ptr(dev_active_idx), _dev_ptr(dev_n_active),
                                      _stream_ptr(stream)), cache)


def speca_verify_partial(cache, metric, fresh, t_target, dev_active_mask, out_pred, dev_sums, stream=None) -> None:
    """``dev_sums``: CUDA float64 tensor [B, 4] that receives the metric's running values of this shard."""
    _check(_lib().speca_verify_partial(cache, int(metric), _dev_ptr(fresh), _doubles(t_target), _dev_ptr(dev_active_mask),
                                       _dev_ptr(out_pred), _dev_ptr(dev_sums), _stream_ptr(stream)), cache)


def speca_verify_decide(metric, dev_sums, batch, tau, eps, dev_active_mask, dev_err, dev_accept, stream=None) -> None:
    _check(_lib().speca_verify_decide(int(metric), _dev_ptr(dev_sums), int(batch), _floats(tau), float(eps),
                                      _dev_ptr(dev_active_mask), _dev_ptr(dev_err), _dev_ptr(dev_accept),
                                      _stream_ptr(stream)))


def speca_select_adaptive(cache, dev_accept, k_max, group, dev_spec_count, dev_active_mask, dev_active_idx=None,
                          dev_n_active=None, stream=None) -> None:
    _check(_lib().speca_select_adaptive(cache, _dev_ptr(dev_accept), int(k_max), int(group), _dev_ptr(dev_spec_count),
                                        _dev_ptr(dev_active_mask), _dev_ptr(dev_active_idx), _dev_ptr(dev_n_active),
                                        _stream_ptr(stream)), cache)


def speca_activate(cache, host_sample_mask, dev_spec_count, dev_active_mask, stream=None) -> None:
    _check(_lib().speca_activate(cache, _bytes(host_sample_mask), _dev_ptr(dev_spec_count), _dev_ptr(dev_active_mask),
                                 _stream_ptr(stream)), cache)


def speca_verify_pred_static(pred, fresh, n_elems, batch, dtype, tau, eps, dev_active_mask, dev_err, dev_accept,
                             device=0, stream=None) -> None:
    """Eq. 4 + accept rule on a forecast the caller holds, with the reduction scratch inside the
    library image: for callers that cannot allocate device memory or hand over an arena. Calls
    whose kernels overlap on the GPU race on that shared scratch; keep them in stream order."""
    _check(_lib().speca_verify_pred_static(_dev_ptr(pred), _dev_ptr(fresh), int(n_elems), int(batch), int(dtype),
                                           _floats(tau), float(eps), _dev_ptr(dev_active_mask), _dev_ptr(dev_err),
                                           _dev_ptr(dev_accept), int(device), _stream_ptr(stream)))


def speca_tau(tau0: float, beta: float, t: float, T: float) -> float:
    return float(_lib().speca_tau(tau0, beta, t, T))


def speca_cache_state(cache, batch: int):
    n = (ctypes.c_int32 * batch)()
    t = (ctypes.c_double * batch)()
    _check(_lib().speca_cache_state(cache, n, t), cache)
    return list(n), list(t)


def speca_cache_get_history(cache, batch: int):
    """(n_refs[B], t_hist[B][SPECA_MAX_ORDER + 1]) -- with the arena bytes, everything a checkpoint needs."""
    n = (ctypes.c_int32 * batch)()
    t = (ctypes.c_double * (batch * (SPECA_MAX_ORDER + 1)))()
    _check(_lib().speca_cache_get_history(cache, n, t), cache)
    w = SPECA_MAX_ORDER + 1
    return list(n), [list(t[b * w:(b + 1) * w]) for b in range(batch)]


def speca_cache_set_history(cache, n_refs, t_hist) -> None:
    n = (ctypes.c_int32 * len(n_refs))(*[int(x) for x in n_refs])
    flat = [float(x) for row in t_hist for x in row]
    t = (ctypes.c_double * len(flat))(*flat)
    _check(_lib().speca_cache_set_history(cache, n, t), cache)


def speca_cache_plane(cache, entry: int, sample: int):
    p = ctypes.c_void_p(None)
    s = ctypes.c_size_t(0)
    _check(_lib().speca_cache_plane(cache, entry, sample, ctypes.byref(p), ctypes.byref(s)), cache)
    return p.value, s.value


def speca_forecast_weights(layout: int, basis: int, max_order: int, n_refs: int, t_hist: Sequence[float], t_target: float):
    """(order, coefficients) a forecast at ``t_target`` hands to the kernels; host only, no GPU needed."""
    order = ctypes.c_int32(0)
    coef = (ctypes.c_float * (SPECA_MAX_ORDER + 1))()
    _check(_lib().speca_forecast_weights(layout, basis, max_order, n_refs, _doubles(t_hist), float(t_target),
                                         ctypes.byref(order), coef))
    return order.value, [float(x) for x in coef]


def speca_cache_next_slot(cache, entry: int, sample: int) -> int:
    """Device address of the plane the next reference step of ``sample`` fills for ``entry`` (raw-feature cache)."""
    out = ctypes.c_void_p(None)
    _check(_lib().speca_cache_next_slot(cache, int(entry), int(sample), ctypes.byref(out)), cache)
    return out.value


def speca_cache_stats(cache, batch: int) -> dict:
    """Host-side counters of the handle: launches per kernel kind, reference steps and resets per sample."""
    st = CacheStats()
    _check(_lib().speca_cache_stats(cache, ctypes.byref(st)), cache)
    out = {name: int(getattr(st, name)) for name, _ in CacheStats._fields_[:8]}
    out["reference_steps"] = [int(x) for x in st.reference_steps[:batch]]
    out["resets"] = [int(x) for x in st.resets[:batch]]
    return out


def speca_cache_check(cache, stream=None) -> None:
    _check(_lib().speca_cache_check(cache, _stream_ptr(stream)), cache)


def speca_cache_launch_count(cache) -> int:
    n = ctypes.c_uint64(0)
    _check(_lib().speca_cache_launch_count(cache, ctypes.byref(n)), cache)
    return n.value


# ---- the verification layer ------------------------------------------------------------------------

_TORCH_DTYPES = {SPECA_F32: torch.float32, SPECA_BF16: torch.bfloat16}


def _layer_config(q_start, dtype, kv_start, n_heads, n_kv_heads, head_dim, causal, scale, norm_eps, axis_dims, theta, pairing):
    def offsets(xs):
        return (ctypes.c_int64 * len(xs))(*[int(x) for x in xs])

    if kv_start is not None and len(kv_start) != len(q_start):
        raise ValueError("kv_start and q_start describe different numbers of sequences")
    if len(axis_dims) > SPECA_MAX_AXES:
        raise ValueError("at most %d rotary axes" % SPECA_MAX_AXES)
    cfg = LayerConfig(n_seqs=len(q_start) - 1, dtype=dtype, n_heads=n_heads, n_kv_heads=n_kv_heads, head_dim=head_dim,
                      causal=int(causal), scale=scale, norm_eps=norm_eps, n_axes=len(axis_dims), theta=theta, pairing=pairing)
    cfg.host_q_start = offsets(q_start)
    if kv_start is not None:
        cfg.host_kv_start = offsets(kv_start)
    cfg.axis_dims[:len(axis_dims)] = [int(d) for d in axis_dims]
    return cfg


def speca_layer_workspace_bytes(q_start, dtype, kv_start=None, n_heads=0, n_kv_heads=0, head_dim=0, causal=False, scale=0.0,
                                norm_eps=0.0, axis_dims=(), theta=10000.0, pairing=SPECA_ROPE_INTERLEAVED) -> int:
    cfg = _layer_config(q_start, dtype, kv_start, n_heads, n_kv_heads, head_dim, causal, scale, norm_eps, axis_dims, theta, pairing)
    out = ctypes.c_size_t(0)
    _check(_lib().speca_layer_workspace_bytes(ctypes.byref(cfg), ctypes.byref(out)))
    return out.value


def speca_layer_create(q_start, dtype, workspace, kv_start=None, n_heads=0, n_kv_heads=0, head_dim=0, causal=False, scale=0.0,
                       norm_eps=0.0, axis_dims=(), theta=10000.0, pairing=SPECA_ROPE_INTERLEAVED, device=None,
                       workspace_bytes=None) -> int:
    """Returns the opaque handle (an integer address). ``workspace`` is a CUDA uint8 tensor the caller keeps alive, or
    a raw device address together with ``workspace_bytes``."""
    if isinstance(workspace, torch.Tensor):
        _dev_ptr(workspace)     # on a GPU
        device = workspace.device.index if device is None else device
        if workspace.device.index != device:
            raise SpecaError(SPECA_ERR_INVALID_ARG, "the workspace is on %s, the layer on device %d" % (workspace.device, device))
        workspace_bytes = workspace.numel() * workspace.element_size() if workspace_bytes is None else workspace_bytes
    cfg = _layer_config(q_start, dtype, kv_start, n_heads, n_kv_heads, head_dim, causal, scale, norm_eps, axis_dims, theta, pairing)
    cfg.workspace, cfg.workspace_bytes, cfg.device = _dev_ptr(workspace), workspace_bytes or 0, device or 0
    out = ctypes.c_void_p(None)
    _check(_lib().speca_layer_create(ctypes.byref(cfg), ctypes.byref(out)))
    return out.value


def speca_layer_destroy(layer) -> None:
    _check(_lib().speca_layer_destroy(layer))


def _check_layer(status: int, layer):
    if status != SPECA_OK:
        raise SpecaError(status, _lib().speca_layer_last_error(layer).decode() if layer else "")


def speca_layer_modulate(layer, dim, x, x_stride, branch, branch_stride, gate, scale, shift, mod_stride, dev_active_mask, x_out,
                         x_out_stride, y, y_stride, stream=None) -> None:
    """Device addresses and strides in elements, as in the header; ``SpecaLayer.modulate`` takes tensors."""
    _check_layer(_lib().speca_layer_modulate(layer, dim, x, x_stride, branch, branch_stride, gate, scale, shift, mod_stride,
                                             dev_active_mask, x_out, x_out_stride, y, y_stride, _stream_ptr(stream)), layer)


def speca_layer_rope(layer, q, q_out, k, k_out, positions, q_weight, k_weight, dev_active_mask, stream=None) -> None:
    """q, q_out, k, k_out: (address, row stride, head stride) each; ``SpecaLayer.rope`` takes tensors."""
    _check_layer(_lib().speca_layer_rope(layer, *q, *q_out, *k, *k_out, positions, q_weight, k_weight, dev_active_mask,
                                         _stream_ptr(stream)), layer)


def speca_layer_attention(layer, q, k, v, o, dev_kv_len, dev_active_mask, dev_lse, stream=None) -> None:
    """q, k, v, o: (address, row stride, head stride) each; ``SpecaLayer.attention`` takes tensors."""
    _check_layer(_lib().speca_layer_attention(layer, *q, *k, *v, *o, dev_kv_len, dev_active_mask, dev_lse,
                                              _stream_ptr(stream)), layer)


def speca_quantize8(rows, dim, x, x_stride, dtype, out, device, stream=None) -> None:
    """``out``: a ``Matrix8Desc``; ``quantize8`` takes tensors."""
    _check(_lib().speca_quantize8(rows, dim, x, x_stride, dtype, ctypes.byref(out), device, _stream_ptr(stream)))


def speca_layer_quantize8(layer, dim, x, x_stride, dev_active_mask, out, stream=None) -> None:
    _check_layer(_lib().speca_layer_quantize8(layer, dim, x, x_stride, dev_active_mask, ctypes.byref(out), _stream_ptr(stream)), layer)


def speca_layer_norm8(layer, kind, dim, x, x_stride, branch, branch_stride, gate, scale, shift, mod_stride, weight, dev_active_mask,
                      x_out, x_out_stride, out, stream=None) -> None:
    _check_layer(_lib().speca_layer_norm8(layer, kind, dim, x, x_stride, branch, branch_stride, gate, scale, shift, mod_stride, weight,
                                          dev_active_mask, x_out, x_out_stride, ctypes.byref(out), _stream_ptr(stream)), layer)


def speca_layer_matmul8(layer, n, k, a, w, bias, activation, residual, residual_stride, gate, gate_stride, dev_active_mask, out,
                        out_stride, out_8bit, stream=None) -> None:
    """a, w, out_8bit: ``Matrix8Desc`` (out_8bit or out is None); ``SpecaLayer.matmul8`` takes tensors."""
    _check_layer(_lib().speca_layer_matmul8(layer, n, k, ctypes.byref(a), ctypes.byref(w), bias, activation, residual, residual_stride,
                                            gate, gate_stride, dev_active_mask, out, out_stride,
                                            None if out_8bit is None else ctypes.byref(out_8bit), _stream_ptr(stream)), layer)


def speca_layer_check(layer, stream=None) -> None:
    _check_layer(_lib().speca_layer_check(layer, _stream_ptr(stream)), layer)


def speca_layer_last_error(layer) -> str:
    return _lib().speca_layer_last_error(layer).decode()


def speca_status_string(status: int) -> str:
    return _lib().speca_status_string(status).decode()


def speca_last_error(cache) -> str:
    return _lib().speca_last_error(cache).decode()


def speca_version() -> str:
    return _lib().speca_version().decode()


class SpecaCache:
    """Owns an arena tensor and a handle; forwards to the entry points above."""

    def __init__(self, entries, batch, max_order, dtype, device="cuda:0", basis=SPECA_BASIS_TAYLOR,
                 verify_entry=-1, eps=0.0, path=SPECA_PATH_AUTO, layout=SPECA_LAYOUT_TABLES):
        self.entries = [(int(n), int(d)) for n, d in entries]
        self.batch, self.max_order, self.dtype, self.basis = batch, max_order, dtype, basis
        self.layout, self.path = layout, path
        self.device = _indexed(device)
        self.verify_entry = verify_entry if verify_entry >= 0 else len(self.entries) - 1
        nbytes = speca_cache_arena_bytes(self.entries, batch, max_order, dtype, basis, verify_entry, path, layout)
        self.arena = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        assert self.arena.data_ptr() % 256 == 0
        self.handle = speca_cache_create(self.entries, batch, max_order, dtype, self.arena, basis, verify_entry,
                                         eps, self.device.index, path, layout=layout)

    def close(self):
        if self.handle:
            speca_cache_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def update(self, feats, t_ref, mask=None, stream=None):
        speca_cache_update(self.handle, feats, t_ref, mask, stream)

    def update_activate(self, feats, t_ref, mask, spec_count, active, stream=None):
        speca_cache_update_activate(self.handle, feats, t_ref, mask, spec_count, active, stream)

    def update_forecast(self, feats, t_ref, t_target, outs, mask=None, active=None, spec_count=None, rearm=None, stream=None):
        """A whole reference step and the first forecast after it in one launch (commits the step)."""
        speca_cache_update_forecast(self.handle, feats, t_ref, mask, t_target, active, outs, spec_count, rearm, stream)

    def update_forecast_multi(self, feats, t_ref, t_targets, outs, mask=None, active=None, spec_count=None, rearm=None, stream=None):
        """The same for K speculative times: outs[e] is [K, B, N_e, D]."""
        speca_cache_update_forecast_multi(self.handle, feats, t_ref, mask, t_targets, active, outs, spec_count, rearm, stream)

    def commit_step(self):
        speca_cache_commit_step(self.handle)

    def forecast(self, t_target, outs, active=None, stream=None):
        speca_forecast(self.handle, t_target, active, outs, stream)

    def forecast_sum(self, entry_ids, t_target, out, base=None, active=None, stream=None):
        speca_forecast_sum(self.handle, entry_ids, t_target, active, base, out, stream)

    def forecast_multi(self, t_targets, outs, active=None, stream=None):
        speca_forecast_multi(self.handle, t_targets, active, outs, stream)

    def verify(self, fresh, t_target, tau, err, accept, active=None, out_pred=None, stream=None, metric=None):
        if metric is None:
            speca_verify(self.handle, fresh, t_target, tau, active, out_pred, err, accept, stream)
        else:
            speca_verify_metric(self.handle, metric, fresh, t_target, tau, active, out_pred, err, accept, stream)

    def verify_select(self, fresh, t_target, tau, err, accept, active, next_active, k_max, group, spec_count, idx=None,
                      n_active=None, out_pred=None, stream=None, metric=0):
        speca_verify_select(self.handle, metric, fresh, t_target, tau, active, next_active, out_pred, err, accept, k_max,
                            group, spec_count, idx, n_active, stream)

    def select_adaptive(self, accept, k_max, group, spec_count, active, idx=None, n_active=None, stream=None):
        speca_select_adaptive(self.handle, accept, k_max, group, spec_count, active, idx, n_active, stream)

    def activate(self, mask, spec_count, active, stream=None):
        speca_activate(self.handle, mask, spec_count, active, stream)

    def reset(self, mask=None):
        speca_cache_reset(self.handle, mask)

    def state(self):
        return speca_cache_state(self.handle, self.batch)

    def plane_tensor(self, entry: int, sample: int) -> torch.Tensor:
        """View of the (entry, sample) table as ``[m+1, n_elems]`` in the storage dtype."""
        ptr, stride = speca_cache_plane(self.handle, entry, sample)
        esz = 2 if self.dtype == SPECA_BF16 else 4
        tdt = torch.bfloat16 if self.dtype == SPECA_BF16 else torch.float32
        n = self.entries[entry][0] * self.entries[entry][1]
        off = ptr - self.arena.data_ptr()
        raw = self.arena[off: off + stride * (self.max_order + 1)].view(tdt).view(self.max_order + 1, stride // esz)
        return raw[:, :n]

    @property
    def launches(self) -> int:
        return speca_cache_launch_count(self.handle)

    def stats(self):
        return speca_cache_stats(self.handle, self.batch)

    def check(self, stream=None):
        """Waits for `stream` and raises if a staged copy of the bulk path gave up."""
        speca_cache_check(self.handle, stream)

    def next_slot_batch(self, entry: int) -> torch.Tensor:
        """All samples' next planes of ``entry`` as one strided ``[B, N_e, D]`` view of the arena (raw-feature
        cache whose samples are at the same ring position): write the block output here and pass
        ``SPECA_FEATURE_IN_PLACE`` for the entry to ``update``."""
        ptrs = [speca_cache_next_slot(self.handle, entry, b) for b in range(self.batch)]
        n, d = self.entries[entry]
        esz = 2 if self.dtype == SPECA_BF16 else 4
        tdt = torch.bfloat16 if self.dtype == SPECA_BF16 else torch.float32
        step = (ptrs[1] - ptrs[0]) if self.batch > 1 else n * d * esz
        if any(ptrs[b] - ptrs[0] != b * step for b in range(self.batch)):
            raise ValueError("the samples are at different ring positions: use next_slot_tensor per sample")
        off = ptrs[0] - self.arena.data_ptr()
        flat = self.arena[off:].view(tdt)
        return torch.as_strided(flat, (self.batch, n, d), (step // esz, d, 1))

    def next_slot_tensor(self, entry: int, sample: int = 0) -> torch.Tensor:
        """The plane that the next reference step of ``sample`` fills, as an ``[N_e, D]`` view of the arena
        (raw-feature cache): write the block output here and pass it to ``update`` to skip the copy."""
        ptr = speca_cache_next_slot(self.handle, entry, sample)
        n, d = self.entries[entry]
        tdt = torch.bfloat16 if self.dtype == SPECA_BF16 else torch.float32
        off = ptr - self.arena.data_ptr()
        return self.arena[off: off + n * d * (2 if self.dtype == SPECA_BF16 else 4)].view(tdt).view(n, d)


class Matrix8:
    """A matrix in 8 bits: ``codes`` float8_e4m3fn ``[rows, dim]`` (rows may be strided, the last dimension is dense) and
    ``scales`` float8_e8m0fnu ``[ceil(dim / 512), rows, 4]``: the scale of column c of row r is ``scales[c // 512, r, c // 128 % 4]``.
    Rows of codes that start on multiples of 16 bytes, as ``empty`` lays them out, can enter a product. A matrix stands for the memory it was
    made of: ``codes`` and ``scales`` cannot be assigned, and one whose tensors have been moved (``set_``, a storage resized) is refused."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor):
        if codes.dtype is not torch.float8_e4m3fn or scales.dtype is not torch.float8_e8m0fnu:
            raise TypeError("codes are float8_e4m3fn and scales float8_e8m0fnu, not %s and %s" % (codes.dtype, scales.dtype))
        if codes.dim() != 2 or scales.shape != (-(-codes.shape[1] // (4 * SPECA_BLOCK8)), codes.shape[0], 4):
            raise ValueError("codes %s and scales %s do not go together" % (tuple(codes.shape), tuple(scales.shape)))
        if codes.device != scales.device:
            raise TypeError("codes on %s, scales on %s" % (codes.device, scales.device))
        rows, dim = codes.shape
        if (dim > 1 and codes.stride(1) != 1) or (rows > 0 and scales.shape[0] > 0 and (scales.stride(2) != 1 or (rows > 1 and scales.stride(1) != 4))):
            raise TypeError("the last dimension of codes, and the last two of scales, must be dense")
        # tensors of its own, so that what is done to the caller's (transposed or resized in place) is not done to these
        codes, scales = codes.detach(), scales.detach()
        self.__dict__.update(codes=codes, scales=scales)
        self.shape, self.device, self.index = codes.shape, codes.device, codes.get_device()
        self.codes_now, self.scales_now = codes.data_ptr, scales.data_ptr
        self.codes_at, self.scales_at = codes.data_ptr(), scales.data_ptr()
        self.desc = Matrix8Desc(self.codes_at, codes.stride(0), self.scales_at, scales.stride(0))
        self.ref = ctypes.byref(self.desc)

    def __setattr__(self, name, value):   # (properties would cost each reader 0.1 us)
        if name in ("codes", "scales"):
            raise AttributeError("%s of a Matrix8 cannot be assigned: make another from the tensors" % name)
        object.__setattr__(self, name, value)

    def stand(self, name: str) -> None:
        """Refuses a matrix whose memory has gone."""
        if self.codes_now() != self.codes_at or self.scales_now() != self.scales_at:
            raise ValueError("%s: the matrix's tensors no longer have the memory it was made of" % name)

    @classmethod
    def empty(cls, rows: int, dim: int, device="cuda:0") -> "Matrix8":
        """Zeros, with rows of codes a multiple of 16 bytes apart."""
        codes = torch.zeros(rows, -(-dim // 16) * 16, dtype=torch.uint8, device=device)[:, :dim].view(torch.float8_e4m3fn)
        scales = torch.zeros(-(-dim // (4 * SPECA_BLOCK8)), rows, 4, dtype=torch.uint8, device=device).view(torch.float8_e8m0fnu)
        return cls(codes, scales)


def quantize8(x: torch.Tensor, out: Optional[Matrix8] = None, stream=None) -> Matrix8:
    """Weights ``[rows, dim]`` (fp32 or bf16, on a GPU) into 8 bits. Without ``out`` the matrix is made on ``stream``, as under
    ``torch.cuda.stream``."""
    dtype = {t: code for code, t in _TORCH_DTYPES.items()}.get(x.dtype)
    if dtype is None:
        raise TypeError("fp32 or bf16 is expected, not %s" % x.dtype)
    if not x.is_cuda:
        raise TypeError("a tensor on a GPU is expected")
    if x.dim() != 2 or (x.shape[1] > 1 and x.stride(1) != 1):
        raise ValueError("a matrix with a dense last dimension is expected")
    if out is None:
        # its zeros are written on the stream that the codes are, or they could come behind them
        with torch.cuda.stream(_stream_object(stream, x.device)):
            out = Matrix8.empty(*x.shape, x.device)
    if out.shape != x.shape:
        raise ValueError("out: shape %s is expected, not %s" % (tuple(x.shape), tuple(out.shape)))
    if out.index != x.get_device():
        raise TypeError("out: a matrix on %s is expected" % x.device)
    out.stand("out")
    speca_quantize8(x.shape[0], x.shape[1], x.data_ptr(), x.stride(0), dtype, out.desc, out.index,
                    torch._C._cuda_getCurrentRawStream(out.index) if stream is None else stream)
    return out


_NO_STRIDE, _NO_MODULATIONS = (0,), (None, None, None)


class SpecaLayer:
    """The parts of a verification layer, its matrix products in 8 bits among them, over packed sequences: sequence s of a
    ``[rows, ...]`` tensor is rows ``q_start[s]`` to ``q_start[s + 1] - 1``. Owns the workspace and the handle. Tensors
    may be strided views whose last dimension is dense; outputs are the caller's."""

    def __init__(self, q_start, dtype, kv_start=None, n_heads=0, n_kv_heads=0, head_dim=0, causal=False, scale=0.0, norm_eps=0.0,
                 axis_dims=(), theta=10000.0, pairing=SPECA_ROPE_INTERLEAVED, device="cuda:0"):
        self.handle = None
        self.device = _indexed(device)
        self.n_seqs, self.n_heads, self.n_kv_heads, self.head_dim = len(q_start) - 1, n_heads, n_kv_heads, head_dim
        self.rows = int(q_start[-1])
        self.kv_rows = int(kv_start[-1]) if kv_start is not None else self.rows
        self.n_axes = len(axis_dims)
        self.torch_dtype = _TORCH_DTYPES[dtype]
        self.index = self.device.index or 0
        self.q_shape = (self.rows, n_heads, head_dim)
        self.k_shape = (self.kv_rows, n_kv_heads, head_dim)     # of keys and values
        self.new_k_shape = (self.rows, n_kv_heads, head_dim)    # of the keys that belong to the query rows
        kw = dict(kv_start=kv_start, n_heads=n_heads, n_kv_heads=n_kv_heads, head_dim=head_dim, causal=causal, scale=scale,
                  norm_eps=norm_eps, axis_dims=axis_dims, theta=theta, pairing=pairing)
        nbytes = speca_layer_workspace_bytes(q_start, dtype, **kw)
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        self.handle = speca_layer_create(q_start, dtype, self.workspace, device=self.index, **kw)
        self.lib = _lib()

    def close(self):
        if self.handle:
            handle, self.handle = self.handle, None
            speca_layer_destroy(handle)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _tensor(self, t, name, shape, dtype):
        """(address, strides) of a device tensor of this shape and type whose last dimension is dense."""
        s = t.stride()
        if t.dtype is not dtype or t.shape != shape or t.get_device() != self.index or (s[-1] != 1 and shape[-1] > 1):
            self._refuse(t, name, shape, dtype)
        return t.data_ptr(), s

    def _refuse(self, t, name, shape, dtype):
        if not t.is_cuda or t.get_device() != self.index:
            raise TypeError("%s: a tensor on %s is expected" % (name, self.device))
        if t.dtype is not dtype:
            raise TypeError("%s: %s is expected, not %s" % (name, dtype, t.dtype))
        if t.shape != shape:
            raise ValueError("%s: shape %s is expected, not %s" % (name, tuple(shape), tuple(t.shape)))
        raise TypeError("%s: the last dimension must be dense" % name)

    def _heads(self, t, name, shape):
        """(address, row stride, head stride) of a [rows, heads, head_dim] tensor."""
        if t is None:
            return None, 0, 0
        p, s = self._tensor(t, name, shape, self.torch_dtype)
        return p, s[0], s[1]

    def _vector(self, t, name, n, dtype):
        return None if t is None else self._tensor(t, name, (n,), dtype)[0]

    def _stream(self, stream):
        """The stream's address; of the device's current stream without the Stream object around it (2 us a call)."""
        if stream is None:
            return torch._C._cuda_getCurrentRawStream(self.index)
        return stream.cuda_stream if isinstance(stream, torch.cuda.Stream) else stream

    def _modulations(self, tensors, dim):
        """Addresses of gate, scale and shift ([n_seqs, dim] or None) and their one row stride."""
        mods, mod_stride = [None, None, None], None
        for i, m in enumerate(tensors):
            if m is not None:
                mods[i], s = self._tensor(m, ("gate", "scale", "shift")[i], (self.n_seqs, dim), self.torch_dtype)
                if mod_stride is None:
                    mod_stride = s[0]
                elif s[0] != mod_stride and self.n_seqs > 1:
                    raise ValueError("gate, scale and shift must share one row stride")
        return mods, mod_stride or 0

    def modulate(self, x, y, branch=None, gate=None, scale=None, shift=None, x_out=None, active=None, stream=None):
        """x' = x + gate * branch; y = layer norm of x' * (1 + scale) + shift, the modulations by sequence."""
        dim, dt = x.shape[-1], self.torch_dtype
        shape = (self.rows, dim)
        px, sx = self._tensor(x, "x", shape, dt)
        py, sy = self._tensor(y, "y", shape, dt)
        pb, sb = (None, (0,)) if branch is None else self._tensor(branch, "branch", shape, dt)
        po, so = (None, (0,)) if x_out is None else self._tensor(x_out, "x_out", shape, dt)
        mods, mod_stride = self._modulations((gate, scale, shift), dim)
        speca_layer_modulate(self.handle, dim, px, sx[0], pb, sb[0], mods[0], mods[1], mods[2], mod_stride,
                             self._vector(active, "active", self.n_seqs, torch.uint8), po, so[0], py, sy[0], self._stream(stream))

    def rope(self, q, q_out, k, k_out, positions, q_weight=None, k_weight=None, active=None, stream=None):
        """Rotary positions (``positions``: fp32 [rows, axes]) of q and k, after an RMS norm where a weight is given."""
        pos, _ = self._tensor(positions, "positions", (self.rows, self.n_axes), torch.float32)
        if not positions.is_contiguous():
            raise TypeError("positions: must be contiguous")
        speca_layer_rope(
            self.handle, self._heads(q, "q", self.q_shape), self._heads(q_out, "q_out", self.q_shape),
            self._heads(k, "k", self.new_k_shape), self._heads(k_out, "k_out", self.new_k_shape), pos,
            self._vector(q_weight, "q_weight", self.head_dim, self.torch_dtype),
            self._vector(k_weight, "k_weight", self.head_dim, self.torch_dtype),
            self._vector(active, "active", self.n_seqs, torch.uint8), self._stream(stream))

    def attention(self, q, k, v, out, lse=None, kv_len=None, active=None, stream=None):
        """out = softmax(scale q k^T) v per sequence; ``kv_len``: int32 per sequence, keys that hold data."""
        p_lse = None
        if lse is not None:
            p_lse, _ = self._tensor(lse, "lse", (self.n_heads, self.rows), torch.float32)
            if not lse.is_contiguous():
                raise TypeError("lse: must be contiguous")
        speca_layer_attention(
            self.handle, self._heads(q, "q", self.q_shape), self._heads(k, "k", self.k_shape), self._heads(v, "v", self.k_shape),
            self._heads(out, "out", self.q_shape), self._vector(kv_len, "kv_len", self.n_seqs, torch.int32),
            self._vector(active, "active", self.n_seqs, torch.uint8), p_lse, self._stream(stream))

    # The 8-bit calls go straight to the library: for a few rows the call costs more than the kernel, so it is kept short.

    def _matrix8(self, m, name, shape):
        """What the library takes for a Matrix8 of this shape."""
        if type(m) is Matrix8 and m.shape == shape and m.index == self.index and m.codes_now() == m.codes_at and m.scales_now() == m.scales_at:
            return m.ref
        if not isinstance(m, Matrix8):
            raise TypeError("%s: a Matrix8 is expected" % name)
        if m.index != self.index:
            raise TypeError("%s: a matrix on %s is expected" % (name, self.device))
        if m.shape != shape:
            raise ValueError("%s: shape %s is expected, not %s" % (name, tuple(shape), tuple(m.shape)))
        m.stand(name)
        return m.ref

    def _active(self, active):
        return self._tensor(active, "active", (self.n_seqs,), torch.uint8)[0]

    def quantize8(self, x, out, active=None, stream=None):
        """The rows of x in 8 bits."""
        dim = x.shape[-1]
        shape = (self.rows, dim)
        px, sx = self._tensor(x, "x", shape, self.torch_dtype)
        status = self.lib.speca_layer_quantize8(self.handle, dim, px, sx[0], None if active is None else self._active(active),
                                                self._matrix8(out, "out", shape),
                                                torch._C._cuda_getCurrentRawStream(self.index) if stream is None else self._stream(stream))
        if status:
            _check_layer(status, self.handle)

    def norm8(self, x, out, kind=SPECA_NORM_RMS, branch=None, gate=None, scale=None, shift=None, weight=None, x_out=None, active=None,
              stream=None):
        """x' = x + gate * branch; out = 8 bits of norm(x') * weight * (1 + scale) + shift, the modulations by sequence."""
        dim, dt, tensor = x.shape[-1], self.torch_dtype, self._tensor
        shape = (self.rows, dim)
        px, sx = tensor(x, "x", shape, dt)
        pb, sb = (None, _NO_STRIDE) if branch is None else tensor(branch, "branch", shape, dt)
        po, so = (None, _NO_STRIDE) if x_out is None else tensor(x_out, "x_out", shape, dt)
        pw = None if weight is None else tensor(weight, "weight", (dim,), dt)[0]
        if gate is None and scale is None and shift is None:
            (pg, ps, pt), mod_stride = _NO_MODULATIONS, 0
        else:
            (pg, ps, pt), mod_stride = self._modulations((gate, scale, shift), dim)
        status = self.lib.speca_layer_norm8(self.handle, kind, dim, px, sx[0], pb, sb[0], pg, ps, pt, mod_stride, pw,
                                            None if active is None else self._active(active), po, so[0],
                                            self._matrix8(out, "out", shape),
                                            torch._C._cuda_getCurrentRawStream(self.index) if stream is None else self._stream(stream))
        if status:
            _check_layer(status, self.handle)

    def matmul8(self, a, w, out, bias=None, activation=SPECA_ACT_NONE, residual=None, gate=None, active=None, stream=None):
        """out = residual + gate * act(a w^T + bias), the gate by sequence; ``out``: a tensor of the layer's type, or a Matrix8 (which
        takes no residual and no gate)."""
        if not isinstance(w, Matrix8):
            raise TypeError("w: a Matrix8 is expected")
        (n, k), dt, tensor = w.shape, self.torch_dtype, self._tensor
        shape = (self.rows, n)
        ra = self._matrix8(a, "a", (self.rows, k))
        rw = w.ref if w.index == self.index and w.codes_now() == w.codes_at and w.scales_now() == w.scales_at else self._matrix8(w, "w", (n, k))
        if isinstance(out, Matrix8):
            eight, po, so = self._matrix8(out, "out", shape), None, _NO_STRIDE
        else:
            eight, (po, so) = None, tensor(out, "out", shape, dt)
        pb = None if bias is None else tensor(bias, "bias", (n,), dt)[0]
        pr, sr = (None, _NO_STRIDE) if residual is None else tensor(residual, "residual", shape, dt)
        pg, sg = (None, _NO_STRIDE) if gate is None else tensor(gate, "gate", (self.n_seqs, n), dt)
        status = self.lib.speca_layer_matmul8(self.handle, n, k, ra, rw, pb, activation, pr, sr[0], pg, sg[0],
                                              None if active is None else self._active(active), po, so[0], eight,
                                              torch._C._cuda_getCurrentRawStream(self.index) if stream is None else self._stream(stream))
        if status:
            _check_layer(status, self.handle)

    def check(self, stream=None):
        """Waits for `stream` and raises if a kernel of this layer gave up on a bounded wait."""
        speca_layer_check(self.handle, self._stream(stream))
