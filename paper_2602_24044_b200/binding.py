"""Thin ctypes binding of liblora_b200.so: same names as the C entry points, argument
marshalling only.  Every step of the LoRA forward runs inside the CUDA library; PyTorch is
used by callers for device memory and streams.

The library must have been built (``python -m paper_2602_24044_b200.build``); loading fails
loudly otherwise.  There is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, Optional, Sequence

import numpy as np

from . import build as _build

LORA_OK = 0
A_DIN_MAJOR = 0
A_RANK_MAJOR = 1
PACKED = 2
META_HEADER_WORDS = 16

EXPORTS = [
    "lora_status_string", "lora_last_cuda_error", "lora_launch_count",
    "lora_pool_bytes", "lora_pool_create", "lora_pool_destroy", "lora_pool_load_slot",
    "lora_pool_evict_slot", "lora_pool_acquire", "lora_pool_read_slot", "lora_pool_slot_info",
    "lora_pool_poll_status", "lora_pool_reset_status", "lora_pool_set_tuning",
    "lora_segments_bytes", "lora_build_segments", "lora_workspace_bytes",
    "lora_bgmv_apply", "lora_sgmv_apply", "lora_apply_host", "lora_bgmv_apply_static",
    "lora_bgmv_apply_multi", "lora_pool_check_status", "lora_pool_selftest_wait_expiry", "lora_pool_plan",
    "lora_policy_create", "lora_policy_destroy", "lora_policy_lookup", "lora_policy_slot",
    "lora_policy_touch", "lora_policy_pin", "lora_policy_unpin", "lora_policy_choose_victim",
    "lora_policy_assign", "lora_policy_release", "lora_policy_admit", "lora_policy_stats",
    "lora_kv_bytes", "lora_kv_layer_range", "lora_kv_create", "lora_kv_destroy", "lora_kv_check_status",
    "lora_kv_tables_bytes", "lora_kv_build_tables", "lora_kv_release", "lora_qk_norm_rope",
    "lora_kv_append", "lora_kv_read", "lora_kv_workspace_bytes", "lora_kv_attention",
    "lora_add_norm", "lora_qk_norm_rope_axes", "lora_kv_append_axes", "lora_kv_axis_positions",
    "lora_sample", "lora_sample_workspace_bytes",
]
STATIC_SCRATCH_BYTES = 2 * 1024 * 1024


class LoraError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = int(status)
        msg = _lib().lora_status_string(status).decode()
        if status == 9:
            msg += " (cudaError %d)" % _lib().lora_last_cuda_error()
        super().__init__("%s: %s" % (where, msg))


class _Target(ctypes.Structure):
    _fields_ = [("d_in", ctypes.c_int32), ("d_out", ctypes.c_int32)]


class _PoolDesc(ctypes.Structure):
    _fields_ = [("device", ctypes.c_int32), ("num_slots", ctypes.c_int32),
                ("r_max", ctypes.c_int32), ("num_targets", ctypes.c_int32),
                ("targets", ctypes.POINTER(_Target)), ("device_buf", ctypes.c_void_p),
                ("device_buf_bytes", ctypes.c_size_t)]


class _AdapterHost(ctypes.Structure):
    _fields_ = [("rank", ctypes.c_int32), ("scale", ctypes.c_float),
                ("A", ctypes.POINTER(ctypes.c_void_p)), ("B", ctypes.POINTER(ctypes.c_void_p)),
                ("a_layout", ctypes.c_int32), ("trust_pinned", ctypes.c_int32)]


class _ApplyItem(ctypes.Structure):
    _fields_ = [("target", ctypes.c_int32), ("x", ctypes.c_void_p), ("ldx", ctypes.c_int64),
                ("y_base", ctypes.c_void_p), ("ldyb", ctypes.c_int64),
                ("y", ctypes.c_void_p), ("ldy", ctypes.c_int64)]


class _StepBuffers(ctypes.Structure):
    _fields_ = [("x_dev", ctypes.c_void_p), ("y_base_dev", ctypes.c_void_p),
                ("y_dev", ctypes.c_void_p), ("slot_idx_dev", ctypes.c_void_p),
                ("meta_dev", ctypes.c_void_p), ("meta_bytes", ctypes.c_size_t),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class _KvDesc(ctypes.Structure):
    _fields_ = [("device", ctypes.c_int32), ("num_layers", ctypes.c_int32),
                ("num_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("device_buf", ctypes.c_void_p),
                ("device_buf_bytes", ctypes.c_size_t)]


class _QkArgs(ctypes.Structure):
    _fields_ = [("device", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("eps", ctypes.c_float), ("num_positions", ctypes.c_int32),
                ("q", ctypes.c_void_p), ("ldq", ctypes.c_int64),
                ("k", ctypes.c_void_p), ("ldk", ctypes.c_int64),
                ("v", ctypes.c_void_p), ("ldv", ctypes.c_int64),
                ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p),
                ("cos_sin", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("q_out", ctypes.c_void_p), ("ldqo", ctypes.c_int64),
                ("k_out", ctypes.c_void_p), ("ldko", ctypes.c_int64)]
    max_tokens = 2 ** 31 - 1
    axes = None                          # a reference to a _RopeAxes where positions are on several axes


class _RopeAxes(ctypes.Structure):
    _fields_ = [("num_axes", ctypes.c_int32), ("ld_positions", ctypes.c_int64),
                ("axis_of_pair", ctypes.c_char_p)]


class _NormArgs(ctypes.Structure):
    _fields_ = [("device", ctypes.c_int32), ("width", ctypes.c_int32),
                ("group", ctypes.c_int32), ("eps", ctypes.c_float),
                ("x", ctypes.c_void_p), ("ldx", ctypes.c_int64), ("weight", ctypes.c_void_p),
                ("residual", ctypes.c_void_p), ("ldr", ctypes.c_int64),
                ("residual_out", ctypes.c_void_p), ("ldro", ctypes.c_int64),
                ("out", ctypes.c_void_p), ("ldo", ctypes.c_int64),
                ("codes", ctypes.c_void_p), ("ldc", ctypes.c_int64),
                ("scales", ctypes.c_void_p), ("lds", ctypes.c_int64)]
    max_tokens = 2 ** 31 - 1


class _SampleArgs(ctypes.Structure):
    _fields_ = [("device", ctypes.c_int32), ("vocab", ctypes.c_int32), ("logits_type", ctypes.c_int32),
                ("logits", ctypes.c_void_p), ("ld", ctypes.c_int64),
                ("temperature", ctypes.c_void_p), ("top_k", ctypes.c_void_p),
                ("top_p", ctypes.c_void_p), ("min_p", ctypes.c_void_p), ("uniform", ctypes.c_void_p),
                ("token", ctypes.c_void_p), ("logprob", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]
    max_tokens = 2 ** 31 - 1
    own_workspace = None                 # made here: kept for the streams of the calls
    streams = frozenset()
    zero_first = False                   # made in a capture: no zeros before a call has put them there


_handle = None


def library_path() -> str:
    return _build.LIB


def _lib():
    global _handle
    if _handle is None:
        path = library_path()
        if not os.path.exists(path):
            raise RuntimeError(
                "liblora_b200.so is missing (%s): build it with "
                "`python -m paper_2602_24044_b200.build`; there is no fallback path" % path)
        lib = ctypes.CDLL(path)
        lib.lora_status_string.restype = ctypes.c_char_p
        lib.lora_status_string.argtypes = [ctypes.c_int]
        lib.lora_last_cuda_error.restype = ctypes.c_int32
        lib.lora_launch_count.restype = ctypes.c_int64
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        sigs = {
            "lora_pool_bytes": [ctypes.POINTER(_PoolDesc), ctypes.POINTER(sz)],
            "lora_pool_create": [ctypes.POINTER(_PoolDesc), ctypes.POINTER(vp)],
            "lora_pool_destroy": [vp],
            "lora_pool_load_slot": [vp, i32, ctypes.POINTER(_AdapterHost), vp, vp],
            "lora_pool_evict_slot": [vp, i32, vp, vp],
            "lora_pool_acquire": [vp, ctypes.POINTER(i32), i32, vp],
            "lora_pool_read_slot": [vp, i32, i32, vp, vp, vp],
            "lora_pool_slot_info": [vp, i32, ctypes.POINTER(i32), ctypes.POINTER(ctypes.c_float)],
            "lora_pool_poll_status": [vp, vp, vp],
            "lora_pool_reset_status": [vp, vp],
            "lora_pool_set_tuning": [vp, i32, i32],
            "lora_segments_bytes": [i32, i32, i32, ctypes.POINTER(sz)],
            "lora_build_segments": [vp, vp, i32, i32, i32, vp, sz, vp],
            "lora_workspace_bytes": [vp, i32, ctypes.POINTER(sz)],
            "lora_bgmv_apply": [vp, i32, vp, i64, vp, i64, vp, i64, vp, i32, vp, vp, sz, vp],
            "lora_sgmv_apply": [vp, i32, vp, i64, vp, i64, vp, i64, vp, i32, vp, sz, vp],
            "lora_bgmv_apply_static": [vp, i32, vp, i64, vp, i64, vp, i64, vp, i32, vp, vp],
            "lora_apply_host": [vp, i32, i32, vp, vp, vp, vp, i32, i32, i32,
                                ctypes.POINTER(_StepBuffers), vp],
            "lora_bgmv_apply_multi": [vp, ctypes.POINTER(_ApplyItem), i32, vp, i32, vp, vp, sz, vp],
            "lora_pool_check_status": [vp, vp, ctypes.POINTER(i32)],
            "lora_pool_selftest_wait_expiry": [vp, i32, vp, vp],
            "lora_pool_plan": [sz, ctypes.POINTER(_Target), i32, i32, ctypes.POINTER(i32),
                               ctypes.POINTER(sz)],
            "lora_policy_create": [i32, ctypes.POINTER(vp)],
            "lora_policy_destroy": [vp],
            "lora_policy_lookup": [vp, i64, ctypes.POINTER(i32)],
            "lora_policy_slot": [vp, i32, ctypes.POINTER(i64), ctypes.POINTER(i32)],
            "lora_policy_touch": [vp, i32],
            "lora_policy_pin": [vp, ctypes.POINTER(i32), i32],
            "lora_policy_unpin": [vp, ctypes.POINTER(i32), i32],
            "lora_policy_choose_victim": [vp, ctypes.POINTER(i32), ctypes.POINTER(i64)],
            "lora_policy_assign": [vp, i32, i64],
            "lora_policy_release": [vp, i32],
            "lora_policy_admit": [vp, ctypes.POINTER(i64), i32, ctypes.POINTER(i32),
                                  ctypes.POINTER(i32), ctypes.POINTER(i64), i32, ctypes.POINTER(i32)],
            "lora_policy_stats": [vp, ctypes.POINTER(i64), ctypes.POINTER(i64), ctypes.POINTER(i64)],
            "lora_kv_bytes": [ctypes.POINTER(_KvDesc), ctypes.POINTER(sz)],
            "lora_kv_layer_range": [ctypes.POINTER(_KvDesc), i32, ctypes.POINTER(sz), ctypes.POINTER(sz)],
            "lora_kv_create": [ctypes.POINTER(_KvDesc), ctypes.POINTER(vp)],
            "lora_kv_destroy": [vp],
            "lora_kv_check_status": [vp, vp, ctypes.POINTER(i32)],
            "lora_kv_tables_bytes": [vp, i32, i32, ctypes.POINTER(sz)],
            "lora_kv_build_tables": [vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, i64, vp, vp, vp, sz, vp],
            "lora_kv_release": [vp, vp, i32, i32, vp, vp, i64, vp, vp, vp],
            "lora_qk_norm_rope": [ctypes.POINTER(_QkArgs), i32, vp],
            "lora_kv_append": [vp, i32, ctypes.POINTER(_QkArgs), vp, i32, vp],
            "lora_kv_read": [vp, i32, vp, i32, vp, i64, vp, i64, vp],
            "lora_kv_workspace_bytes": [vp, ctypes.POINTER(sz)],
            "lora_kv_attention": [vp, i32, vp, i64, vp, i64, vp, ctypes.c_float, vp, i32, i32, vp, i64,
                                  vp, sz, vp],
            "lora_sample_workspace_bytes": [i32, ctypes.POINTER(sz)],
            "lora_sample": [ctypes.POINTER(_SampleArgs), i32, vp],
            "lora_add_norm": [ctypes.POINTER(_NormArgs), i32, vp],
            "lora_qk_norm_rope_axes": [ctypes.POINTER(_QkArgs), ctypes.POINTER(_RopeAxes), i32, vp],
            "lora_kv_append_axes": [vp, i32, ctypes.POINTER(_QkArgs), ctypes.POINTER(_RopeAxes), vp, i32, vp],
            "lora_kv_axis_positions": [vp, vp, i32, i32, vp, vp, i32, vp, i64, vp],
        }
        for name, args in sigs.items():
            fn = getattr(lib, name)
            fn.restype = ctypes.c_int
            fn.argtypes = args
        _handle = lib
    return _handle


def _check(status: int, where: str) -> None:
    if status != LORA_OK:
        raise LoraError(status, where)


def _ptr(obj) -> Optional[int]:
    """Address of a torch tensor / numpy array / int / None."""
    if obj is None or type(obj) is int:
        return obj
    try:
        return obj.data_ptr()
    except AttributeError:
        pass
    if isinstance(obj, int):
        return int(obj)
    if isinstance(obj, np.ndarray):
        return int(obj.ctypes.data)
    raise TypeError("cannot take the address of %r" % type(obj))


def _stream(s) -> Optional[int]:
    if s is None or type(s) is int:
        return s
    return int(s.cuda_stream)


def stream_handle(s) -> int:
    """The cudaStream_t behind a torch stream, an int or None (0: the device's default stream)."""
    return s if type(s) is int else 0 if s is None else int(s.cuda_stream)


def _nbytes(obj) -> int:
    if hasattr(obj, "element_size"):
        return int(obj.numel() * obj.element_size())
    return int(obj.nbytes)


def _desc(num_slots, r_max, targets, device, buf=None, buf_bytes=0):
    arr = (_Target * len(targets))(*[_Target(int(a), int(b)) for a, b in targets])
    d = _PoolDesc(int(device), int(num_slots), int(r_max), len(targets), arr, _ptr(buf),
                  int(buf_bytes))
    d._keep = arr
    return d


# ------------------------------------------------------------------------------------------
# the C entry points
# ------------------------------------------------------------------------------------------
def status_string(status: int) -> str:
    return _lib().lora_status_string(int(status)).decode()


def launch_count() -> int:
    return int(_lib().lora_launch_count())


def pool_bytes(num_slots: int, r_max: int, targets: Sequence, device: int = 0) -> int:
    out = ctypes.c_size_t(0)
    d = _desc(num_slots, r_max, targets, device)
    _check(_lib().lora_pool_bytes(ctypes.byref(d), ctypes.byref(out)), "lora_pool_bytes")
    return int(out.value)


def pool_create(num_slots: int, r_max: int, targets: Sequence, device_buf, device: int = 0,
                device_buf_bytes: Optional[int] = None) -> int:
    out = ctypes.c_void_p(None)
    nbytes = _nbytes(device_buf) if device_buf_bytes is None else device_buf_bytes
    d = _desc(num_slots, r_max, targets, device, device_buf, nbytes)
    _check(_lib().lora_pool_create(ctypes.byref(d), ctypes.byref(out)), "lora_pool_create")
    return int(out.value)


def pool_destroy(pool: int) -> None:
    _check(_lib().lora_pool_destroy(pool), "lora_pool_destroy")


def pool_load_slot(pool: int, slot: int, rank: int, scale: float, A: Sequence, B: Sequence,
                   a_layout: int = A_DIN_MAJOR, load_stream=None, compute_stream=None,
                   trust_pinned: bool = False) -> None:
    n = len(A)
    Ap = (ctypes.c_void_p * n)(*[_ptr(a) for a in A])
    Bp = (ctypes.c_void_p * n)(*[_ptr(b) for b in B])
    ad = _AdapterHost(int(rank), float(scale), Ap, Bp, int(a_layout), int(bool(trust_pinned)))
    _check(_lib().lora_pool_load_slot(pool, int(slot), ctypes.byref(ad), _stream(load_stream),
                                      _stream(compute_stream)), "lora_pool_load_slot")


def pool_evict_slot(pool: int, slot: int, load_stream=None, compute_stream=None) -> None:
    _check(_lib().lora_pool_evict_slot(pool, int(slot), _stream(load_stream),
                                       _stream(compute_stream)), "lora_pool_evict_slot")


def pool_acquire(pool: int, slots: Sequence[int], compute_stream=None) -> None:
    arr = (ctypes.c_int32 * max(len(slots), 1))(*[int(s) for s in slots])
    _check(_lib().lora_pool_acquire(pool, arr, len(slots), _stream(compute_stream)),
           "lora_pool_acquire")


def pool_read_slot(pool: int, slot: int, target: int, A_host, B_host, stream=None) -> None:
    _check(_lib().lora_pool_read_slot(pool, int(slot), int(target), _ptr(A_host), _ptr(B_host),
                                      _stream(stream)), "lora_pool_read_slot")


def pool_slot_info(pool: int, slot: int):
    r = ctypes.c_int32(0)
    s = ctypes.c_float(0)
    _check(_lib().lora_pool_slot_info(pool, int(slot), ctypes.byref(r), ctypes.byref(s)),
           "lora_pool_slot_info")
    return int(r.value), float(s.value)


def pool_poll_status(pool: int, host_out, stream=None) -> None:
    _check(_lib().lora_pool_poll_status(pool, _ptr(host_out), _stream(stream)),
           "lora_pool_poll_status")


def pool_reset_status(pool: int, stream=None) -> None:
    _check(_lib().lora_pool_reset_status(pool, _stream(stream)), "lora_pool_reset_status")


def pool_check_status(pool: int, stream=None):
    """Synchronises `stream`; returns the four status words.  Raises LoraError(10) when a bounded
    device-side wait has expired since the last reset."""
    w = (ctypes.c_int32 * 4)()
    _check(_lib().lora_pool_check_status(pool, _stream(stream), w), "lora_pool_check_status")
    return [int(v) for v in w]


def pool_selftest_wait_expiry(pool: int, polls: int, witness_dev=None, stream=None) -> None:
    _check(_lib().lora_pool_selftest_wait_expiry(pool, int(polls), _ptr(witness_dev),
                                                 _stream(stream)), "lora_pool_selftest_wait_expiry")


def pool_plan(bytes_budget: int, targets: Sequence, r_max: int):
    """(num_slots that fit in bytes_budget, bytes one slot costs)."""
    arr = (_Target * len(targets))(*[_Target(int(a), int(b)) for a, b in targets])
    n, per = ctypes.c_int32(0), ctypes.c_size_t(0)
    _check(_lib().lora_pool_plan(int(bytes_budget), arr, len(targets), int(r_max), ctypes.byref(n),
                                 ctypes.byref(per)), "lora_pool_plan")
    return int(n.value), int(per.value)


# slot policy (host-side bookkeeping, no CUDA call)
def policy_create(num_slots: int) -> int:
    out = ctypes.c_void_p(None)
    _check(_lib().lora_policy_create(int(num_slots), ctypes.byref(out)), "lora_policy_create")
    return int(out.value)


def policy_destroy(policy: int) -> None:
    _check(_lib().lora_policy_destroy(policy), "lora_policy_destroy")


def policy_lookup(policy: int, adapter: int) -> int:
    out = ctypes.c_int32(0)
    _check(_lib().lora_policy_lookup(policy, int(adapter), ctypes.byref(out)), "lora_policy_lookup")
    return int(out.value)


def policy_slot(policy: int, slot: int):
    a, p = ctypes.c_int64(0), ctypes.c_int32(0)
    _check(_lib().lora_policy_slot(policy, int(slot), ctypes.byref(a), ctypes.byref(p)),
           "lora_policy_slot")
    return int(a.value), int(p.value)


def policy_touch(policy: int, slot: int) -> None:
    _check(_lib().lora_policy_touch(policy, int(slot)), "lora_policy_touch")


def _i32_array(values):
    return (ctypes.c_int32 * max(len(values), 1))(*[int(v) for v in values])


def policy_pin(policy: int, slots: Sequence[int]) -> None:
    _check(_lib().lora_policy_pin(policy, _i32_array(slots), len(slots)), "lora_policy_pin")


def policy_unpin(policy: int, slots: Sequence[int]) -> None:
    _check(_lib().lora_policy_unpin(policy, _i32_array(slots), len(slots)), "lora_policy_unpin")


def policy_choose_victim(policy: int):
    """(slot, adapter it holds now or -1)."""
    s, a = ctypes.c_int32(0), ctypes.c_int64(0)
    _check(_lib().lora_policy_choose_victim(policy, ctypes.byref(s), ctypes.byref(a)),
           "lora_policy_choose_victim")
    return int(s.value), int(a.value)


def policy_assign(policy: int, slot: int, adapter: int) -> None:
    _check(_lib().lora_policy_assign(policy, int(slot), int(adapter)), "lora_policy_assign")


def policy_release(policy: int, slot: int) -> None:
    _check(_lib().lora_policy_release(policy, int(slot)), "lora_policy_release")


def policy_admit(policy: int, adapters: Sequence[int], miss_cap: Optional[int] = None):
    """(slot_idx int32 array, [(slot, adapter) to load, ...]) for one batch of requests."""
    n = len(adapters)
    cap = n if miss_cap is None else int(miss_cap)
    ids = (ctypes.c_int64 * max(n, 1))(*[int(a) for a in adapters])
    sidx = (ctypes.c_int32 * max(n, 1))()
    ms = (ctypes.c_int32 * max(cap, 1))()
    ma = (ctypes.c_int64 * max(cap, 1))()
    nm = ctypes.c_int32(0)
    _check(_lib().lora_policy_admit(policy, ids, n, sidx, ms, ma, cap, ctypes.byref(nm)),
           "lora_policy_admit")
    return (np.array(sidx[:n], dtype=np.int32),
            [(int(ms[k]), int(ma[k])) for k in range(nm.value)])


def policy_stats(policy: int):
    h, m, e = ctypes.c_int64(0), ctypes.c_int64(0), ctypes.c_int64(0)
    _check(_lib().lora_policy_stats(policy, ctypes.byref(h), ctypes.byref(m), ctypes.byref(e)),
           "lora_policy_stats")
    return int(h.value), int(m.value), int(e.value)


def pool_set_tuning(pool: int, key: int, value: int) -> None:
    _check(_lib().lora_pool_set_tuning(pool, int(key), int(value)), "lora_pool_set_tuning")


def segments_bytes(T: int, num_slots: int, tile_m: int) -> int:
    out = ctypes.c_size_t(0)
    _check(_lib().lora_segments_bytes(int(T), int(num_slots), int(tile_m), ctypes.byref(out)),
           "lora_segments_bytes")
    return int(out.value)


def build_segments(pool: int, slot_idx_dev, T: int, tile_m: int, long_min: int, meta_dev,
                   meta_bytes: Optional[int] = None, stream=None) -> None:
    nbytes = _nbytes(meta_dev) if meta_bytes is None else meta_bytes
    _check(_lib().lora_build_segments(pool, _ptr(slot_idx_dev), int(T), int(tile_m), int(long_min),
                                      _ptr(meta_dev), nbytes, _stream(stream)),
           "lora_build_segments")


def workspace_bytes(pool: int, T_max: int) -> int:
    out = ctypes.c_size_t(0)
    _check(_lib().lora_workspace_bytes(pool, int(T_max), ctypes.byref(out)), "lora_workspace_bytes")
    return int(out.value)


def bgmv_apply(pool: int, target: int, x, ldx: int, y_base, ldyb: int, y, ldy: int, slot_idx_dev,
               T: int, meta_dev, workspace, workspace_bytes_: Optional[int] = None,
               stream=None) -> None:
    nbytes = (_nbytes(workspace) if workspace is not None else 0) \
        if workspace_bytes_ is None else workspace_bytes_
    _check(_lib().lora_bgmv_apply(pool, int(target), _ptr(x), int(ldx), _ptr(y_base), int(ldyb),
                                  _ptr(y), int(ldy), _ptr(slot_idx_dev), int(T), _ptr(meta_dev),
                                  _ptr(workspace), nbytes, _stream(stream)), "lora_bgmv_apply")


def make_apply_items(items: Sequence):
    """items: (target, x, ldx, y_base, ldyb, y, ldy) tuples -> a C array for bgmv_apply_multi (build
    it once when the same launch is issued repeatedly)."""
    arr = (_ApplyItem * max(len(items), 1))()
    for k, (target, x, ldx, yb, ldyb, y, ldy) in enumerate(items):
        arr[k] = _ApplyItem(int(target), _ptr(x), int(ldx), _ptr(yb), int(ldyb), _ptr(y), int(ldy))
    return arr, len(items)


def bgmv_apply_multi(pool: int, items, slot_idx_dev, T: int, meta_dev, workspace,
                     workspace_bytes_: Optional[int] = None, stream=None) -> None:
    """Several projections of one decode batch in one launch; `items` as for make_apply_items (or
    its result)."""
    arr, n = items if isinstance(items, tuple) and len(items) == 2 and not isinstance(items[0], tuple) \
        else make_apply_items(items)
    nbytes = (_nbytes(workspace) if workspace is not None else 0) \
        if workspace_bytes_ is None else workspace_bytes_
    _check(_lib().lora_bgmv_apply_multi(pool, arr, n, _ptr(slot_idx_dev), int(T), _ptr(meta_dev),
                                        _ptr(workspace), nbytes, _stream(stream)),
           "lora_bgmv_apply_multi")


def bgmv_apply_static(pool: int, target: int, x, ldx: int, y_base, ldyb: int, y, ldy: int,
                      slot_idx_dev, T: int, meta_dev, stream=None) -> None:
    """lora_bgmv_apply without a workspace argument: the scratch is a fixed array inside the
    library (for callers that must not allocate device memory).  See lora_b200.h for the size
    limit and the rule about overlapping calls."""
    _check(_lib().lora_bgmv_apply_static(pool, int(target), _ptr(x), int(ldx), _ptr(y_base),
                                         int(ldyb), _ptr(y), int(ldy), _ptr(slot_idx_dev), int(T),
                                         _ptr(meta_dev), _stream(stream)), "lora_bgmv_apply_static")


def sgmv_apply(pool: int, target: int, x, ldx: int, y_base, ldyb: int, y, ldy: int, meta_dev,
               T: int, workspace, workspace_bytes_: Optional[int] = None, stream=None) -> None:
    nbytes = (_nbytes(workspace) if workspace is not None else 0) \
        if workspace_bytes_ is None else workspace_bytes_
    _check(_lib().lora_sgmv_apply(pool, int(target), _ptr(x), int(ldx), _ptr(y_base), int(ldyb),
                                  _ptr(y), int(ldy), _ptr(meta_dev), int(T), _ptr(workspace),
                                  nbytes, _stream(stream)), "lora_sgmv_apply")


def apply_host(pool: int, target: int, kind: int, x_host, y_base_host, y_host, slot_idx_host,
               T: int, tile_m: int, long_min: int, x_dev, y_base_dev, y_dev, slot_idx_dev,
               meta_dev, workspace, stream=None) -> None:
    sb = _StepBuffers(_ptr(x_dev), _ptr(y_base_dev), _ptr(y_dev), _ptr(slot_idx_dev),
                      _ptr(meta_dev), _nbytes(meta_dev), _ptr(workspace), _nbytes(workspace))
    _check(_lib().lora_apply_host(pool, int(target), int(kind), _ptr(x_host), _ptr(y_base_host),
                                  _ptr(y_host), _ptr(slot_idx_host), int(T), int(tile_m),
                                  int(long_min), ctypes.byref(sb), _stream(stream)),
           "lora_apply_host")


# ------------------------------------------------------------------------------------------
# the paged 4-bit key/value cache and the operators around it
# ------------------------------------------------------------------------------------------
def _kv_desc(num_layers, num_pages, page_size, num_q_heads, num_kv_heads, head_dim, device, buf=None,
             buf_bytes=0):
    return _KvDesc(int(device), int(num_layers), int(num_pages), int(page_size), int(num_q_heads),
                   int(num_kv_heads), int(head_dim), _ptr(buf), int(buf_bytes))


def kv_bytes(num_layers: int, num_pages: int, page_size: int, num_q_heads: int, num_kv_heads: int,
             head_dim: int, device: int = 0) -> int:
    out = ctypes.c_size_t(0)
    d = _kv_desc(num_layers, num_pages, page_size, num_q_heads, num_kv_heads, head_dim, device)
    _check(_lib().lora_kv_bytes(ctypes.byref(d), ctypes.byref(out)), "lora_kv_bytes")
    return int(out.value)


def kv_layer_range(layer: int, num_layers: int, num_pages: int, page_size: int, num_q_heads: int,
                   num_kv_heads: int, head_dim: int, device: int = 0):
    """(byte offset inside the device buffer, bytes) of one layer's pages."""
    off, n = ctypes.c_size_t(0), ctypes.c_size_t(0)
    d = _kv_desc(num_layers, num_pages, page_size, num_q_heads, num_kv_heads, head_dim, device)
    _check(_lib().lora_kv_layer_range(ctypes.byref(d), int(layer), ctypes.byref(off), ctypes.byref(n)),
           "lora_kv_layer_range")
    return int(off.value), int(n.value)


def kv_create(num_layers: int, num_pages: int, page_size: int, num_q_heads: int, num_kv_heads: int,
              head_dim: int, device_buf, device: int = 0, device_buf_bytes: Optional[int] = None) -> int:
    out = ctypes.c_void_p(None)
    nbytes = _nbytes(device_buf) if device_buf_bytes is None else device_buf_bytes
    d = _kv_desc(num_layers, num_pages, page_size, num_q_heads, num_kv_heads, head_dim, device,
                 device_buf, nbytes)
    _check(_lib().lora_kv_create(ctypes.byref(d), ctypes.byref(out)), "lora_kv_create")
    return int(out.value)


def kv_destroy(kv: int) -> None:
    _check(_lib().lora_kv_destroy(kv), "lora_kv_destroy")


def kv_check_status(kv: int, stream=None):
    """Synchronises `stream`; returns the four status words.  Raises LoraError(10) when a bounded
    device-side wait has expired since the handle was created."""
    w = (ctypes.c_int32 * 4)()
    _check(_lib().lora_kv_check_status(kv, _stream(stream), w), "lora_kv_check_status")
    return [int(v) for v in w]


def kv_tables_bytes(kv: int, R: int, T: int) -> int:
    out = ctypes.c_size_t(0)
    _check(_lib().lora_kv_tables_bytes(kv, int(R), int(T), ctypes.byref(out)), "lora_kv_tables_bytes")
    return int(out.value)


def kv_build_tables(kv: int, kv_len, q_len, R: int, T: int, free_pages, free_count, block_table,
                    ld_table: int, tables, *, max_q: int = 0, window: int = 0, kv_len_out=None,
                    free_count_out=None, tables_bytes: Optional[int] = None, stream=None) -> None:
    nbytes = _nbytes(tables) if tables_bytes is None else tables_bytes
    p = _ptr
    status = _lib().lora_kv_build_tables(kv, p(kv_len), p(q_len), R, T, max_q, window, p(free_pages), p(free_count),
                                         p(block_table), ld_table, p(kv_len_out), p(free_count_out), p(tables), nbytes,
                                         _stream(stream))
    if status:
        _check(status, "lora_kv_build_tables")


def kv_release(kv: int, requests, n: int, R: int, kv_len, block_table, ld_table: int, free_pages,
               free_count, stream=None) -> None:
    _check(_lib().lora_kv_release(kv, _ptr(requests), int(n), int(R), _ptr(kv_len), _ptr(block_table),
                                  int(ld_table), _ptr(free_pages), _ptr(free_count), _stream(stream)),
           "lora_kv_release")


def _elements(what: str, t, dtype: str, device: int, n: int = 0) -> Optional[int]:
    """How many elements lie from a tensor's first to the end of its memory; None for a bare address.  n > 0: the
    tensor itself has to have that many, in a row."""
    if not hasattr(t, "untyped_storage"):
        return None
    if str(t.dtype) != "torch." + dtype or t.get_device() != device:
        raise LoraError(1, "%s (%s on %s, not %s on device %d)" % (what, t.dtype, t.device, dtype, device))
    if n and (t.numel() < n or not t.is_contiguous()):
        raise LoraError(1, "%s (needs %d values in a row)" % (what, n))
    return t.untyped_storage().nbytes() // t.element_size() - t.storage_offset()


def qk_args(*, num_q_heads: int, num_kv_heads: int, head_dim: int, q=None, ldq: int = 0, k=None,
            ldk: int = 0, v=None, ldv: int = 0, q_weight=None, k_weight=None, eps: float = 0.0,
            cos_sin=None, rot_dim: Optional[int] = None, num_positions: Optional[int] = None,
            interleaved: bool = False, positions=None, q_out=None, ldqo: Optional[int] = None, k_out=None,
            ldko: Optional[int] = None, axis_of_pair: Optional[Sequence[int]] = None, num_axes: Optional[int] = None,
            ld_positions: Optional[int] = None, device: int = 0):
    """The argument block of qk_norm_rope and kv_append (build it once when the same buffers are used
    again).  rot_dim, num_positions and the outputs' leading dimensions default to those of the tensors
    given.  The tensors must stay alive while the block is used; it keeps them, and a call for more tokens than
    they hold is refused.

    axis_of_pair: which axis turns each of the rot_dim / 2 rotation pairs; positions is then [axes, tokens], and
    the calls go to lora_qk_norm_rope_axes and lora_kv_append_axes (num_axes and ld_positions: as positions has
    them)."""
    if cos_sin is not None:
        num_positions = int(cos_sin.shape[0]) if num_positions is None else num_positions
        rot_dim = int(cos_sin.shape[1]) if rot_dim is None else rot_dim
    if q_out is not None and ldqo is None:
        ldqo = int(q_out.stride(0))
    if k_out is not None and ldko is None:
        ldko = int(k_out.stride(0))
    a = _QkArgs(int(device), int(num_q_heads), int(num_kv_heads), int(head_dim), int(rot_dim or 0),
                int(bool(interleaved)), float(eps), int(num_positions or 0), _ptr(q), int(ldq), _ptr(k),
                int(ldk), _ptr(v), int(ldv), _ptr(q_weight), _ptr(k_weight), _ptr(cos_sin),
                _ptr(positions), _ptr(q_out), int(ldqo or 0), _ptr(k_out), int(ldko or 0))
    a._keep = (q, k, v, q_weight, k_weight, cos_sin, positions, q_out, k_out)
    if axis_of_pair is not None:
        _set_axes(a, axis_of_pair, num_axes, ld_positions, positions)
    a.max_tokens = _max_tokens(a)
    return a


def _set_axes(a, axis_of_pair, num_axes, ld_positions, positions) -> None:
    axis = [int(x) for x in axis_of_pair]
    if len(axis) != a.rot_dim // 2 or min(axis, default=0) < 0 or max(axis, default=0) > 255:
        raise LoraError(2, "axis_of_pair (needs the axis of each of the %d rotation pairs)" % (a.rot_dim // 2))
    if hasattr(positions, "stride"):
        if (positions.dim() != 2 or (positions.stride(1) != 1 and positions.shape[1] > 1) or
                (ld_positions is None and positions.shape[0] > 1 and positions.stride(0) < positions.shape[1])):
            raise LoraError(1, "positions (needs a row of tokens for each axis)")
        num_axes = int(positions.shape[0]) if num_axes is None else num_axes
        if ld_positions is None:
            ld_positions = max(int(positions.stride(0)), int(positions.shape[1]))
    a._axes = _RopeAxes(int(num_axes or 0), int(ld_positions or 0), bytes(axis))
    a.axes = ctypes.byref(a._axes)


def _max_tokens(a) -> int:
    """The tokens that fit the memory from the tensors of an argument block on."""
    q, k, v, q_weight, k_weight, cos_sin, positions, q_out, k_out = a._keep
    most, d, device = 2 ** 31 - 1, a.head_dim, a.device
    for what, t, heads, ld in (("q", q, a.num_q_heads, a.ldq), ("k", k, a.num_kv_heads, a.ldk),
                               ("v", v, a.num_kv_heads, a.ldv), ("q_out", q_out, a.num_q_heads, a.ldqo),
                               ("k_out", k_out, a.num_kv_heads, a.ldko)):
        n = _elements(what, t, "bfloat16", device) if heads > 0 else None
        if n is not None:
            most = min(most, 0 if n < heads * d else most if ld <= 0 else (n - heads * d) // ld + 1)
    _elements("q_weight", q_weight, "bfloat16", device, d)
    _elements("k_weight", k_weight, "bfloat16", device, d)
    if cos_sin is not None:
        _elements("cos_sin", cos_sin, "float32", device, a.num_positions * a.rot_dim)
        n = _elements("positions", positions, "int32", device)
        if n is not None and a.axes is not None:
            if positions.shape[0] < a._axes.num_axes:
                raise LoraError(1, "positions (needs %d axes)" % a._axes.num_axes)
            most = min(most, a._axes.ld_positions, max(0, n - (a._axes.num_axes - 1) * a._axes.ld_positions))
        elif n is not None:
            if not positions.is_contiguous():
                raise LoraError(1, "positions (needs its values in a row)")
            most = min(most, n)
    return most


def _too_many(args, T: int, where: str) -> None:
    raise LoraError(1, "%s (the tensors given hold %d tokens, not %d)" % (where, args.max_tokens, T))


def qk_norm_rope(args, T: int, stream=None) -> None:
    """Per-head norm and rotation of T tokens' queries and keys; `args` from qk_args."""
    if T > args.max_tokens:
        _too_many(args, T, "qk_norm_rope")
    if args.axes is None:
        status = _lib().lora_qk_norm_rope(ctypes.byref(args), T, _stream(stream))
    else:
        status = _lib().lora_qk_norm_rope_axes(ctypes.byref(args), args.axes, T, _stream(stream))
    if status:
        _check(status, "lora_qk_norm_rope")


def kv_append(kv: int, layer: int, args, slots, T: int, stream=None) -> None:
    """qk_norm_rope with the keys and values also going to their slots of the cache as 4-bit rows."""
    if T > args.max_tokens:
        _too_many(args, T, "kv_append")
    if args.axes is None:
        status = _lib().lora_kv_append(kv, layer, ctypes.byref(args), _ptr(slots), T, _stream(stream))
    else:
        status = _lib().lora_kv_append_axes(kv, layer, ctypes.byref(args), args.axes, _ptr(slots), T, _stream(stream))
    if status:
        _check(status, "lora_kv_append")


def kv_axis_positions(kv: int, tables, R: int, T: int, spans, span_begin, num_spans: int, positions,
                      ld_positions: int, stream=None) -> None:
    """Positions of a batch's tokens on the three axes of images and videos."""
    status = _lib().lora_kv_axis_positions(kv, _ptr(tables), R, T, _ptr(spans), _ptr(span_begin), num_spans,
                                           _ptr(positions), ld_positions, _stream(stream))
    if status:
        _check(status, "lora_kv_axis_positions")


def kv_read(kv: int, layer: int, slots, n: int, k_out, ldk: int, v_out, ldv: int, stream=None) -> None:
    """Rows of the cache as the bf16 values they stand for."""
    status = _lib().lora_kv_read(kv, layer, _ptr(slots), n, _ptr(k_out), ldk, _ptr(v_out), ldv, _stream(stream))
    if status:
        _check(status, "lora_kv_read")


def kv_workspace_bytes(kv: int) -> int:
    out = ctypes.c_size_t(0)
    _check(_lib().lora_kv_workspace_bytes(kv, ctypes.byref(out)), "lora_kv_workspace_bytes")
    return int(out.value)


def kv_attention(kv: int, layer: int, q, ldq: int, out, ldo: int, lse, scale: float, tables, R: int,
                 T: int, block_table, ld_table: int, workspace, workspace_bytes_: Optional[int] = None,
                 stream=None) -> None:
    nbytes = workspace_bytes_
    if nbytes is None:
        nbytes = 0 if workspace is None else _nbytes(workspace)
    p = _ptr
    status = _lib().lora_kv_attention(kv, layer, p(q), ldq, p(out), ldo, p(lse), scale, p(tables), R, T, p(block_table),
                                      ld_table, p(workspace), nbytes, _stream(stream))
    if status:
        _check(status, "lora_kv_attention")


# ------------------------------------------------------------------------------------------
# rows between two projections
# ------------------------------------------------------------------------------------------
def _ld(what: str, t, ld: Optional[int], width: int) -> int:
    """The leading dimension of rows: as given, or that of a tensor of two dimensions."""
    if t is None or ld is not None or not hasattr(t, "stride"):
        return int(ld or 0)
    if t.dim() != 2 or t.shape[1] < width or (t.stride(1) != 1 and t.shape[1] > 1):
        raise LoraError(1, "%s (needs rows of %d values, each in a row)" % (what, width))
    return int(t.stride(0)) if t.shape[0] > 1 else max(int(t.stride(0)), int(t.shape[1]))


def norm_args(*, x, weight=None, eps: float = 1e-6, residual=None, residual_out=None, out=None, codes=None,
              scales=None, group: int = 0, width: Optional[int] = None, ldx: Optional[int] = None,
              ldr: Optional[int] = None, ldro: Optional[int] = None, ldo: Optional[int] = None,
              ldc: Optional[int] = None, lds: Optional[int] = None, device: int = 0):
    """The argument block of add_norm (build it once when the same buffers are used again).  width and the
    leading dimensions default to those of the tensors given; codes: float8_e4m3fn; scales: float32, with
    group = 32 uint8.  The tensors must stay alive while the block is used; it keeps them, and a call for more
    rows than they hold is refused."""
    n = int(x.shape[-1]) if width is None else int(width)
    groups = n // int(group) if group else 0
    lds = _ld("scales", scales, lds, groups)
    rows = [(what, t, _ld(what, t, ld, n)) for what, t, ld in (
        ("x", x, ldx), ("residual", residual, ldr), ("residual_out", residual_out, ldro), ("out", out, ldo),
        ("codes", codes, ldc))]
    (ldx, ldr, ldro, ldo, ldc) = (ld for _, _, ld in rows)
    a = _NormArgs(int(device), n, int(group), float(eps), _ptr(x), ldx, _ptr(weight), _ptr(residual), ldr,
                  _ptr(residual_out), ldro, _ptr(out), ldo, _ptr(codes), ldc, _ptr(scales), lds)
    a._keep = (x, weight, residual, residual_out, out, codes, scales)
    most = 2 ** 31 - 1
    for what, t, ld in rows + [("scales", scales, lds)]:
        need = groups if what == "scales" else n
        dtype = "float8_e4m3fn" if what == "codes" else "bfloat16" if what != "scales" else \
            "uint8" if group == 32 else "float32"
        have = None if t is None else _elements(what, t, dtype, int(device))
        if have is not None:
            most = min(most, 0 if have < need else most if ld <= 0 else (have - need) // ld + 1)
    if weight is not None:
        _elements("weight", weight, "bfloat16", int(device), n)
    a.max_tokens = most
    return a


def add_norm(args, T: int, stream=None) -> None:
    """Residual addition and norm of T rows; `args` from norm_args."""
    if T > args.max_tokens:
        _too_many(args, T, "add_norm")
    status = _lib().lora_add_norm(ctypes.byref(args), T, _stream(stream))
    if status:
        _check(status, "lora_add_norm")


# ------------------------------------------------------------------------------------------
# the next tokens
# ------------------------------------------------------------------------------------------
LOGITS_BF16, LOGITS_FP32 = 0, 1


def sample_workspace_bytes(R: int) -> int:
    out = ctypes.c_size_t(0)
    _check(_lib().lora_sample_workspace_bytes(int(R), ctypes.byref(out)), "lora_sample_workspace_bytes")
    return int(out.value)


def sample_args(*, logits, temperature, uniform, token, logprob=None, top_k=None, top_p=None, min_p=None,
                vocab: Optional[int] = None, ld: Optional[int] = None, logits_type: Optional[int] = None, workspace=None,
                workspace_bytes: Optional[int] = None, device: int = 0):
    """The argument block of sample (build it once when the same buffers are used again).  logits: bf16 or fp32
    rows; vocab, their type and leading dimension default to the tensor's.  The others hold one entry a row.  The
    tensors must stay alive while the block is used; it keeps them, and a call for more rows than they hold is
    refused.  workspace: made here where token is a tensor and none is given (calls with one block are then to be
    ordered on one stream, as they share their outputs too; a block made in a graph's capture clears its first words
    with every call; a block called on a bare stream handle is kept until that work is done)."""
    V = int(logits.shape[-1]) if vocab is None else int(vocab)
    ld = _ld("logits", logits, ld, V)
    kind = "bfloat16" if logits_type == LOGITS_BF16 else "float32"
    if logits_type is None:
        kind = "bfloat16" if str(getattr(logits, "dtype", "")) == "torch.bfloat16" else "float32"
        logits_type = LOGITS_BF16 if kind == "bfloat16" else LOGITS_FP32
    a = _SampleArgs(int(device), V, int(logits_type), _ptr(logits), ld, _ptr(temperature), _ptr(top_k), _ptr(top_p),
                    _ptr(min_p), _ptr(uniform), _ptr(token), _ptr(logprob))
    a._keep = (logits, temperature, top_k, top_p, min_p, uniform, token, logprob)
    most = 2 ** 31 - 1
    have = None if logits is None else _elements("logits", logits, kind, int(device))
    if have is not None:
        most = 0 if have < V else most if ld <= 0 else (have - V) // ld + 1
    for what, t, dtype in (("temperature", temperature, "float32"), ("top_k", top_k, "int32"), ("top_p", top_p, "float32"),
                           ("min_p", min_p, "float32"), ("uniform", uniform, "float32"), ("token", token, "int32"),
                           ("logprob", logprob, "float32")):
        have = None if t is None else _elements(what, t, dtype, int(device))
        if have is not None:
            if not t.is_contiguous():
                raise LoraError(1, "%s (needs its values in a row)" % what)
            most = min(most, have)
    a.max_tokens = most
    if workspace is None and hasattr(token, "new_zeros"):
        workspace, a.zero_first = _zeros(token, sample_workspace_bytes(min(most, 1 << 24)))
        a.own_workspace = workspace
    if workspace is not None:
        a.workspace = _ptr(workspace)
        a.workspace_bytes = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    return a


def _zeros(like, nbytes: int):
    """(int32 zeros beside a device tensor, ready for calls on any stream; False), or in a graph's capture (memory, True):
    zeros would be there from the graph's first replay on, and not for calls before that or in another graph."""
    import torch
    if torch.cuda.is_current_stream_capturing():
        return like.new_empty((nbytes + 3) // 4), True
    t = like.new_zeros((nbytes + 3) // 4)
    torch.cuda.current_stream(t.device).synchronize()
    return t, False


def _torch_stream(stream, device):
    import torch
    if type(stream) is int and stream:
        return torch.cuda.ExternalStream(stream, device)
    return stream if stream else torch.cuda.default_stream(device)


def _zero_counts(t, stream) -> None:
    """The words that a sampling workspace begins with, on the stream of the call that follows."""
    import torch
    with torch.cuda.stream(_torch_stream(stream, t.device)):
        t[:4].zero_()


def _record(t, stream) -> None:
    """A tensor made here is not given back to the allocator while work on `stream` may use it (a bare handle says
    nothing of how long its stream lives: there the caller keeps the block until the work is done)."""
    import torch
    if type(stream) is not int:
        t.record_stream(torch.cuda.default_stream(t.device) if stream is None else stream)


def sample(args, R: int, stream=None) -> None:
    """The next tokens of R requests; `args` from sample_args."""
    if R > args.max_tokens:
        _too_many(args, R, "sample")
    if args.own_workspace is not None and stream not in args.streams:
        _record(args.own_workspace, stream)
        args.streams = args.streams | {stream}
    if args.zero_first and args.workspace:
        _zero_counts(args.own_workspace, stream)
    status = _lib().lora_sample(ctypes.byref(args), R, _stream(stream))
    if status:
        _check(status, "lora_sample")


# ------------------------------------------------------------------------------------------
# reading a metadata buffer copied back to the host
# ------------------------------------------------------------------------------------------
def unpack_segments(meta: np.ndarray, T: int, num_slots: int, tile_m: int) -> Dict[str, np.ndarray]:
    """Split the int32 words of a metadata buffer into its named arrays (see lora_b200.h)."""
    meta = np.asarray(meta, dtype=np.int32)
    cap_seg = min(T, num_slots)
    cap_tile = cap_seg + T // tile_m
    out: Dict[str, np.ndarray] = {"header_full": meta[:META_HEADER_WORDS].copy()}
    out["header"] = meta[:5].copy()
    o = META_HEADER_WORDS
    for name, n in [("perm", T), ("seg_slot", cap_seg), ("seg_start", cap_seg + 1),
                    ("seg_rank", cap_seg), ("seg_flags", cap_seg), ("tile_seg", cap_tile),
                    ("tile_row0", cap_tile), ("tile_rows", cap_tile), ("tile_flags", cap_tile)]:
        out[name] = meta[o:o + n].copy()
        o += n
    o = (o + 3) & ~3
    out["tile_desc"] = meta[o:o + 4 * cap_tile].reshape(cap_tile, 4).copy()   # library-private
    return out


def kv_table_views(tables, R: int, T: int):
    """The public arrays inside a table buffer (a flat int32 tensor or array), as views of it."""
    o = META_HEADER_WORDS
    out = {"header": tables[:o]}
    for name, n in [("start", R + 1), ("kv_len", R), ("position", T), ("slot", T)]:
        out[name] = tables[o:o + n]
        o += n
    return out
