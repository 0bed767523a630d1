"""ctypes binding of ``libscar.so``: argument marshalling only.

The module-level ``scar_*`` functions mirror ``include/scar.h`` one to one and
take raw device addresses (``int``) or torch CUDA tensors (their ``data_ptr()``
is used).  :class:`ScarCheckpoint` is a small convenience wrapper that owns one
context.  Nothing here computes anything: if the library cannot be loaded the
import of a ``scar_*`` call raises, there is no fallback.
"""

from __future__ import annotations

import ctypes as C
import os
import re
from typing import Optional

import numpy as np

SCAR_F32, SCAR_I32, SCAR_BF16, SCAR_F16 = 0, 1, 2, 3
SCAR_NORM_DEFAULT, SCAR_NORM_L1 = 0, 1
SCAR_MEAN, SCAR_SUM = 0, 1
SCAR_GNORM_L2, SCAR_GNORM_L1, SCAR_GNORM_MAX = 0, 1, 2
SCAR_ACT_IDENTITY, SCAR_ACT_RELU, SCAR_ACT_GELU, SCAR_ACT_SILU = 0, 1, 2, 3
SCAR_RESNORM_RMS, SCAR_RESNORM_LAYER = 0, 1
SCAR_OK = 0

_PKG = os.path.dirname(os.path.abspath(__file__))
_HEADER = os.path.join(os.path.dirname(_PKG), "include", "scar.h")
_lib = None


class ScarError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {scar_strerror(code)} ({code})")
        self.code = code


class scar_layout(C.Structure):
    _fields_ = [("n_elems", C.c_uint64), ("row_elems", C.c_uint64), ("block_elems", C.c_uint32),
                ("n_shards", C.c_uint32), ("block_offsets", C.POINTER(C.c_uint64)), ("n_blocks", C.c_uint64)]


class scar_save_info(C.Structure):
    _fields_ = [("k", C.c_uint64), ("payload_elems", C.c_uint64), ("nonfinite_blocks", C.c_uint64)]


class scar_norm_info(C.Structure):
    _fields_ = [("l2", C.c_double), ("l1", C.c_uint64), ("lost_blocks", C.c_uint64), ("lost_elems", C.c_uint64)]


class scar_drain_view(C.Structure):
    _fields_ = [("info", scar_save_info), ("h_sel", C.c_void_p), ("h_poff", C.c_void_p), ("h_payload", C.c_void_p)]


class scar_xent_config(C.Structure):
    _fields_ = [("max_tokens", C.c_uint64), ("n_classes", C.c_uint64), ("dim", C.c_uint64),
                ("ignore_label", C.c_int64), ("workspace_bytes", C.c_uint64), ("dtype", C.c_int),
                ("reduction", C.c_int), ("loss_only", C.c_int)]


class scar_xent_info(C.Structure):
    _fields_ = [("loss", C.c_float), ("rows", C.c_uint64), ("ignored", C.c_uint64), ("bad", C.c_uint64)]


class scar_tensor(C.Structure):
    _fields_ = [("d_data", C.c_void_p), ("d_out", C.c_void_p), ("n_elems", C.c_uint64), ("dtype", C.c_int)]


class scar_gnorm_info(C.Structure):
    _fields_ = [("norm", C.c_double), ("coef", C.c_double), ("nonfinite", C.c_uint64)]


class scar_dropout(C.Structure):
    _fields_ = [("p", C.c_double), ("seed", C.c_uint64), ("offset", C.c_uint64), ("d_offset", C.c_void_p)]


class scar_linear_config(C.Structure):
    _fields_ = [("max_rows", C.c_uint64), ("in_features", C.c_uint64), ("out_features", C.c_uint64), ("dtype", C.c_int),
                ("activation", C.c_int), ("forward_only", C.c_int)]


class scar_resnorm_config(C.Structure):
    _fields_ = [("max_rows", C.c_uint64), ("dim", C.c_uint64), ("eps", C.c_double), ("dtype", C.c_int), ("kind", C.c_int),
                ("forward_only", C.c_int)]


class scar_resnorm_block(C.Structure):
    _fields_ = [("post", C.c_int), ("pre", C.c_int), ("scale", C.c_float), ("d_gate", C.c_void_p), ("gate_pitch", C.c_uint64),
                ("rows_per_gate", C.c_uint64), ("d_w_post", C.c_void_p), ("d_b_post", C.c_void_p), ("d_w_pre", C.c_void_p),
                ("d_b_pre", C.c_void_p)]


def lib_path() -> str:
    return os.path.join(_PKG, "libscar.so")


def exported_symbols() -> list:
    """Names of the functions ``include/scar.h`` declares."""
    with open(_HEADER) as f:
        text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    return sorted(set(re.findall(r"\b(scar_[a-z_0-9]+)\s*\(", text)))


_vp, _u64, _int, _dbl = C.c_void_p, C.c_uint64, C.c_int, C.c_double
_SIGS = {
    "scar_ckpt_init": (_int, [C.POINTER(_vp), _vp, _int, C.POINTER(scar_layout), _vp]),
    "scar_ckpt_init_guarded": (_int, [C.POINTER(_vp), _vp, _int, C.POINTER(scar_layout), _vp]),
    "scar_ckpt_debug_check_guards": (_int, [_vp, C.POINTER(_u64)]),
    "scar_static_debug_check_guard": (_int, [C.POINTER(_u64)]),
    "scar_ckpt_set_norm": (_int, [_vp, _int, _vp]),
    "scar_ckpt_block_scores": (_int, [_vp]),
    "scar_ckpt_priority_save": (_int, [_vp, _dbl, C.POINTER(scar_save_info)]),
    "scar_k_from_r": (_int, [_dbl, _u64, C.POINTER(_u64)]),
    "scar_ckpt_priority_save_k": (_int, [_vp, _u64, C.POINTER(scar_save_info)]),
    "scar_ckpt_priority_save_sharded": (_int, [_vp, _vp, _u64, _u64, _u64, C.POINTER(scar_save_info)]),
    "scar_ckpt_save_round": (_int, [_vp, _u64, C.POINTER(scar_save_info)]),
    "scar_ckpt_save_random": (_int, [_vp, _u64, _vp, C.POINTER(scar_save_info)]),
    "scar_ckpt_round_cursor": (_int, [_vp, C.POINTER(_u64), C.POINTER(_u64)]),
    "scar_recover_partial": (_int, [_vp, _vp, C.POINTER(scar_norm_info)]),
    "scar_recover_partial_blocks": (_int, [_vp, _vp, C.POINTER(scar_norm_info)]),
    "scar_perturbation_norm": (_int, [_vp, _vp, C.POINTER(scar_norm_info)]),
    "scar_perturbation_norm_blocks": (_int, [_vp, _vp, C.POINTER(scar_norm_info)]),
    "scar_perturbation_norm_static": (_int, [_vp, _vp, _int, C.POINTER(scar_layout), _vp, _vp, _vp]),
    "scar_ckpt_priority_save_host": (_int, [_vp, _vp, _dbl, _vp, _vp, _vp, C.POINTER(scar_save_info)]),
    "scar_recover_partial_host": (_int, [_vp, _vp, _vp, C.POINTER(scar_norm_info)]),
    "scar_ckpt_drain_init": (_int, [_vp, _u64, _u64]),
    "scar_ckpt_drain_enqueue": (_int, [_vp, C.POINTER(_u64)]),
    "scar_ckpt_drain_done": (_int, [_vp, _u64]),
    "scar_ckpt_drain_wait": (_int, [_vp, _u64, C.POINTER(scar_drain_view)]),
    "scar_ckpt_drain_release": (_int, [_vp, _u64]),
    "scar_ckpt_store_full": (_int, [_vp, _int]),
    "scar_ckpt_store_drained": (_int, [_vp, _u64, _int]),
    "scar_ckpt_load_stored": (_int, [_vp, _int]),
    "scar_ckpt_load": (_int, [_vp, _vp]),
    "scar_ckpt_last_info": (_int, [_vp, C.POINTER(scar_save_info), C.POINTER(scar_norm_info)]),
    "scar_ckpt_view": (_int, [_vp] + [C.POINTER(_vp)] * 5),
    "scar_ckpt_n_blocks": (_u64, [_vp]),
    "scar_ckpt_launch_count": (_u64, [_vp]),
    "scar_ckpt_profile": (_int, [_vp, _int]),
    "scar_ckpt_profile_read": (_int, [_vp, C.POINTER(C.c_float)]),
    "scar_baseline_iterations": (_dbl, [_dbl, _dbl, _dbl]),
    "scar_discounted_perturbation": (_dbl, [_vp, _vp, _u64, _dbl]),
    "scar_iteration_cost_bound": (_dbl, [_dbl, _dbl, _dbl]),
    "scar_irreducible_error": (_dbl, [_dbl, _dbl]),
    "scar_ckpt_selftest_arm_timeout": (_int, [_vp]),
    "scar_ckpt_debug_select_stamps": (_int, [_vp, C.POINTER(C.c_int64)]),
    "scar_xent_init": (_int, [C.POINTER(_vp), C.POINTER(scar_xent_config), _vp]),
    "scar_xent_loss": (_int, [_vp, _vp, _u64, _vp, _u64, _vp, _u64, _vp, _vp]),
    "scar_xent_loss_grad": (_int, [_vp, _vp, _u64, _vp, _u64, _vp, _u64, C.c_float, _vp, _vp, _vp, _u64, _vp, _u64]),
    "scar_xent_status": (_int, [_vp, C.POINTER(scar_xent_info)]),
    "scar_xent_selftest_arm_timeout": (_int, [_vp]),
    "scar_xent_workspace_bytes": (_u64, [_vp]),
    "scar_xent_launch_count": (_u64, [_vp]),
    "scar_xent_destroy": (_int, [_vp]),
    "scar_gnorm_init": (_int, [C.POINTER(_vp), C.POINTER(scar_tensor), _u64, _int, _vp]),
    "scar_gnorm_bind": (_int, [_vp, C.POINTER(scar_tensor), _u64]),
    "scar_gnorm_norm": (_int, [_vp, _vp]),
    "scar_gnorm_clip": (_int, [_vp, C.c_float, _vp]),
    "scar_gnorm_status": (_int, [_vp, C.POINTER(scar_gnorm_info)]),
    "scar_gnorm_finished_alone": (_int, [_vp, C.POINTER(_u64)]),
    "scar_gnorm_selftest_arm_timeout": (_int, [_vp]),
    "scar_gnorm_launch_count": (_u64, [_vp]),
    "scar_gnorm_destroy": (_int, [_vp]),
    "scar_dropout_apply": (_int, [C.POINTER(scar_dropout), _int, _vp, _u64, _vp, _u64, _vp, _u64, _u64, _u64, _vp]),
    "scar_linear_init": (_int, [C.POINTER(_vp), C.POINTER(scar_linear_config), _vp]),
    "scar_linear_forward": (_int, [_vp, _vp, _u64, _vp, _u64, _vp, _vp, _u64, C.POINTER(scar_dropout), _u64, _vp, _u64, _vp]),
    "scar_linear_slope_bytes": (_u64, [_vp, _u64]),
    "scar_linear_backward": (_int, [_vp, _vp, _u64, _vp, _u64, _vp, _u64, _vp, C.POINTER(scar_dropout), _u64, _vp, _u64, _vp, _u64, _vp]),
    "scar_linear_status": (_int, [_vp]),
    "scar_linear_selftest_arm_timeout": (_int, [_vp]),
    "scar_linear_workspace_bytes": (_u64, [_vp]),
    "scar_linear_launch_count": (_u64, [_vp]),
    "scar_linear_destroy": (_int, [_vp]),
    "scar_resnorm_init": (_int, [C.POINTER(_vp), C.POINTER(scar_resnorm_config), _vp]),
    "scar_resnorm_forward": (_int, [_vp, C.POINTER(scar_resnorm_block), _vp, _u64, _vp, _u64, _u64, _vp, _u64, _vp, _u64]),
    "scar_resnorm_backward": (_int, [_vp, C.POINTER(scar_resnorm_block), _vp, _u64, _vp, _u64, _vp, _u64, _vp, _u64, _u64, _vp, _u64, _vp, _u64, _vp,
                                     _u64, _vp, _vp, _vp, _vp]),
    "scar_resnorm_status": (_int, [_vp]),
    "scar_resnorm_selftest_arm_timeout": (_int, [_vp]),
    "scar_resnorm_launch_count": (_u64, [_vp]),
    "scar_resnorm_destroy": (_int, [_vp]),
    "scar_ckpt_destroy": (_int, [_vp]),
    "scar_strerror": (C.c_char_p, [_int]),
}


def load_library():
    """Loads ``libscar.so`` from the package directory; raises if it is not there."""
    global _lib
    if _lib is None:
        path = lib_path()
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'` "
                               "(there is no CPU fallback)")
        lib = C.CDLL(path)
        for name, (res, args) in _SIGS.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


def _addr(a) -> Optional[int]:
    """Device or host address of ``a``: int, None, torch tensor or numpy array."""
    if a is None:
        return None
    if isinstance(a, int):
        return a
    if isinstance(a, np.ndarray):
        assert a.flags.c_contiguous
        return a.ctypes.data
    if hasattr(a, "data_ptr"):
        assert a.is_contiguous()
        return a.data_ptr()
    raise TypeError(type(a))


def _check(code: int, what: str):
    if code != SCAR_OK:
        raise ScarError(code, what)


def scar_strerror(code: int) -> str:
    return load_library().scar_strerror(code).decode()


def make_layout(n_elems: int, row_elems: int = 0, block_elems: int = 0, n_shards: int = 1,
                block_offsets: Optional[np.ndarray] = None):
    """Builds a ``scar_layout``; keeps the offsets array alive on the returned object."""
    L = scar_layout()
    L.n_elems, L.row_elems, L.block_elems, L.n_shards = n_elems, row_elems, block_elems, n_shards
    if block_offsets is not None:
        off = np.ascontiguousarray(block_offsets, dtype=np.uint64)
        L.block_offsets = off.ctypes.data_as(C.POINTER(C.c_uint64))
        L.n_blocks = off.size - 1
        L._keepalive = off
    return L


def scar_ckpt_init(d_x, dtype: int, layout: scar_layout, cuda_stream: int = 0, guarded: bool = False) -> int:
    ctx = _vp()
    name = "scar_ckpt_init_guarded" if guarded else "scar_ckpt_init"
    _check(getattr(load_library(), name)(C.byref(ctx), _addr(d_x), dtype, C.byref(layout), cuda_stream or None), name)
    return ctx.value


def scar_ckpt_init_guarded(d_x, dtype: int, layout: scar_layout, cuda_stream: int = 0) -> int:
    """``scar_ckpt_init`` for a debug context whose device buffers sit between guard bands."""
    return scar_ckpt_init(d_x, dtype, layout, cuda_stream, guarded=True)


def scar_ckpt_debug_check_guards(ctx: int) -> int:
    """Band bytes of a guarded context that no longer hold the pattern (0 = nothing wrote outside a buffer)."""
    bad = _u64(0)
    _check(load_library().scar_ckpt_debug_check_guards(ctx, C.byref(bad)), "scar_ckpt_debug_check_guards")
    return int(bad.value)


def scar_static_debug_check_guard() -> int:
    bad = _u64(0)
    _check(load_library().scar_static_debug_check_guard(C.byref(bad)), "scar_static_debug_check_guard")
    return int(bad.value)


def scar_ckpt_set_norm(ctx: int, norm: int, h_block_weights: Optional[np.ndarray] = None) -> None:
    w = None if h_block_weights is None else np.ascontiguousarray(h_block_weights, dtype=np.float32)
    _check(load_library().scar_ckpt_set_norm(ctx, norm, _addr(w)), "scar_ckpt_set_norm")


def scar_ckpt_block_scores(ctx: int) -> None:
    _check(load_library().scar_ckpt_block_scores(ctx), "scar_ckpt_block_scores")


def _save_out(sync: bool):
    return scar_save_info() if sync else None


def scar_ckpt_priority_save(ctx: int, r: float, sync: bool = True) -> Optional[scar_save_info]:
    out = _save_out(sync)
    _check(load_library().scar_ckpt_priority_save(ctx, r, C.byref(out) if sync else None), "scar_ckpt_priority_save")
    return out


def scar_k_from_r(r: float, n_blocks: int) -> int:
    """The library's rule for the number of blocks a fraction r stands for."""
    k = _u64(0)
    _check(load_library().scar_k_from_r(r, n_blocks, C.byref(k)), "scar_k_from_r")
    return int(k.value)


def scar_ckpt_priority_save_k(ctx: int, k: int, sync: bool = True) -> Optional[scar_save_info]:
    out = _save_out(sync)
    _check(load_library().scar_ckpt_priority_save_k(ctx, k, C.byref(out) if sync else None),
           "scar_ckpt_priority_save_k")
    return out


def scar_ckpt_priority_save_sharded(ctx: int, d_global_scores, n_global_blocks: int, first_block: int,
                                    k_global: int) -> scar_save_info:
    out = scar_save_info()
    _check(load_library().scar_ckpt_priority_save_sharded(ctx, _addr(d_global_scores), n_global_blocks, first_block,
                                                          k_global, C.byref(out)), "scar_ckpt_priority_save_sharded")
    return out


def scar_ckpt_save_round(ctx: int, k: int, sync: bool = True) -> Optional[scar_save_info]:
    out = _save_out(sync)
    _check(load_library().scar_ckpt_save_round(ctx, k, C.byref(out) if sync else None), "scar_ckpt_save_round")
    return out


def scar_ckpt_save_random(ctx: int, k: int, d_priorities, sync: bool = True) -> Optional[scar_save_info]:
    out = _save_out(sync)
    _check(load_library().scar_ckpt_save_random(ctx, k, _addr(d_priorities), C.byref(out) if sync else None),
           "scar_ckpt_save_random")
    return out


def scar_ckpt_round_cursor(ctx: int, set_to: Optional[int] = None) -> int:
    """Returns the round-robin cursor, after setting it when ``set_to`` is given."""
    got = _u64(0)
    new = _u64(set_to) if set_to is not None else None
    _check(load_library().scar_ckpt_round_cursor(ctx, C.byref(new) if new is not None else None, C.byref(got)),
           "scar_ckpt_round_cursor")
    return int(got.value)


def _norm_call(fn_name: str, ctx: int, mask, sync: bool) -> Optional[scar_norm_info]:
    out = scar_norm_info() if sync else None
    _check(getattr(load_library(), fn_name)(ctx, _addr(mask), C.byref(out) if sync else None), fn_name)
    return out


def scar_recover_partial(ctx: int, h_lost_shards: np.ndarray, sync: bool = True):
    return _norm_call("scar_recover_partial", ctx, np.ascontiguousarray(h_lost_shards, dtype=np.uint8), sync)


def scar_recover_partial_blocks(ctx: int, d_lost_blocks, sync: bool = True):
    return _norm_call("scar_recover_partial_blocks", ctx, d_lost_blocks, sync)


def scar_perturbation_norm(ctx: int, h_lost_shards: Optional[np.ndarray] = None, sync: bool = True):
    m = None if h_lost_shards is None else np.ascontiguousarray(h_lost_shards, dtype=np.uint8)
    return _norm_call("scar_perturbation_norm", ctx, m, sync)


def scar_perturbation_norm_blocks(ctx: int, d_lost_blocks=None, sync: bool = True):
    return _norm_call("scar_perturbation_norm_blocks", ctx, d_lost_blocks, sync)


def scar_perturbation_norm_static(d_x, d_z, dtype: int, layout: scar_layout, d_lost_blocks, d_out,
                                  cuda_stream: int = 0) -> None:
    """Allocation-free perturbation norm: enqueues on ``cuda_stream`` and writes a ``scar_norm_info`` to the
    caller's device buffer ``d_out`` (32 bytes).  See ``include/scar.h`` for who needs it and its limits."""
    _check(load_library().scar_perturbation_norm_static(_addr(d_x), _addr(d_z), dtype, C.byref(layout),
                                                        _addr(d_lost_blocks), _addr(d_out), cuda_stream or None),
           "scar_perturbation_norm_static")


def scar_ckpt_priority_save_host(ctx: int, h_x, r: float, h_payload, h_sel, h_poff) -> scar_save_info:
    out = scar_save_info()
    _check(load_library().scar_ckpt_priority_save_host(ctx, _addr(h_x), r, _addr(h_payload), _addr(h_sel),
                                                       _addr(h_poff), C.byref(out)), "scar_ckpt_priority_save_host")
    return out


def scar_recover_partial_host(ctx: int, h_x, h_lost_shards: np.ndarray) -> scar_norm_info:
    out = scar_norm_info()
    m = np.ascontiguousarray(h_lost_shards, dtype=np.uint8)
    _check(load_library().scar_recover_partial_host(ctx, _addr(h_x), _addr(m), C.byref(out)),
           "scar_recover_partial_host")
    return out


def scar_ckpt_drain_init(ctx: int, max_k: int, max_payload_elems: int) -> None:
    _check(load_library().scar_ckpt_drain_init(ctx, max_k, max_payload_elems), "scar_ckpt_drain_init")


def scar_ckpt_drain_enqueue(ctx: int) -> int:
    t = _u64(0)
    _check(load_library().scar_ckpt_drain_enqueue(ctx, C.byref(t)), "scar_ckpt_drain_enqueue")
    return int(t.value)


def scar_ckpt_drain_done(ctx: int, ticket: int) -> bool:
    rc = load_library().scar_ckpt_drain_done(ctx, ticket)
    if rc < 0:
        raise ScarError(rc, "scar_ckpt_drain_done")
    return bool(rc)


def scar_ckpt_drain_wait(ctx: int, ticket: int, elem_dtype=np.float32) -> dict:
    """Waits for the drain of ``ticket``; returns numpy views (no copy) of the pinned host mirror, valid until
    ``scar_ckpt_drain_release``."""
    v = scar_drain_view()
    _check(load_library().scar_ckpt_drain_wait(ctx, ticket, C.byref(v)), "scar_ckpt_drain_wait")
    k, n = int(v.info.k), int(v.info.payload_elems)

    def view(addr, count, dt):
        if count == 0:
            return np.empty(0, dtype=dt)
        buf = (C.c_char * (count * np.dtype(dt).itemsize)).from_address(addr)
        return np.frombuffer(buf, dtype=dt, count=count)

    return {"info": v.info, "sel": view(v.h_sel, k, np.uint32), "poff": view(v.h_poff, k + 1, np.uint64),
            "payload": view(v.h_payload, n, elem_dtype)}


def scar_ckpt_drain_release(ctx: int, ticket: int) -> None:
    _check(load_library().scar_ckpt_drain_release(ctx, ticket), "scar_ckpt_drain_release")


def scar_ckpt_store_full(ctx: int, fd: int) -> None:
    _check(load_library().scar_ckpt_store_full(ctx, fd), "scar_ckpt_store_full")


def scar_ckpt_store_drained(ctx: int, ticket: int, fd: int) -> None:
    _check(load_library().scar_ckpt_store_drained(ctx, ticket, fd), "scar_ckpt_store_drained")


def scar_ckpt_load_stored(ctx: int, fd: int) -> None:
    _check(load_library().scar_ckpt_load_stored(ctx, fd), "scar_ckpt_load_stored")


def scar_ckpt_load(ctx: int, d_z_src) -> None:
    _check(load_library().scar_ckpt_load(ctx, _addr(d_z_src)), "scar_ckpt_load")


def scar_ckpt_last_info(ctx: int, want_save: bool = True, want_norm: bool = True):
    s = scar_save_info() if want_save else None
    n = scar_norm_info() if want_norm else None
    _check(load_library().scar_ckpt_last_info(ctx, C.byref(s) if s else None, C.byref(n) if n else None),
           "scar_ckpt_last_info")
    return s, n


def scar_ckpt_view(ctx: int) -> dict:
    """Device addresses of z, scores, sel, poff, payload."""
    p = [_vp() for _ in range(5)]
    _check(load_library().scar_ckpt_view(ctx, *[C.byref(q) for q in p]), "scar_ckpt_view")
    return dict(zip(("z", "scores", "sel", "poff", "payload"), (q.value for q in p)))


def scar_ckpt_n_blocks(ctx: int) -> int:
    return int(load_library().scar_ckpt_n_blocks(ctx))


def scar_ckpt_launch_count(ctx: int) -> int:
    return int(load_library().scar_ckpt_launch_count(ctx))


def scar_ckpt_profile(ctx: int, enable: bool) -> None:
    _check(load_library().scar_ckpt_profile(ctx, int(enable)), "scar_ckpt_profile")


def scar_ckpt_profile_read(ctx: int) -> list:
    ms = (C.c_float * 5)()
    _check(load_library().scar_ckpt_profile_read(ctx, ms), "scar_ckpt_profile_read")
    return list(ms)


def scar_baseline_iterations(dist0: float, eps: float, c: float) -> float:
    return float(load_library().scar_baseline_iterations(dist0, eps, c))


def scar_discounted_perturbation(norms, iters, c: float) -> float:
    nrm = np.ascontiguousarray(norms, dtype=np.float64)
    its = np.ascontiguousarray(iters, dtype=np.uint64)
    assert nrm.shape == its.shape and nrm.ndim == 1
    return float(load_library().scar_discounted_perturbation(_addr(nrm) if nrm.size else None,
                                                             _addr(its) if its.size else None, nrm.size, c))


def scar_iteration_cost_bound(delta_T: float, dist0: float, c: float) -> float:
    return float(load_library().scar_iteration_cost_bound(delta_T, dist0, c))


def scar_irreducible_error(delta_max: float, c: float) -> float:
    return float(load_library().scar_irreducible_error(delta_max, c))


def scar_ckpt_selftest_arm_timeout(ctx: int) -> None:
    _check(load_library().scar_ckpt_selftest_arm_timeout(ctx), "scar_ckpt_selftest_arm_timeout")


def scar_ckpt_debug_select_stamps(ctx: int) -> list:
    """Cycle stamps of the last selection kernel (diagnostic builds of the library only)."""
    st = (C.c_int64 * 32)()
    _check(load_library().scar_ckpt_debug_select_stamps(ctx, st), "scar_ckpt_debug_select_stamps")
    return list(st)


def scar_ckpt_destroy(ctx: int) -> None:
    _check(load_library().scar_ckpt_destroy(ctx), "scar_ckpt_destroy")


# ---- the training step ----------------------------------------------------------------------


def scar_xent_init(config: scar_xent_config, cuda_stream: int = 0) -> int:
    op = _vp()
    _check(load_library().scar_xent_init(C.byref(op), C.byref(config), cuda_stream or None), "scar_xent_init")
    return op.value


def scar_xent_loss(op: int, d_h, h_pitch: int, d_w, w_pitch: int, d_labels, n_tokens: int, d_row_loss, d_loss) -> None:
    _check(load_library().scar_xent_loss(op, d_h, h_pitch, d_w, w_pitch, d_labels, n_tokens, d_row_loss, d_loss),
           "scar_xent_loss")


def scar_xent_loss_grad(op: int, d_h, h_pitch: int, d_w, w_pitch: int, d_labels, n_tokens: int, grad_scale: float,
                        d_row_loss, d_loss, d_dh, dh_pitch: int, d_dw, dw_pitch: int) -> None:
    """Raw device addresses throughout (rows may be further apart than ``dim``: a tensor's own strides decide)."""
    _check(load_library().scar_xent_loss_grad(op, d_h, h_pitch, d_w, w_pitch, d_labels, n_tokens, grad_scale, d_row_loss,
                                              d_loss, d_dh, dh_pitch, d_dw, dw_pitch), "scar_xent_loss_grad")


def scar_xent_status(op: int) -> scar_xent_info:
    out = scar_xent_info()
    _check(load_library().scar_xent_status(op, C.byref(out)), "scar_xent_status")
    return out


def scar_xent_selftest_arm_timeout(op: int) -> None:
    _check(load_library().scar_xent_selftest_arm_timeout(op), "scar_xent_selftest_arm_timeout")


def scar_xent_workspace_bytes(op: int) -> int:
    return int(load_library().scar_xent_workspace_bytes(op))


def scar_xent_launch_count(op: int) -> int:
    return int(load_library().scar_xent_launch_count(op))


def scar_xent_destroy(op: int) -> None:
    _check(load_library().scar_xent_destroy(op), "scar_xent_destroy")


def scar_gnorm_init(tensors, kind: int = SCAR_GNORM_L2, cuda_stream: int = 0) -> int:
    """``tensors``: a ctypes array of :class:`scar_tensor`."""
    op = _vp()
    _check(load_library().scar_gnorm_init(C.byref(op), tensors, len(tensors), kind, cuda_stream or None),
           "scar_gnorm_init")
    return op.value


def scar_gnorm_bind(op: int, tensors) -> None:
    _check(load_library().scar_gnorm_bind(op, tensors, len(tensors)), "scar_gnorm_bind")


def scar_gnorm_norm(op: int, d_norm) -> None:
    _check(load_library().scar_gnorm_norm(op, d_norm), "scar_gnorm_norm")


def scar_gnorm_clip(op: int, max_norm: float, d_norm) -> None:
    _check(load_library().scar_gnorm_clip(op, max_norm, d_norm), "scar_gnorm_clip")


def scar_gnorm_status(op: int) -> scar_gnorm_info:
    out = scar_gnorm_info()
    _check(load_library().scar_gnorm_status(op, C.byref(out)), "scar_gnorm_status")
    return out


def scar_gnorm_finished_alone(op: int) -> int:
    calls = _u64()
    _check(load_library().scar_gnorm_finished_alone(op, C.byref(calls)), "scar_gnorm_finished_alone")
    return int(calls.value)


def scar_gnorm_selftest_arm_timeout(op: int) -> None:
    _check(load_library().scar_gnorm_selftest_arm_timeout(op), "scar_gnorm_selftest_arm_timeout")


def scar_gnorm_launch_count(op: int) -> int:
    return int(load_library().scar_gnorm_launch_count(op))


def scar_gnorm_destroy(op: int) -> None:
    _check(load_library().scar_gnorm_destroy(op), "scar_gnorm_destroy")


def scar_dropout_apply(rule: scar_dropout, dtype: int, d_x, x_pitch: int, d_residual, residual_pitch: int, d_y, y_pitch: int, rows: int, cols: int,
                       cuda_stream: int = 0) -> None:
    _check(load_library().scar_dropout_apply(C.byref(rule), dtype, d_x, x_pitch, d_residual, residual_pitch, d_y, y_pitch, rows, cols,
                                             cuda_stream or None), "scar_dropout_apply")


def scar_linear_init(config: scar_linear_config, cuda_stream: int = 0) -> int:
    op = _vp()
    _check(load_library().scar_linear_init(C.byref(op), C.byref(config), cuda_stream or None), "scar_linear_init")
    return op.value


def scar_linear_forward(op: int, d_x, x_pitch: int, d_w, w_pitch: int, d_bias, d_residual, residual_pitch: int, dropout: Optional[scar_dropout],
                        n_rows: int, d_y, y_pitch: int, d_slope=None) -> None:
    _check(load_library().scar_linear_forward(op, d_x, x_pitch, d_w, w_pitch, d_bias, d_residual, residual_pitch, dropout, n_rows, d_y, y_pitch,
                                              d_slope), "scar_linear_forward")


def scar_linear_slope_bytes(op: int, n_rows: int) -> int:
    return int(load_library().scar_linear_slope_bytes(op, n_rows))


def scar_linear_backward(op: int, d_dy, dy_pitch: int, d_x, x_pitch: int, d_w, w_pitch: int, d_slope, dropout: Optional[scar_dropout], n_rows: int,
                         d_dx, dx_pitch: int, d_dw, dw_pitch: int, d_dbias) -> None:
    _check(load_library().scar_linear_backward(op, d_dy, dy_pitch, d_x, x_pitch, d_w, w_pitch, d_slope, dropout, n_rows, d_dx, dx_pitch, d_dw,
                                               dw_pitch, d_dbias), "scar_linear_backward")


def scar_linear_status(op: int) -> None:
    _check(load_library().scar_linear_status(op), "scar_linear_status")


def scar_linear_selftest_arm_timeout(op: int) -> None:
    _check(load_library().scar_linear_selftest_arm_timeout(op), "scar_linear_selftest_arm_timeout")


def scar_linear_workspace_bytes(op: int) -> int:
    return int(load_library().scar_linear_workspace_bytes(op))


def scar_linear_launch_count(op: int) -> int:
    return int(load_library().scar_linear_launch_count(op))


def scar_linear_destroy(op: int) -> None:
    _check(load_library().scar_linear_destroy(op), "scar_linear_destroy")


def scar_resnorm_init(config: scar_resnorm_config, cuda_stream: int = 0) -> int:
    op = _vp()
    _check(load_library().scar_resnorm_init(C.byref(op), C.byref(config), cuda_stream or None), "scar_resnorm_init")
    return op.value


def scar_resnorm_forward(op: int, block: scar_resnorm_block, d_x, x_pitch: int, d_f, f_pitch: int, n_rows: int, d_y, y_pitch: int, d_n,
                         n_pitch: int) -> None:
    _check(load_library().scar_resnorm_forward(op, C.byref(block), d_x, x_pitch, d_f, f_pitch, n_rows, d_y, y_pitch, d_n, n_pitch),
           "scar_resnorm_forward")


def scar_resnorm_backward(op: int, block: scar_resnorm_block, d_dy, dy_pitch: int, d_dn, dn_pitch: int, d_y, y_pitch: int, d_f, f_pitch: int,
                          n_rows: int, d_dx, dx_pitch: int, d_df, df_pitch: int, d_dgate, dgate_pitch: int, d_dw_post, d_db_post, d_dw_pre,
                          d_db_pre) -> None:
    _check(load_library().scar_resnorm_backward(op, C.byref(block), d_dy, dy_pitch, d_dn, dn_pitch, d_y, y_pitch, d_f, f_pitch, n_rows, d_dx, dx_pitch,
                                                d_df, df_pitch, d_dgate, dgate_pitch, d_dw_post, d_db_post, d_dw_pre, d_db_pre), "scar_resnorm_backward")


def scar_resnorm_status(op: int) -> None:
    _check(load_library().scar_resnorm_status(op), "scar_resnorm_status")


def scar_resnorm_selftest_arm_timeout(op: int) -> None:
    _check(load_library().scar_resnorm_selftest_arm_timeout(op), "scar_resnorm_selftest_arm_timeout")


def scar_resnorm_launch_count(op: int) -> int:
    return int(load_library().scar_resnorm_launch_count(op))


def scar_resnorm_destroy(op: int) -> None:
    _check(load_library().scar_resnorm_destroy(op), "scar_resnorm_destroy")


# ---------------------------------------------------------------------------------------------


class _DevView:
    """Lets torch wrap a raw device address without copying."""

    def __init__(self, addr: int, n: int, typestr: str):
        self.__cuda_array_interface__ = {"shape": (n,), "typestr": typestr, "data": (addr, False), "version": 3}


def device_array(addr: int, n: int, dtype):
    """A torch tensor aliasing ``n`` elements of ``dtype`` at device address ``addr`` (no copy)."""
    import torch

    np_dt = np.dtype(dtype)
    if n == 0:
        return torch.empty(0, dtype=getattr(torch, np_dt.name), device="cuda")
    return torch.as_tensor(_DevView(addr, n, np_dt.str), device="cuda")


class ScarCheckpoint:
    """One context over a torch CUDA tensor ``x`` (float32 or int32, flat, contiguous)."""

    def __init__(self, x, n_shards: int = 8, row_elems: int = 0, block_elems: int = 0,
                 block_offsets: Optional[np.ndarray] = None, stream=None, guarded: bool = False):
        import torch

        assert x.is_cuda and x.is_contiguous() and x.dim() == 1
        self.dtype = {torch.float32: SCAR_F32, torch.int32: SCAR_I32}[x.dtype]
        self.guarded = guarded
        self.x = x
        self.n_elems = x.numel()
        self._stream = stream if stream is not None else torch.cuda.current_stream(x.device)
        self._layout = make_layout(self.n_elems, row_elems, block_elems, n_shards, block_offsets)
        with torch.cuda.device(x.device):
            self.ctx = scar_ckpt_init(x, self.dtype, self._layout, self._stream.cuda_stream, guarded)
        self.n_blocks = scar_ckpt_n_blocks(self.ctx)

    # views -----------------------------------------------------------------
    def views(self, k: Optional[int] = None, payload_elems: Optional[int] = None) -> dict:
        v = scar_ckpt_view(self.ctx)
        elem = np.float32 if self.dtype == SCAR_F32 else np.int32
        score = np.float32 if self.dtype == SCAR_F32 else np.int64  # bit pattern of uint64 scores
        out = {"z": device_array(v["z"], self.n_elems, elem),
               "scores": device_array(v["scores"], self.n_blocks, score)}
        if k is not None:
            out["sel"] = device_array(v["sel"], k, np.int32)  # bit pattern of uint32 ids
            out["poff"] = device_array(v["poff"], k + 1, np.int64)
            if payload_elems is not None:
                out["payload"] = device_array(v["payload"], payload_elems, elem)
        return out

    # calls -------------------------------------------------------------------
    def set_norm(self, norm: int, block_weights: Optional[np.ndarray] = None):
        if block_weights is not None:
            assert len(block_weights) == self.n_blocks
        scar_ckpt_set_norm(self.ctx, norm, block_weights)

    def check_guards(self) -> int:
        return scar_ckpt_debug_check_guards(self.ctx)

    def block_scores(self):
        scar_ckpt_block_scores(self.ctx)

    def priority_save(self, r: float, sync: bool = True):
        return scar_ckpt_priority_save(self.ctx, r, sync)

    def priority_save_k(self, k: int, sync: bool = True):
        return scar_ckpt_priority_save_k(self.ctx, k, sync)

    def priority_save_sharded(self, d_global_scores, n_global_blocks: int, first_block: int, k_global: int):
        return scar_ckpt_priority_save_sharded(self.ctx, d_global_scores, n_global_blocks, first_block, k_global)

    def save_round(self, k: int, sync: bool = True):
        return scar_ckpt_save_round(self.ctx, k, sync)

    def save_random(self, k: int, d_priorities, sync: bool = True):
        return scar_ckpt_save_random(self.ctx, k, d_priorities, sync)

    def round_cursor(self, set_to: Optional[int] = None) -> int:
        return scar_ckpt_round_cursor(self.ctx, set_to)

    def recover_partial(self, lost_shards: np.ndarray, sync: bool = True):
        return scar_recover_partial(self.ctx, lost_shards, sync)

    def recover_partial_blocks(self, d_lost_blocks, sync: bool = True):
        return scar_recover_partial_blocks(self.ctx, d_lost_blocks, sync)

    def perturbation_norm(self, lost_shards: Optional[np.ndarray] = None, sync: bool = True):
        return scar_perturbation_norm(self.ctx, lost_shards, sync)

    def perturbation_norm_blocks(self, d_lost_blocks=None, sync: bool = True):
        return scar_perturbation_norm_blocks(self.ctx, d_lost_blocks, sync)

    def drain_init(self, max_k: int, max_payload_elems: int):
        scar_ckpt_drain_init(self.ctx, max_k, max_payload_elems)

    def drain_enqueue(self) -> int:
        return scar_ckpt_drain_enqueue(self.ctx)

    def drain_done(self, ticket: int) -> bool:
        return scar_ckpt_drain_done(self.ctx, ticket)

    def drain_wait(self, ticket: int) -> dict:
        return scar_ckpt_drain_wait(self.ctx, ticket, np.float32 if self.dtype == SCAR_F32 else np.int32)

    def drain_release(self, ticket: int):
        scar_ckpt_drain_release(self.ctx, ticket)

    def store_full(self, fd: int):
        scar_ckpt_store_full(self.ctx, fd)

    def store_drained(self, ticket: int, fd: int):
        scar_ckpt_store_drained(self.ctx, ticket, fd)

    def load_stored(self, fd: int):
        scar_ckpt_load_stored(self.ctx, fd)

    def load(self, d_z_src):
        scar_ckpt_load(self.ctx, d_z_src)

    def close(self):
        if getattr(self, "ctx", None):
            scar_ckpt_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class _OnStream:
    """Runs a handle's calls on its own stream and orders them with the stream the caller is working on: the handle's
    stream first waits for the caller's, and the caller's for the handle's afterwards.  Nothing happens where the two
    are the same."""

    def _bind_stream(self, stream, device):
        import torch

        device = torch.device(device)
        self._device = torch.device(device.type, torch.cuda.current_device() if device.index is None else device.index)
        self._stream = stream if stream is not None else torch.cuda.current_stream(self._device)
        self._torch, self._here = torch, torch._C._cuda_getCurrentRawStream  # the stream's address alone: no object per call

    def _enter(self, *tensors):
        if self._here(self._device.index) == self._stream.cuda_stream:
            return None
        here = self._torch.cuda.current_stream(self._device)
        self._stream.wait_stream(here)
        for t in tensors:
            if t is not None:
                t.record_stream(self._stream)
        return here

    def _leave(self, here):
        if here is not None:
            here.wait_stream(self._stream)


_OPERAND_TYPES = {}


def _operand_type(dtype) -> int:
    if not _OPERAND_TYPES:
        import torch

        _OPERAND_TYPES.update({torch.float32: SCAR_F32, torch.bfloat16: SCAR_BF16, torch.float16: SCAR_F16})
    if dtype not in _OPERAND_TYPES:
        raise TypeError(f"{dtype}: the training-step operators take float32, bfloat16 and float16")
    return _OPERAND_TYPES[dtype]


class LinearCrossEntropy(_OnStream):
    """Softmax cross entropy of ``h @ w.T`` against integer labels, with its gradients, a piece of the rows at a time.

    ``max_tokens`` rows at most per call, ``n_classes`` x ``dim`` weights, all operands of ``dtype`` (float32,
    bfloat16 or float16).  Rows whose label is ``ignore_label`` do not count; ``reduction`` is ``"mean"`` (over the
    rows that count) or ``"sum"``.  ``workspace_bytes`` bounds the block of logit gradients held at a time (0: 1 GiB;
    at least 256 rows, and all rows where that needs less memory than the float32 sums of ``dw`` over several pieces
    would).  ``loss_only`` handles hold no workspace for gradients."""

    def __init__(self, max_tokens: int, n_classes: int, dim: int, dtype, reduction: str = "mean",
                 ignore_label: int = -100, workspace_bytes: int = 0, loss_only: bool = False, stream=None,
                 device="cuda"):
        import torch

        cfg = scar_xent_config(max_tokens=max_tokens, n_classes=n_classes, dim=dim, ignore_label=ignore_label,
                               workspace_bytes=workspace_bytes, dtype=_operand_type(dtype),
                               reduction={"mean": SCAR_MEAN, "sum": SCAR_SUM}[reduction], loss_only=int(loss_only))
        self.max_tokens, self.n_classes, self.dim, self.dtype = max_tokens, n_classes, dim, dtype
        self._bind_stream(stream, device)
        with torch.cuda.device(self._device):
            self.op = scar_xent_init(cfg, self._stream.cuda_stream)

    def _matrix(self, name: str, m, rows: int):
        if m.dtype != self.dtype or m.device != self._device:
            raise TypeError(f"{name}: a tensor of {self.dtype} on {self._device} is wanted")
        if m.dim() != 2 or tuple(m.shape) != (rows, self.dim) or (self.dim > 1 and m.stride(1) != 1):
            raise ValueError(f"{name}: shape ({rows}, {self.dim}) with contiguous rows is wanted")
        return m.data_ptr(), (m.stride(0) if rows > 1 else max(m.stride(0), self.dim))

    def _call(self, grad: bool, h, w, labels, grad_scale, row_loss, dh, dw):
        torch = self._torch
        n = labels.numel()
        dev = self._device
        if labels.dtype != torch.int64 or labels.device != dev or not labels.is_contiguous():
            raise TypeError(f"labels: a contiguous tensor of int64 on {dev} is wanted")
        hp, wp = self._matrix("h", h, n), self._matrix("w", w, self.n_classes)
        if row_loss is None:
            row_loss = torch.empty(n, dtype=torch.float32, device=dev)
        elif row_loss.dtype != torch.float32 or row_loss.device != dev or row_loss.numel() != n or not row_loss.is_contiguous():
            raise ValueError(f"row_loss: one contiguous float32 per row on {dev} is wanted")
        loss = torch.empty((), dtype=torch.float32, device=dev)
        if grad:
            dh = torch.empty((n, self.dim), dtype=self.dtype, device=dev) if dh is None else dh
            dw = torch.empty((self.n_classes, self.dim), dtype=self.dtype, device=dev) if dw is None else dw
            dhp, dwp = self._matrix("dh", dh, n), self._matrix("dw", dw, self.n_classes)
        here = self._enter(h, w, labels, row_loss, loss, dh, dw)
        if grad:
            scar_xent_loss_grad(self.op, *hp, *wp, labels.data_ptr(), n, grad_scale, row_loss.data_ptr(), loss.data_ptr(),
                                *dhp, *dwp)
        else:
            scar_xent_loss(self.op, *hp, *wp, labels.data_ptr(), n, row_loss.data_ptr(), loss.data_ptr())
        self._leave(here)
        return (loss, row_loss, dh, dw) if grad else (loss, row_loss)

    def loss(self, h, w, labels, row_loss=None):
        """``(loss, row_loss)``: a float32 scalar and one float32 per row, on the device."""
        return self._call(False, h, w, labels, 0.0, row_loss, None, None)

    def loss_and_grad(self, h, w, labels, grad_scale: float = 1.0, row_loss=None, dh=None, dw=None):
        """``(loss, row_loss, dh, dw)``: the gradients are those of ``grad_scale * loss``, in the operands' type."""
        return self._call(True, h, w, labels, grad_scale, row_loss, dh, dw)

    def status(self) -> scar_xent_info:
        """Waits; rows that counted, rows ignored, labels out of range in the most recent call."""
        return scar_xent_status(self.op)

    def workspace_bytes(self) -> int:
        return scar_xent_workspace_bytes(self.op)

    def close(self):
        if getattr(self, "op", None):
            scar_xent_destroy(self.op)
            self.op = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class GradientNorm(_OnStream):
    """Global norm over a list of CUDA tensors (contiguous; float32, bfloat16, float16, mixed) and clipping by it.

    ``out``: tensors that receive the scaled values, or None to scale in place.  ``kind``: ``"l2"``, ``"l1"`` or
    ``"max"``.  The tensors are registered once; :meth:`bind` gives new ones of the same lengths and types."""

    def __init__(self, tensors, out=None, kind: str = "l2", stream=None):
        import torch

        tensors = list(tensors)
        self._bind_stream(stream, tensors[0].device if tensors else "cuda")
        out = self._outputs(tensors, out)
        table = self._table(tensors, out)
        with torch.cuda.device(self._device):
            self.op = scar_gnorm_init(table, {"l2": SCAR_GNORM_L2, "l1": SCAR_GNORM_L1, "max": SCAR_GNORM_MAX}[kind],
                                      self._stream.cuda_stream)
        self._tensors, self._out = tensors, out  # kept alive as long as they are registered

    @staticmethod
    def _outputs(tensors, out):
        return [None] * len(tensors) if out is None else list(out)

    def _table(self, tensors, out):
        if len(out) != len(tensors):
            raise ValueError("out: one tensor per input is wanted")
        table = (scar_tensor * len(tensors))()
        for e, t, o in zip(table, tensors, out):
            for x in (t, o):
                if x is not None and (x.device != self._device or not x.is_contiguous()):
                    raise ValueError(f"contiguous tensors on {self._device} are wanted")
            if o is not None and (o.dtype != t.dtype or o.numel() != t.numel()):
                raise ValueError("an output has its input's type and length")
            e.d_data, e.n_elems, e.dtype = t.data_ptr(), t.numel(), _operand_type(t.dtype)
            e.d_out = None if o is None else o.data_ptr()
        return table

    def bind(self, tensors, out=None):
        tensors = list(tensors)
        out = self._outputs(tensors, out)
        scar_gnorm_bind(self.op, self._table(tensors, out))
        self._tensors, self._out = tensors, out  # a refused list leaves the handle on the one before

    def _run(self, call):
        norm = self._torch.empty((), dtype=self._torch.float32, device=self._device)
        here = self._enter(norm)
        call(norm.data_ptr())
        self._leave(here)
        return norm

    def norm(self):
        """The norm, a float32 scalar on the device."""
        return self._run(lambda d: scar_gnorm_norm(self.op, d))

    def clip(self, max_norm: float):
        """Scales every tensor by ``min(1, max_norm / norm)``; returns the norm before scaling."""
        return self._run(lambda d: scar_gnorm_clip(self.op, max_norm, d))

    def status(self) -> scar_gnorm_info:
        """Waits; norm and factor of the most recent call in double, and whether the norm was finite."""
        return scar_gnorm_status(self.op)

    def close(self):
        if getattr(self, "op", None):
            scar_gnorm_destroy(self.op)
            self.op = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class DropoutMask:
    """One mask of a :class:`Dropout`: its rule, and the tensor its offset lies in (or None)."""

    def __init__(self, rule: scar_dropout, tensor=None):
        self.rule, self.tensor = rule, tensor

    def at(self, device):
        if self.tensor is not None and self.tensor.device != device:
            raise ValueError(f"offset: a tensor on {device} is wanted")
        return self.rule


class Dropout(_OnStream):
    """Dropout whose mask is computed from ``(seed, offset)`` and stored nowhere: ``forward`` and ``backward`` with one offset
    share it, and so does a :class:`LinearLayer` given ``mask(offset)``.  ``p`` is the share that is dropped (taken to the nearest
    multiple of 2^-16); what is kept is scaled by ``1 / (1 - p)``.  The last dimension of a tensor are its columns, all others its
    rows.  Offsets that differ give other masks: an int, or a tensor of one int64 on the device that is read when the call runs (a
    captured graph then takes the mask of its value at each replay)."""

    def __init__(self, p: float, seed: int = 0, stream=None, device="cuda"):
        if not 0.0 <= p <= 1.0:
            raise ValueError("p: a share between 0 and 1 is wanted")
        self.p, self.seed = float(p), seed
        self._bind_stream(stream, device)

    def _rule(self, offset):
        """The rule, and the tensor its offset lies in."""
        if isinstance(offset, int):
            return scar_dropout(self.p, self.seed & (2**64 - 1), offset & (2**64 - 1), None), None
        if offset.dtype != self._torch.int64 or offset.numel() != 1 or offset.device != self._device:
            raise TypeError(f"offset: an int or a tensor of one int64 on {self._device} is wanted")
        return scar_dropout(self.p, self.seed & (2**64 - 1), 0, offset.data_ptr()), offset

    def mask(self, offset=0) -> DropoutMask:
        return DropoutMask(*self._rule(offset))

    def _rows(self, name: str, m, like):
        """Address and pitch of m's rows."""
        if m.dtype != like.dtype or m.device != self._device:
            raise TypeError(f"{name}: a tensor of {like.dtype} on {self._device} is wanted")
        shape = m.shape
        if shape != like.shape:
            raise ValueError(f"{name}: shape {tuple(like.shape)} is wanted")
        if m.is_contiguous():
            return m.data_ptr(), (shape[-1] if shape else 1)
        if len(shape) > 2:
            try:
                m = m.view(-1, shape[-1])
            except RuntimeError:
                raise ValueError(f"{name}: rows the same distance apart are wanted") from None
        cols, stride = shape[-1], m.stride()
        if cols > 1 and stride[-1] != 1:
            raise ValueError(f"{name}: contiguous rows are wanted")
        pitch = cols if m.dim() == 1 or m.shape[0] == 1 else stride[0]
        if pitch < cols:
            raise ValueError(f"{name}: rows that do not overlap are wanted")
        return m.data_ptr(), pitch

    def _call(self, x, offset, residual, out):
        dtype = _operand_type(x.dtype)
        rule, tensor = self._rule(offset)
        if out is None:
            out = self._torch.empty_like(x)
        xp, yp = self._rows("x", x, x), self._rows("out", out, x)
        rp = (None, 0) if residual is None else self._rows("residual", residual, x)
        n = x.numel()
        if n == 0:
            return out
        cols = x.shape[-1] if x.dim() else 1
        here = self._enter(x, residual, out, tensor)
        if self._torch.cuda.current_device() == self._device.index:
            scar_dropout_apply(rule, dtype, *xp, *rp, *yp, n // cols, cols, self._stream.cuda_stream)
        else:
            with self._torch.cuda.device(self._device):
                scar_dropout_apply(rule, dtype, *xp, *rp, *yp, n // cols, cols, self._stream.cuda_stream)
        self._leave(here)
        return out

    def forward(self, x, offset=0, residual=None, out=None):
        """``residual + mask * x``; ``out`` may be ``x`` or the residual."""
        return self._call(x, offset, residual, out)

    def backward(self, dy, offset=0, out=None):
        """The gradient of x from that of the output (the residual's is ``dy`` itself)."""
        return self._call(dy, offset, None, out)


class _Rows(_OnStream):
    """Checks of matrices and vectors of one type on one device."""

    def _matrix(self, name: str, m, rows: int, cols: int):
        """Address and pitch."""
        if m.dtype != self.dtype or m.device != self._device:
            raise TypeError(f"{name}: a tensor of {self.dtype} on {self._device} is wanted")
        if m.shape != (rows, cols):
            raise ValueError(f"{name}: shape ({rows}, {cols}) is wanted")
        pitch, step = m.stride()
        if cols > 1 and step != 1:
            raise ValueError(f"{name}: contiguous rows are wanted")
        if rows <= 1:
            return m.data_ptr(), cols
        if pitch < cols:
            raise ValueError(f"{name}: rows that do not overlap are wanted")
        return m.data_ptr(), pitch

    def _vector(self, name: str, v, n: int):
        if v is None:
            return None
        if v.dtype != self.dtype or v.device != self._device:
            raise TypeError(f"{name}: a tensor of {self.dtype} on {self._device} is wanted")
        if v.numel() != n or not v.is_contiguous():
            raise ValueError(f"{name}: {n} contiguous values are wanted")
        return v.data_ptr()


_ACTIVATIONS = {"identity": SCAR_ACT_IDENTITY, "relu": SCAR_ACT_RELU, "gelu": SCAR_ACT_GELU, "silu": SCAR_ACT_SILU}


class LinearLayer(_Rows):
    """``residual + mask * act(x @ w.T + bias)`` in one operator, with its gradients.

    ``max_rows`` rows at most per call, ``out_features`` x ``in_features`` weights, all operands of ``dtype`` (float32,
    bfloat16 or float16).  ``activation``: ``"identity"``, ``"relu"``, ``"gelu"`` (with the Gaussian's distribution function)
    or ``"silu"``.  ``forward_only`` handles hold no workspace for gradients."""

    def __init__(self, max_rows: int, in_features: int, out_features: int, dtype, activation: str = "gelu", forward_only: bool = False,
                 stream=None, device="cuda"):
        import torch

        cfg = scar_linear_config(max_rows=max_rows, in_features=in_features, out_features=out_features, dtype=_operand_type(dtype),
                                 activation=_ACTIVATIONS[activation], forward_only=int(forward_only))
        self.max_rows, self.in_features, self.out_features, self.dtype, self.activation = max_rows, in_features, out_features, dtype, activation
        self._bind_stream(stream, device)
        with torch.cuda.device(self._device):
            self.op = scar_linear_init(cfg, self._stream.cuda_stream)

    def _mask(self, dropout):
        return (None, None) if dropout is None else (dropout.at(self._device), dropout.tensor)

    def _slope_type(self):
        return self._torch.float16 if self.dtype == self._torch.bfloat16 else self._torch.float32

    def _slope(self, slope, rows: int):
        if self.activation == "identity":
            if slope is not None:
                raise ValueError("slope: the identity has none")
            return None
        shape = (rows, -(-self.out_features // 8) * 8)
        if slope is None or slope.dtype != self._slope_type() or slope.device != self._device or slope.shape != shape or not slope.is_contiguous():
            raise ValueError(f"slope: a contiguous tensor of {shape} of {self._slope_type()} on {self._device} is wanted")
        return slope.data_ptr()

    def _forward(self, train, x, w, bias, residual, dropout, out, slope):
        rows, K, N = len(x) if x.dim() else 0, self.in_features, self.out_features
        xp, wp, bp = self._matrix("x", x, rows, K), self._matrix("w", w, N, K), self._vector("bias", bias, N)
        rp = (None, 0) if residual is None else self._matrix("residual", residual, rows, N)
        out = x.new_empty((rows, N)) if out is None else out
        yp = self._matrix("out", out, rows, N)
        if train and slope is None and self.activation != "identity":
            slope = x.new_empty((rows, -(-N // 8) * 8), dtype=self._slope_type())
        sp = self._slope(slope, rows) if train else None
        rule, offset = self._mask(dropout)
        here = self._enter(x, w, bias, residual, out, slope, offset)
        scar_linear_forward(self.op, *xp, *wp, bp, *rp, rule, rows, *yp, sp)
        self._leave(here)
        return (out, slope) if train else out

    def forward(self, x, w, bias=None, residual=None, dropout=None, out=None):
        """The layer's output.  ``dropout``: a mask of a :class:`Dropout` (``drop.mask(offset)``); ``out`` may be the residual and
        overlaps nothing else."""
        return self._forward(False, x, w, bias, residual, dropout, out, None)

    def forward_train(self, x, w, bias=None, residual=None, dropout=None, out=None, slope=None):
        """``(y, slope)``: the output, and the activation's derivative for :meth:`backward` (None for the identity)."""
        return self._forward(True, x, w, bias, residual, dropout, out, slope)

    def backward(self, dy, x, w, slope, dropout=None, dx=None, dw=None, dbias=None, need_dx: bool = True, need_dw: bool = True, need_dbias: bool = True):
        """``(dx, dw, dbias)`` from the gradient of the output, which is the residual's own; None for what is not needed."""
        rows, K, N = len(dy) if dy.dim() else 0, self.in_features, self.out_features
        dyp, xp, wp, sp = self._matrix("dy", dy, rows, N), self._matrix("x", x, rows, K), self._matrix("w", w, N, K), self._slope(slope, rows)
        dx = None if not need_dx else self._torch.empty_like(x) if dx is None else dx
        dw = None if not need_dw else self._torch.empty_like(w) if dw is None else dw
        dbias = None if not need_dbias else dy.new_empty((N,)) if dbias is None else dbias
        dxp = (None, 0) if dx is None else self._matrix("dx", dx, rows, K)
        dwp = (None, 0) if dw is None else self._matrix("dw", dw, N, K)
        dbp = self._vector("dbias", dbias, N)
        rule, offset = self._mask(dropout)
        here = self._enter(dy, x, w, slope, dx, dw, dbias, offset)
        scar_linear_backward(self.op, *dyp, *xp, *wp, sp, rule, rows, *dxp, *dwp, dbp)
        self._leave(here)
        return dx, dw, dbias

    def status(self) -> None:
        """Waits; raises if a wait inside a kernel of the calls since the last status gave up."""
        scar_linear_status(self.op)

    def workspace_bytes(self) -> int:
        return scar_linear_workspace_bytes(self.op)

    def close(self):
        if getattr(self, "op", None):
            scar_linear_destroy(self.op)
            self.op = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class ResidualNorm(_Rows):
    """The norms around a residual block: ``y = x + scale * gate * N(f; w_post, b_post)`` and ``n = N(y; w_pre, b_pre)`` in one pass
    over the rows, with the gradients.

    ``max_rows`` rows of ``dim`` values of ``dtype`` (float32, bfloat16 or float16); ``kind``: ``"rms"`` or ``"layer"`` (with means
    and biases).  ``post`` and ``pre`` say which of the norms a call has; a weight or bias that is None is 1 or 0.  The gate has one
    row for every ``rows_per_gate`` rows.  Without ``f`` (the first norm of a model) y is x.  ``forward_only`` handles hold no
    workspace for gradients."""

    def __init__(self, max_rows: int, dim: int, dtype, kind: str = "rms", eps: float = 1e-6, forward_only: bool = False, stream=None, device="cuda"):
        import torch

        cfg = scar_resnorm_config(max_rows=max_rows, dim=dim, eps=eps, dtype=_operand_type(dtype),
                                  kind={"rms": SCAR_RESNORM_RMS, "layer": SCAR_RESNORM_LAYER}[kind], forward_only=int(forward_only))
        self.max_rows, self.dim, self.dtype, self.kind = max_rows, dim, dtype, kind
        self._bind_stream(stream, device)
        with torch.cuda.device(self._device):
            self.op = scar_resnorm_init(cfg, self._stream.cuda_stream)

    def _block(self, rows, post, pre, scale, gate, rows_per_gate, w_post, b_post, w_pre, b_pre):
        if rows_per_gate < 1:
            raise ValueError("rows_per_gate: at least 1 is wanted")
        gp = (None, 0) if gate is None else self._matrix("gate", gate, -(-rows // rows_per_gate), self.dim)
        return scar_resnorm_block(post, pre, scale, *gp, rows_per_gate, self._vector("w_post", w_post, self.dim), self._vector("b_post", b_post, self.dim),
                                  self._vector("w_pre", w_pre, self.dim), self._vector("b_pre", b_pre, self.dim))

    def _maybe(self, name, m, rows):
        return (None, 0) if m is None else self._matrix(name, m, rows, self.dim)

    def forward(self, x, f=None, post: bool = True, pre: bool = True, scale: float = 1.0, gate=None, rows_per_gate: int = 1, w_post=None, b_post=None,
                w_pre=None, b_pre=None, y=None, n=None):
        """``(y, n)``; n is None without ``pre``, y is x itself without ``f``.  ``y`` may be given as x or f."""
        rows = len(x) if x.dim() else 0
        post = bool(post and f is not None)
        block = self._block(rows, post, pre, scale, gate, rows_per_gate, w_post, b_post, w_pre, b_pre)
        xp, fp = self._matrix("x", x, rows, self.dim), self._maybe("f", f, rows)
        if f is None and y is None:
            yp = (None, 0)
        else:
            y = self._torch.empty_like(x) if y is None else y
            yp = self._matrix("y", y, rows, self.dim)
        n = None if not pre else self._torch.empty_like(x) if n is None else n
        np_ = self._maybe("n", n, rows)
        here = self._enter(x, f, gate, w_post, b_post, w_pre, b_pre, y, n)
        scar_resnorm_forward(self.op, block, *xp, *fp, rows, *yp, *np_)
        self._leave(here)
        return (x if y is None else y), n

    def backward(self, dy, dn, y, f=None, post: bool = True, pre: bool = True, scale: float = 1.0, gate=None, rows_per_gate: int = 1, w_post=None,
                 b_post=None, w_pre=None, b_pre=None, out=None):
        """The gradients, by name: ``dx``, ``df``, ``dgate``, ``dw_post``, ``db_post``, ``dw_pre``, ``db_pre``, None where the call has no such
        input.  ``dy`` may be None (with ``pre``) where y goes nowhere else; without ``pre``, ``dn`` is None and ``y`` is not read.
        ``out``: a dictionary of tensors to write some of them to (None: not wanted)."""
        if dn is not None and not pre:
            raise ValueError("dn: a call without pre has no such gradient")
        some = dy if dy is not None else dn
        if some is None:
            raise ValueError("dy, dn: one of them is wanted")
        rows = len(some) if some.dim() else 0
        post = bool(post and f is not None)
        block = self._block(rows, post, pre, scale, gate, rows_per_gate, w_post, b_post, w_pre, b_pre)
        dyp, dnp = self._maybe("dy", dy, rows), self._maybe("dn", dn, rows)
        yp, fp = self._maybe("y", y if pre else None, rows), self._maybe("f", f, rows)
        has = {"dx": some, "df": f, "dgate": gate, "dw_post": w_post if post else None, "db_post": b_post if post else None,
               "dw_pre": w_pre if pre else None, "db_pre": b_pre if pre else None}
        out = out or {}
        for k, v in out.items():
            if k not in has or (v is not None and has[k] is None):
                raise ValueError(f"out: {k} is none of this call's gradients")
        got = {k: None if v is None else out[k] if k in out else self._torch.empty_like(v) for k, v in has.items()}
        matrices = [self._maybe(k, got[k], rows if k != "dgate" or gate is None else gate.shape[0]) for k in ("dx", "df", "dgate")]
        vectors = [self._vector(k, got[k], self.dim) for k in ("dw_post", "db_post", "dw_pre", "db_pre")]
        here = self._enter(dy, dn, y, f, gate, w_post, b_post, w_pre, b_pre, *got.values())
        scar_resnorm_backward(self.op, block, *dyp, *dnp, *yp, *fp, rows, *matrices[0], *matrices[1], *matrices[2], *vectors)
        self._leave(here)
        return got

    def status(self) -> None:
        """Waits; raises if a wait inside a kernel of the calls since the last status gave up."""
        scar_resnorm_status(self.op)

    def close(self):
        if getattr(self, "op", None):
            scar_resnorm_destroy(self.op)
            self.op = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
