"""Python binding of libpvlm.so, the MI355X (gfx950) ParallelVLM hot path.

Argument marshalling only: every step runs in the library's HIP kernels.
Tensors must be CUDA (HIP) tensors on the current device, C-contiguous, with
the dtypes the C ABI (include/pvlm.h) names.  Calls are enqueued on
``torch.cuda.current_stream()`` and return without synchronising.

There is no CPU fallback: if libpvlm.so is missing the import of a call's
library raises, telling the caller to build it.
"""
from __future__ import annotations

import ctypes
import os
import threading
from typing import Optional

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libpvlm.so")

PVLM_F32, PVLM_BF16, PVLM_E4M3, PVLM_E2M1 = 0, 1, 2, 3
PVLM_CRIT_MASS, PVLM_CRIT_COSSIM = 0, 1
PVLM_DEV_RANGE, PVLM_DEV_TIMEOUT, PVLM_DEV_PLACEMENT, PVLM_DEV_NO_PAGES = 1, 2, 4, 8

EXPORTS = (
    "pvlm_status_string", "pvlm_last_hip_error", "pvlm_version",
    "pvlm_set_stream_cu_budget", "pvlm_stream_cu_budget",
    "pvlm_verify_attn_workspace_size", "pvlm_verify_attn", "pvlm_verify_attn_paged",
    "pvlm_verify_attn_noalloc", "pvlm_verify_attn_noalloc_max_bytes",
    "pvlm_uvprune_workspace_size", "pvlm_uvprune_score", "pvlm_uvprune_criterion_cossim",
    "pvlm_prefill_epilogue_cossim",
    "pvlm_topk_workspace_size", "pvlm_topk_select", "pvlm_uvprune_topk_mass",
    "pvlm_gather_kv", "pvlm_gather_kv_paged",
    "pvlm_rope_append_q8", "pvlm_rope_append_q8_paged", "pvlm_quantize_kv", "pvlm_quantize_kv_paged",
    "pvlm_verify_attn_q8_workspace_size", "pvlm_verify_attn_q8", "pvlm_verify_attn_q8_paged",
    "pvlm_gather_kv_q8", "pvlm_gather_kv_q8_paged",
    "pvlm_pages_resize", "pvlm_slot_map", "pvlm_rotary_freqs", "pvlm_rotary_append", "pvlm_rotary_append_q4",
    "pvlm_quantize_kv_q4", "pvlm_quantize_kv_q4_paged",
    "pvlm_verify_attn_q4_workspace_size", "pvlm_verify_attn_q4", "pvlm_verify_attn_q4_paged",
    "pvlm_verify_attn_q4_ragged", "pvlm_verify_attn_q4_ragged_paged",
    "pvlm_gather_kv_q4", "pvlm_gather_kv_q4_paged",
    "pvlm_spec_accept_workspace_size", "pvlm_spec_accept",
    "pvlm_rope_append", "pvlm_rope_append_paged",
    "pvlm_speedup", "pvlm_window_size",
    "pvlm_pd_create", "pvlm_pd_destroy", "pvlm_pd_start", "pvlm_pd_plan", "pvlm_pd_finish",
    "pvlm_pd_output", "pvlm_pd_pending", "pvlm_pd_get_stats",
)


class PvlmError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str = ""):
        self.status = status
        msg = f"{where}: pvlm status {status}"
        if detail:
            msg += f" ({detail})"
        super().__init__(msg)


_lib = None
_lib_lock = threading.Lock()

_c = ctypes
_P = _c.c_void_p
_I = _c.c_int
_I64 = _c.c_int64
_SZ = _c.c_size_t
_F = _c.c_float
_D = _c.c_double

PVLM_ROUND_DOWN, PVLM_ROUND_UP, PVLM_ROUND_NEAREST, PVLM_ROUND_BEST = 0, 1, 2, 3
_ROUNDING = {"down": PVLM_ROUND_DOWN, "up": PVLM_ROUND_UP, "nearest": PVLM_ROUND_NEAREST,
             "best": PVLM_ROUND_BEST}


class SpeedupModel(_c.Structure):
    """pvlm_speedup_model: per-token times (units of the draft forward t) and
    speedups against target-only decoding."""
    _fields_ = [(n, _c.c_double) for n in (
        "t_sd_ideal", "t_psd_ideal", "t_sd", "t_psd", "t_psd_rollback",
        "v_sd_ideal", "v_psd_ideal", "v_sd", "v_psd", "v_psd_rollback",
        "expected_accepted", "expected_total")]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


PVLM_PD_PRE_VERIFY, PVLM_PD_POST_VERIFY, PVLM_PD_DONE = 0, 1, 2
_PD_MODES = {PVLM_PD_PRE_VERIFY: "pre", PVLM_PD_POST_VERIFY: "post", PVLM_PD_DONE: "done"}


class PdRound(_c.Structure):
    """pvlm_pd_round: what one round of the parallel decoding pipeline runs."""
    _fields_ = [("mode", _c.c_int32), ("verify_begin", _c.c_int32),
                ("verify_count", _c.c_int32), ("draft_begin", _c.c_int32),
                ("draft_count", _c.c_int32), ("cost", _c.c_double)]


class PdStats(_c.Structure):
    """pvlm_pd_stats: the scheduler's counters."""
    _fields_ = [("mode", _c.c_int32), ("committed", _c.c_int32), ("pending", _c.c_int32),
                ("target_rounds", _c.c_int32), ("max_draft_run", _c.c_int32),
                ("draft_keep", _c.c_int32), ("elapsed", _c.c_double)]


class RotaryParams(_c.Structure):
    """pvlm_rotary: how a model rotates its heads (see ``Rotary``)."""
    _fields_ = ([(n, _c.c_double) for n in ("base", "factor", "orig_ctx", "alpha", "beta", "mscale")]
                + [("rot_dim", _c.c_int32), ("layout", _c.c_int32), ("scaling", _c.c_int32),
                   ("sections", _c.c_int32 * 3)])


_ROTARY = [_I, _I64, _I, _I, _I, _c.POINTER(RotaryParams), _P, _P, _I64, _P, _I64, _P, _I64, _P, _I64, _I64]

_SIGS = {
    "pvlm_status_string": (_c.c_char_p, [_I]),
    "pvlm_last_hip_error": (_c.c_char_p, []),
    "pvlm_version": (_I, []),
    "pvlm_set_stream_cu_budget": (_I, [_P, _I]),
    "pvlm_stream_cu_budget": (_I, [_P]),
    "pvlm_verify_attn_workspace_size": (_SZ, [_I, _I, _I, _I, _I, _I, _I64, _I64]),
    "pvlm_verify_attn": (_I, [_I, _I, _I, _I, _I, _I, _I64, _I64, _F, _P, _P, _P, _P, _P, _P, _P,
                              _P, _SZ, _P, _P]),
    "pvlm_verify_attn_paged": (_I, [_I, _I, _I, _I, _I, _I, _I, _I, _I64, _I64, _F, _P, _P, _P,
                                    _P, _P, _P, _P, _P, _P, _SZ, _P, _P]),
    "pvlm_verify_attn_noalloc": (_I, [_I, _I, _I, _I, _I, _I, _I64, _I64, _F, _P, _P, _P, _P, _P,
                                      _P, _P, _P, _P]),
    "pvlm_verify_attn_noalloc_max_bytes": (_SZ, []),
    "pvlm_uvprune_workspace_size": (_SZ, [_I, _I, _I, _I64]),
    "pvlm_uvprune_score": (_I, [_I, _I, _I, _I64, _P, _P, _I, _I, _I64, _P, _P, _P, _P, _P, _SZ,
                                _P, _P]),
    "pvlm_uvprune_criterion_cossim": (_I, [_I, _I64, _P, _I, _I, _I64, _P, _P, _P, _P, _P, _SZ,
                                           _P, _P]),
    "pvlm_prefill_epilogue_cossim": (_I, [_I, _I64, _P, _I64, _P, _I, _I, _P, _P, _P, _P, _P, _P,
                                          _P, _P, _SZ, _P, _P]),
    "pvlm_topk_workspace_size": (_SZ, [_I, _I64]),
    "pvlm_topk_select": (_I, [_I, _I64, _P, _P, _I, _P, _P, _P, _SZ, _P, _P]),
    "pvlm_uvprune_topk_mass": (_I, [_I, _I, _I64, _P, _P, _P, _I, _P, _P, _P, _SZ, _P, _P]),
    "pvlm_gather_kv": (_I, [_I, _I, _I, _I, _I, _I64, _P, _P, _P, _P, _I, _P, _P, _I64, _P, _P,
                            _P, _P]),
    "pvlm_gather_kv_paged": (_I, [_I, _I, _I, _I, _I, _I, _I, _I64, _P, _P, _P, _P, _P, _I, _P,
                                  _P, _I64, _P, _P, _P, _P]),
    "pvlm_spec_accept_workspace_size": (_SZ, [_I, _I, _I]),
    "pvlm_spec_accept": (_I, [_I, _I, _I, _F, _P, _P, _P, _P, _P, _P, _P, _P, _P, _SZ, _P, _P]),
    "pvlm_speedup": (_I, [_D, _D, _I, _c.POINTER(SpeedupModel)]),
    "pvlm_window_size": (_I, [_D, _D, _I, _D, _I, _c.POINTER(_I), _c.POINTER(_D)]),
    "pvlm_rope_append": (_I, [_I, _I, _I, _I, _I, _I, _I64, _D, _P, _P, _P, _P, _P, _P, _P, _P,
                              _P, _P, _P]),
    "pvlm_rope_append_paged": (_I, [_I, _I, _I, _I, _I, _I, _I, _I, _I64, _D, _P, _P, _P, _P, _P,
                                    _P, _P, _P, _P, _P, _P, _P]),
    "pvlm_rope_append_q8": (_I, [_I, _I, _I, _I, _I, _I, _I64, _D] + [_P] * 13),
    "pvlm_rope_append_q8_paged": (_I, [_I, _I, _I, _I, _I, _I, _I, _I, _I64, _D] + [_P] * 14),
    "pvlm_quantize_kv": (_I, [_I, _I, _I, _I, _I, _I64, _P, _P, _P, _I64] + [_P] * 6),
    "pvlm_quantize_kv_paged": (_I, [_I, _I, _I, _I, _I, _I, _I, _I64, _I64] + [_P] * 10),
    "pvlm_verify_attn_q8_workspace_size": (_SZ, [_I, _I, _I, _I, _I, _I64, _I64]),
    "pvlm_verify_attn_q8": (_I, [_I, _I, _I, _I, _I, _I, _I64, _I64, _F] + [_P] * 10
                            + [_SZ, _P, _P]),
    "pvlm_verify_attn_q8_paged": (_I, [_I, _I, _I, _I, _I, _I, _I, _I, _I64, _I64, _F] + [_P] * 11
                                  + [_SZ, _P, _P]),
    "pvlm_gather_kv_q8": (_I, [_I, _I, _I, _I, _I, _I64, _P, _P, _P, _P, _P, _P, _I, _P, _P, _I64, _I]
                          + [_P] * 6),
    "pvlm_gather_kv_q8_paged": (_I, [_I, _I, _I, _I, _I, _I, _I, _I64, _P, _P, _P, _P, _P, _P, _P,
                                     _I, _P, _P, _I64, _I] + [_P] * 6),
    "pvlm_pages_resize": (_I, [_I, _I, _I, _I64] + [_P] * 8),
    "pvlm_slot_map": (_I, [_I, _I64, _I, _I, _I, _I64] + [_P] * 9),
    "pvlm_rotary_freqs": (_I, [_c.POINTER(RotaryParams), _c.POINTER(_D)]),
    "pvlm_rotary_append": (_I, _ROTARY + [_P] * 5),
    "pvlm_rotary_append_q4": (_I, _ROTARY + [_P] * 7),
    "pvlm_pd_create": (_I, [_I, _D, _I, _c.POINTER(_P)]),
    "pvlm_pd_destroy": (None, [_P]),
    "pvlm_pd_start": (_I, [_P, _P]),
    "pvlm_pd_plan": (_I, [_P, _c.POINTER(PdRound)]),
    "pvlm_pd_finish": (_I, [_P, _P, _I, _I, _c.c_int32]),
    "pvlm_pd_output": (_I, [_P, _P, _I, _c.POINTER(_I)]),
    "pvlm_pd_pending": (_I, [_P, _P, _I, _c.POINTER(_I)]),
    "pvlm_pd_get_stats": (_I, [_P, _c.POINTER(PdStats)]),
}

for _n in ("quantize_kv", "verify_attn", "gather_kv"):   # the same arguments as the 8-bit calls
    for _x in ("", "_paged"):
        _SIGS[f"pvlm_{_n}_q4{_x}"] = _SIGS[f"pvlm_{_n}{'' if _n == 'quantize_kv' else '_q8'}{_x}"]
for _x, _n in (("", 15), ("_paged", 18)):   # (n_new behind ctx_len)
    _r, _a = _SIGS[f"pvlm_verify_attn_q4{_x}"]
    _SIGS[f"pvlm_verify_attn_q4_ragged{_x}"] = (_r, _a[:_n] + [_P] + _a[_n:])
_SIGS["pvlm_verify_attn_q4_workspace_size"] = _SIGS["pvlm_verify_attn_q8_workspace_size"]


def lib():
    """The loaded libpvlm.so (loads it on first use; raises if not built)."""
    global _lib
    if _lib is None:
        with _lib_lock:
            if _lib is None:
                if not os.path.exists(LIB_PATH):
                    raise RuntimeError(
                        f"{LIB_PATH} is not built; run `python -c 'import __graft_entry__ as g; "
                        "g.build()'` or `python -m paper_2603_19610_amd.build`")
                L = ctypes.CDLL(LIB_PATH)
                for name, (res, args) in _SIGS.items():
                    fn = getattr(L, name)
                    fn.restype = res
                    fn.argtypes = args
                _lib = L
    return _lib


def _check(status: int, where: str):
    if status != 0:
        L = lib()
        detail = L.pvlm_status_string(status).decode()
        if status == 5:
            detail += ": " + L.pvlm_last_hip_error().decode()
        raise PvlmError(status, where, detail)


# A small call is bound by this module, not by its kernels: pointers and
# streams go to ctypes as plain integers (the argument types make the
# conversion), the raw stream is asked for directly (no torch.cuda.Stream object
# is built), and an argument that passes takes one test.  A rotary append with
# a verify call of one small layer: 35.7 -> 33.3 us (T = 4 rows over 504, paged).
def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _raw_stream(device: int) -> int:
    return torch._C._cuda_getCurrentRawStream(device)


def _stream():
    return _raw_stream(torch.cuda.current_device())


def _need(t: torch.Tensor, name: str, dtype=None, device=None):
    if (isinstance(t, torch.Tensor) and t.is_cuda and (device is None or t.device == device)
            and (dtype is None or t.dtype is dtype) and t.is_contiguous()):
        return t
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return PVLM_BF16
    if t.dtype == torch.float32:
        return PVLM_F32
    raise ValueError(f"unsupported dtype {t.dtype}")


class Workspace:
    """A zero-initialised device scratch buffer that grows on demand.

    The library leaves the words that it waits on zero after every call, so
    one buffer can serve successive calls on one stream (not concurrent
    calls: give each stream its own workspace).  A buffer that is outgrown is
    kept alive, not freed: a graph captured earlier, or a call still running,
    may use it.
    """

    def __init__(self, device=None):
        self.device = torch.device("cuda", torch.cuda.current_device()) if device is None else device
        self.buf = torch.zeros(256, dtype=torch.uint8, device=self.device)
        self._retired = []

    def get(self, nbytes: int) -> torch.Tensor:
        if nbytes > self.buf.numel():
            self._retired.append(self.buf)
            self.buf = torch.zeros(max(nbytes, 2 * self.buf.numel()), dtype=torch.uint8,
                                   device=self.device)
        return self.buf


# Default workspaces, one per (call kind, device, stream): calls on different
# streams never share records or data.
_ws_cache = {}
# Default status words, one per device (see synchronize()).
_status_cache = {}


def _no_capture(what: str):
    if torch.cuda.is_current_stream_capturing():
        raise PvlmError(4, "status", f"cannot {what} during graph capture: call "
                        "default_status() once before capturing, or pass status=")


def _default_ws(kind: str) -> Workspace:
    dev = torch.cuda.current_device()
    key = (kind, dev, _raw_stream(dev))
    ws = _ws_cache.get(key)
    if ws is None:
        # (under graph capture the buffer comes from the graph's pool and its
        # zero fill replays with the graph, ahead of the call)
        ws = _ws_cache[key] = Workspace()
    return ws


def _status(status):
    """The caller's status word, or this device's default one."""
    if status is not None:
        return status
    dev = torch.cuda.current_device()
    st = _status_cache.get(dev)
    if st is None:
        _no_capture("allocate the default status word")
        st = _status_cache[dev] = torch.zeros(1, dtype=torch.int32, device=torch.device("cuda", dev))
    return st


def default_status() -> torch.Tensor:
    """The status word calls without an explicit ``status`` OR their device
    flags (PVLM_DEV_*) into, on the current device."""
    return _status(None)


def synchronize(raise_on_status: bool = True) -> int:
    """Wait for the current device, then read and clear its default status
    word.  Raises PvlmError when a call flagged a device-side condition (an
    out-of-range device size, a wait that gave up, a misplaced workgroup)
    unless ``raise_on_status`` is False; returns the flags."""
    torch.cuda.synchronize()
    st = _status(None)
    flags = int(st.item())
    if flags:
        st.zero_()
        torch.cuda.synchronize()
        if raise_on_status:
            raise PvlmError(flags, "device status", _flag_text(flags))
    return flags


def _flag_text(flags: int) -> str:
    names = [(PVLM_DEV_RANGE, "device size out of range"), (PVLM_DEV_TIMEOUT, "wait gave up"),
             (PVLM_DEV_PLACEMENT, "workgroup placement"), (PVLM_DEV_NO_PAGES, "too few free pages")]
    return ", ".join(n for bit, n in names if flags & bit)


def release_workspaces():
    """Drop the default workspaces and status words (every call using them must
    have completed, and no live graph may reference them)."""
    torch.cuda.synchronize()
    _ws_cache.clear()
    _status_cache.clear()


# ------------------------------------------------------------------ calls --
def set_stream_cu_budget(stream, cus: int):
    """Give ``stream`` (a torch.cuda.Stream) a compute-unit budget: its verify
    and long-row top-k calls then plan for at most ``cus`` workgroups, so
    captured verify calls may run beside those of streams whose budgets sum
    with it to at most the device's compute units.  0 removes the budget."""
    _check(lib().pvlm_set_stream_cu_budget(_P(stream.cuda_stream), int(cus)),
           "pvlm_set_stream_cu_budget")


def stream_cu_budget(stream) -> int:
    return int(lib().pvlm_stream_cu_budget(_P(stream.cuda_stream)))


def verify_attn_workspace_size(dtype: int, B, T, Hq, Hkv, D, n_cap, max_ctx) -> int:
    return int(lib().pvlm_verify_attn_workspace_size(dtype, B, T, Hq, Hkv, D, n_cap, max_ctx))


def verify_attn(q, k_cache, v_cache, ctx_len, *, scale: Optional[float] = None,
                max_ctx: Optional[int] = None, out=None, mass=None, lse=None,
                want_mass: bool = True, want_lse: bool = True, ws: Optional[Workspace] = None,
                status=None):
    """Verify attention + attention mass.  q [B][T][Hq][D]; caches [B][Hkv][n_cap][D];
    ctx_len [B] int32.  Returns (out, mass or None, lse or None)."""
    _need(q, "q")
    dev = q.device
    _need(k_cache, "k_cache", q.dtype, dev)
    _need(v_cache, "v_cache", q.dtype, dev)
    _need(ctx_len, "ctx_len", torch.int32, dev)
    B, T, Hq, D = q.shape
    Bk, Hkv, n_cap, Dk = k_cache.shape
    if Bk != B or Dk != D or tuple(v_cache.shape) != tuple(k_cache.shape) or ctx_len.numel() != B:
        raise ValueError("inconsistent verify_attn shapes")
    dt = _dt(q)
    if scale is None:
        scale = D ** -0.5
    if max_ctx is None:
        max_ctx = n_cap - T
    if out is None:
        out = torch.empty_like(q)
    _need(out, "out", q.dtype, dev)
    if mass is None and want_mass:
        mass = torch.empty((B, n_cap), dtype=torch.float32, device=dev)
    if mass is not None:
        _need(mass, "mass", torch.float32, dev)
    if lse is None and want_lse:
        lse = torch.empty((B, Hq, T), dtype=torch.float32, device=dev)
    if lse is not None:
        _need(lse, "lse", torch.float32, dev)
    need = verify_attn_workspace_size(dt, B, T, Hq, Hkv, D, n_cap, max_ctx)
    wsb = (ws or _default_ws("verify")).get(need)
    st = lib().pvlm_verify_attn(dt, B, T, Hq, Hkv, D, n_cap, max_ctx, float(scale), _ptr(q),
                                _ptr(k_cache), _ptr(v_cache), _ptr(ctx_len), _ptr(out), _ptr(mass),
                                _ptr(lse), _ptr(wsb), wsb.numel(), _ptr(_status(status)), _stream())
    _check(st, "pvlm_verify_attn")
    return out, mass, lse


def _pool_shape(k_pool, v_pool, page_table, dev, dtype, stacked=False):
    _need(k_pool, "k_pool", dtype, dev)
    _need(v_pool, "v_pool", dtype, dev)
    _need(page_table, "page_table", torch.int32, dev)
    want = 5 if stacked else 4
    if k_pool.dim() != want or tuple(v_pool.shape) != tuple(k_pool.shape):
        raise ValueError("pools must be [n_pages][Hkv][page][D]" if not stacked else
                         "pools must be [n_pages][Hkv][page][D] or [L][n_pages][Hkv][page][D]")
    if page_table.dim() != 2:
        raise ValueError("page_table must be [B][max_pages]")
    return tuple(k_pool.shape)


def verify_attn_paged(q, k_pool, v_pool, page_table, ctx_len, *, scale: Optional[float] = None,
                      max_ctx: Optional[int] = None, out=None, mass=None, lse=None,
                      want_mass: bool = True, want_lse: bool = True,
                      ws: Optional[Workspace] = None, status=None):
    """pvlm_verify_attn_paged: verify attention + mass over a paged cache.
    q [B][T][Hq][D] bf16; pools [n_pages][Hkv][page][D]; page_table
    [B][max_pages] int32; mass is [B][max_pages * page] by logical row."""
    _need(q, "q", torch.bfloat16)
    dev = q.device
    n_pages, Hkv, page, Dk = _pool_shape(k_pool, v_pool, page_table, dev, q.dtype)
    _need(ctx_len, "ctx_len", torch.int32, dev)
    B, T, Hq, D = q.shape
    if Dk != D or page_table.shape[0] != B or ctx_len.numel() != B:
        raise ValueError("inconsistent verify_attn_paged shapes")
    max_pages = page_table.shape[1]
    n_cap = max_pages * page
    if scale is None:
        scale = D ** -0.5
    if max_ctx is None:
        max_ctx = n_cap - T
    if out is None:
        out = torch.empty_like(q)
    _need(out, "out", q.dtype, dev)
    if mass is None and want_mass:
        mass = torch.empty((B, n_cap), dtype=torch.float32, device=dev)
    if mass is not None:
        _need(mass, "mass", torch.float32, dev)
    if lse is None and want_lse:
        lse = torch.empty((B, Hq, T), dtype=torch.float32, device=dev)
    if lse is not None:
        _need(lse, "lse", torch.float32, dev)
    need = verify_attn_workspace_size(PVLM_BF16, B, T, Hq, Hkv, D, n_cap, max_ctx)
    wsb = (ws or _default_ws("verify")).get(need)
    st = lib().pvlm_verify_attn_paged(PVLM_BF16, B, T, Hq, Hkv, D, page, max_pages, n_pages,
                                      max_ctx, float(scale), _ptr(q), _ptr(k_pool), _ptr(v_pool),
                                      _ptr(page_table), _ptr(ctx_len), _ptr(out), _ptr(mass),
                                      _ptr(lse), _ptr(wsb), wsb.numel(), _ptr(_status(status)),
                                      _stream())
    _check(st, "pvlm_verify_attn_paged")
    return out, mass, lse


def verify_attn_noalloc(q, k_cache, v_cache, ctx_len, *, out, mass=None, lse=None,
                        scale: Optional[float] = None, max_ctx: Optional[int] = None, status=None):
    """pvlm_verify_attn_noalloc: verify attention + mass with the library's
    fixed device scratch (no workspace, nothing allocated: ``out`` and the
    optional ``mass`` / ``lse`` are the caller's).  Calls that overlap on one
    GPU race on the shared scratch."""
    _need(q, "q")
    dev = q.device
    _need(k_cache, "k_cache", q.dtype, dev)
    _need(v_cache, "v_cache", q.dtype, dev)
    _need(ctx_len, "ctx_len", torch.int32, dev)
    _need(out, "out", q.dtype, dev)
    B, T, Hq, D = q.shape
    Bk, Hkv, n_cap, Dk = k_cache.shape
    if Bk != B or Dk != D or tuple(v_cache.shape) != tuple(k_cache.shape) or ctx_len.numel() != B:
        raise ValueError("inconsistent verify_attn shapes")
    if mass is not None:
        _need(mass, "mass", torch.float32, dev)
    if lse is not None:
        _need(lse, "lse", torch.float32, dev)
    st = lib().pvlm_verify_attn_noalloc(_dt(q), B, T, Hq, Hkv, D, n_cap,
                                        n_cap - T if max_ctx is None else max_ctx,
                                        float(D ** -0.5 if scale is None else scale), _ptr(q),
                                        _ptr(k_cache), _ptr(v_cache), _ptr(ctx_len), _ptr(out),
                                        _ptr(mass), _ptr(lse), _ptr(status), _stream())
    _check(st, "pvlm_verify_attn_noalloc")
    return out, mass, lse


def uvprune_score_mass(crit_stack, m, *, score=None, status=None):
    """score = UV-Prune variation over a criterion stack crit_stack [L+1][B][m_cap] fp32."""
    _need(crit_stack, "crit_stack", torch.float32)
    dev = crit_stack.device
    _need(m, "m", torch.int32, dev)
    Lp1, B, m_cap = crit_stack.shape
    if score is None:
        score = torch.empty((B, m_cap), dtype=torch.float32, device=dev)
    _need(score, "score", torch.float32, dev)
    st = lib().pvlm_uvprune_score(PVLM_CRIT_MASS, B, Lp1 - 1, m_cap, _ptr(m), _ptr(crit_stack),
                                  PVLM_F32, 0, 0, None, None, None, _ptr(score), None, 0,
                                  _ptr(_status(status)), _stream())
    _check(st, "pvlm_uvprune_score")
    return score


def uvprune_score_cossim(hs_vis, hs_txt, m, n_txt, *, score=None, ws=None, status=None):
    """Eq. (average_similarity) from hidden states hs_vis [L+1][B][m_cap][Dh], hs_txt [L+1][B][n_cap][Dh]."""
    _need(hs_vis, "hs_vis")
    dev = hs_vis.device
    _need(hs_txt, "hs_txt", hs_vis.dtype, dev)
    _need(m, "m", torch.int32, dev)
    _need(n_txt, "n_txt", torch.int32, dev)
    Lp1, B, m_cap, Dh = hs_vis.shape
    n_cap = hs_txt.shape[2]
    if hs_txt.shape[0] != Lp1 or hs_txt.shape[1] != B or hs_txt.shape[3] != Dh:
        raise ValueError("inconsistent hidden-state shapes")
    if score is None:
        score = torch.empty((B, m_cap), dtype=torch.float32, device=dev)
    _need(score, "score", torch.float32, dev)
    need = int(lib().pvlm_uvprune_workspace_size(PVLM_CRIT_COSSIM, B, Dh, n_cap))
    wsb = (ws or _default_ws("uvprune")).get(need)
    st = lib().pvlm_uvprune_score(PVLM_CRIT_COSSIM, B, Lp1 - 1, m_cap, _ptr(m), None,
                                  _dt(hs_vis), Dh, n_cap, _ptr(n_txt), _ptr(hs_vis), _ptr(hs_txt),
                                  _ptr(score), _ptr(wsb), wsb.numel(), _ptr(_status(status)), _stream())
    _check(st, "pvlm_uvprune_score")
    return score


def uvprune_criterion_cossim(hv, ht, m, n_txt, *, out=None, ws=None, status=None):
    """One layer: c[b,i] = sum_j cos(hv[b,i], ht[b,j]); hv [B][m_cap][Dh], ht [B][n_cap][Dh]."""
    _need(hv, "hv")
    dev = hv.device
    _need(ht, "ht", hv.dtype, dev)
    _need(m, "m", torch.int32, dev)
    _need(n_txt, "n_txt", torch.int32, dev)
    B, m_cap, Dh = hv.shape
    n_cap = ht.shape[1]
    if out is None:
        out = torch.empty((B, m_cap), dtype=torch.float32, device=dev)
    _need(out, "out", torch.float32, dev)
    need = int(lib().pvlm_uvprune_workspace_size(PVLM_CRIT_COSSIM, B, Dh, n_cap))
    wsb = (ws or _default_ws("uvprune")).get(need)
    st = lib().pvlm_uvprune_criterion_cossim(B, m_cap, _ptr(m), _dt(hv), Dh, n_cap, _ptr(n_txt),
                                             _ptr(hv), _ptr(ht), _ptr(out), _ptr(wsb), wsb.numel(),
                                             _ptr(_status(status)), _stream())
    _check(st, "pvlm_uvprune_criterion_cossim")
    return out


def prefill_epilogue_cossim(vis_prev, vis_delta, txt_prev, txt_delta, m, n_txt, *, vis_out=None,
                            txt_out=None, crit=None, ws=None, status=None):
    """pvlm_prefill_epilogue_cossim: the residual add of a prefill layer's
    visual [B][m_cap][Dh] and text [B][n_cap][Dh] rows with the layer's
    COSSIM criterion of the result fused in.  Outputs default to new tensors
    (pass vis_out=vis_prev for an in-place add).  Returns (vis_out, txt_out,
    crit [B][m_cap])."""
    _need(vis_prev, "vis_prev")
    dev = vis_prev.device
    dtp = vis_prev.dtype
    for t, name in ((vis_delta, "vis_delta"), (txt_prev, "txt_prev"), (txt_delta, "txt_delta")):
        _need(t, name, dtp, dev)
    _need(m, "m", torch.int32, dev)
    _need(n_txt, "n_txt", torch.int32, dev)
    B, m_cap, Dh = vis_prev.shape
    n_cap = txt_prev.shape[1]
    if (tuple(vis_delta.shape) != (B, m_cap, Dh) or tuple(txt_prev.shape) != (B, n_cap, Dh)
            or tuple(txt_delta.shape) != (B, n_cap, Dh)):
        raise ValueError("inconsistent prefill_epilogue_cossim shapes")
    if vis_out is None:
        vis_out = torch.empty_like(vis_prev)
    if txt_out is None:
        txt_out = torch.empty_like(txt_prev)
    _need(vis_out, "vis_out", dtp, dev)
    _need(txt_out, "txt_out", dtp, dev)
    if crit is None:
        crit = torch.empty((B, m_cap), dtype=torch.float32, device=dev)
    _need(crit, "crit", torch.float32, dev)
    need = int(lib().pvlm_uvprune_workspace_size(PVLM_CRIT_COSSIM, B, Dh, n_cap))
    wsb = (ws or _default_ws("uvprune")).get(need)
    st = lib().pvlm_prefill_epilogue_cossim(B, m_cap, _ptr(m), n_cap, _ptr(n_txt), _dt(vis_prev), Dh,
                                            _ptr(vis_prev), _ptr(vis_delta), _ptr(vis_out),
                                            _ptr(txt_prev), _ptr(txt_delta), _ptr(txt_out),
                                            _ptr(crit), _ptr(wsb), wsb.numel(), _ptr(_status(status)),
                                            _stream())
    _check(st, "pvlm_prefill_epilogue_cossim")
    return vis_out, txt_out, crit


def topk_select(score, m, k, k_cap: int, *, idx=None, ws=None, status=None):
    """Ascending kept indices [B][k_cap] (-1 padded)."""
    _need(score, "score", torch.float32)
    dev = score.device
    _need(m, "m", torch.int32, dev)
    _need(k, "k", torch.int32, dev)
    B, m_cap = score.shape
    if idx is None:
        idx = torch.empty((B, k_cap), dtype=torch.int32, device=dev)
    _need(idx, "idx", torch.int32, dev)
    need = int(lib().pvlm_topk_workspace_size(B, m_cap))
    wsb = (ws or _default_ws("topk")).get(need) if need else None
    st = lib().pvlm_topk_select(B, m_cap, _ptr(m), _ptr(k), int(k_cap), _ptr(score), _ptr(idx),
                                _ptr(wsb), 0 if wsb is None else wsb.numel(), _ptr(_status(status)),
                                _stream())
    _check(st, "pvlm_topk_select")
    return idx


def uvprune_topk_mass(crit_stack, m, k, k_cap: int, *, score=None, want_score: bool = True,
                      idx=None, ws=None, status=None):
    """pvlm_uvprune_topk_mass: the MASS score crit_stack[L] - crit_stack[0]
    ([L+1][B][m_cap] fp32) and its top-k in one call.  Returns (score or
    None, idx)."""
    _need(crit_stack, "crit_stack", torch.float32)
    dev = crit_stack.device
    _need(m, "m", torch.int32, dev)
    _need(k, "k", torch.int32, dev)
    L1, B, m_cap = crit_stack.shape
    if score is None and want_score:
        score = torch.empty((B, m_cap), dtype=torch.float32, device=dev)
    if score is not None:
        _need(score, "score", torch.float32, dev)
    if idx is None:
        idx = torch.empty((B, k_cap), dtype=torch.int32, device=dev)
    _need(idx, "idx", torch.int32, dev)
    need = int(lib().pvlm_topk_workspace_size(B, m_cap))
    wsb = (ws or _default_ws("topk")).get(need) if need else None
    st = lib().pvlm_uvprune_topk_mass(B, L1 - 1, m_cap, _ptr(m), _ptr(crit_stack), _ptr(k),
                                      int(k_cap), _ptr(score), _ptr(idx), _ptr(wsb),
                                      0 if wsb is None else wsb.numel(), _ptr(_status(status)),
                                      _stream())
    _check(st, "pvlm_uvprune_topk_mass")
    return score, idx


def gather_kv(k_cache, v_cache, idx, k, tail_begin, tail_len, dst_cap: int, *, k_dst=None,
              v_dst=None, status=None):
    """Compact cache: kept rows then tail rows.  Caches are [B][Hkv][n_cap][D]
    (one layer) or [L][B][Hkv][n_cap][D] (a stacked cache, one launch);
    outputs have the same leading dims with dst_cap rows."""
    _need(k_cache, "k_cache")
    dev = k_cache.device
    _need(v_cache, "v_cache", k_cache.dtype, dev)
    _need(idx, "idx", torch.int32, dev)
    for name, t in (("k", k), ("tail_begin", tail_begin), ("tail_len", tail_len)):
        _need(t, name, torch.int32, dev)
    if k_cache.dim() == 4:
        n_layers, (B, Hkv, n_cap, D) = 1, k_cache.shape
    elif k_cache.dim() == 5:
        n_layers, B, Hkv, n_cap, D = k_cache.shape
    else:
        raise ValueError("k_cache must be [B][Hkv][n_cap][D] or [L][B][Hkv][n_cap][D]")
    if tuple(v_cache.shape) != tuple(k_cache.shape) or idx.shape[0] != B:
        raise ValueError("inconsistent gather_kv shapes")
    dst_shape = tuple(k_cache.shape[:-2]) + (dst_cap, D)
    if k_dst is None:
        k_dst = torch.zeros(dst_shape, dtype=k_cache.dtype, device=dev)
    if v_dst is None:
        v_dst = torch.zeros(dst_shape, dtype=k_cache.dtype, device=dev)
    _need(k_dst, "k_dst", k_cache.dtype, dev)
    _need(v_dst, "v_dst", k_cache.dtype, dev)
    if tuple(k_dst.shape) != dst_shape or tuple(v_dst.shape) != dst_shape:
        raise ValueError("destination shape mismatch")
    st = lib().pvlm_gather_kv(_dt(k_cache), n_layers, B, Hkv, D, n_cap, _ptr(k_cache),
                              _ptr(v_cache), _ptr(idx), _ptr(k), idx.shape[1], _ptr(tail_begin),
                              _ptr(tail_len), dst_cap, _ptr(k_dst), _ptr(v_dst),
                              _ptr(_status(status)), _stream())
    _check(st, "pvlm_gather_kv")
    return k_dst, v_dst


def gather_kv_paged(k_pool, v_pool, page_table, idx, k, tail_begin, tail_len, dst_cap: int, *,
                    k_dst=None, v_dst=None, status=None):
    """pvlm_gather_kv_paged: compact cache from a paged pool.  Pools are
    [n_pages][Hkv][page][D] (one layer) or [L][n_pages][Hkv][page][D]; one
    page_table [B][max_pages] serves every layer; outputs [(L,) B, Hkv, dst_cap, D]."""
    _need(k_pool, "k_pool")
    dev = k_pool.device
    if k_pool.dim() == 4:
        n_layers, (n_pages, Hkv, page, D) = 1, k_pool.shape
    elif k_pool.dim() == 5:
        n_layers, n_pages, Hkv, page, D = k_pool.shape
    else:
        raise ValueError("pools must be [n_pages][Hkv][page][D] or [L][n_pages][Hkv][page][D]")
    _need(v_pool, "v_pool", k_pool.dtype, dev)
    _need(page_table, "page_table", torch.int32, dev)
    _need(idx, "idx", torch.int32, dev)
    for name, t in (("k", k), ("tail_begin", tail_begin), ("tail_len", tail_len)):
        _need(t, name, torch.int32, dev)
    if tuple(v_pool.shape) != tuple(k_pool.shape) or page_table.dim() != 2:
        raise ValueError("inconsistent gather_kv_paged shapes")
    B, max_pages = page_table.shape
    if idx.shape[0] != B:
        raise ValueError("idx must be [B][k_cap]")
    dst_shape = ((n_layers,) if k_pool.dim() == 5 else ()) + (B, Hkv, dst_cap, D)
    if k_dst is None:
        k_dst = torch.zeros(dst_shape, dtype=k_pool.dtype, device=dev)
    if v_dst is None:
        v_dst = torch.zeros(dst_shape, dtype=k_pool.dtype, device=dev)
    _need(k_dst, "k_dst", k_pool.dtype, dev)
    _need(v_dst, "v_dst", k_pool.dtype, dev)
    if tuple(k_dst.shape) != dst_shape or tuple(v_dst.shape) != dst_shape:
        raise ValueError("destination shape mismatch")
    st = lib().pvlm_gather_kv_paged(_dt(k_pool), n_layers, B, Hkv, D, page, max_pages, n_pages,
                                    _ptr(k_pool), _ptr(v_pool), _ptr(page_table), _ptr(idx),
                                    _ptr(k), idx.shape[1], _ptr(tail_begin), _ptr(tail_len),
                                    dst_cap, _ptr(k_dst), _ptr(v_dst), _ptr(_status(status)),
                                    _stream())
    _check(st, "pvlm_gather_kv_paged")
    return k_dst, v_dst


def spec_accept(draft_logits, target_logits, draft_tokens, u_accept, u_sample,
                temperature: float, *, n_accepted=None, next_token=None, near_tie=None,
                ws: Optional[Workspace] = None, status=None):
    """Returns (n_accepted [B], next_token [B], near_tie [B]) int32 tensors."""
    _need(draft_logits, "draft_logits", torch.float32)
    dev = draft_logits.device
    _need(target_logits, "target_logits", torch.float32, dev)
    _need(draft_tokens, "draft_tokens", torch.int32, dev)
    _need(u_accept, "u_accept", torch.float64, dev)
    _need(u_sample, "u_sample", torch.float64, dev)
    B, gamma, V = draft_logits.shape
    if tuple(target_logits.shape) != (B, gamma + 1, V):
        raise ValueError("target_logits must be [B][gamma+1][V]")
    if n_accepted is None:
        n_accepted = torch.empty(B, dtype=torch.int32, device=dev)
    if next_token is None:
        next_token = torch.empty(B, dtype=torch.int32, device=dev)
    if near_tie is None:
        near_tie = torch.empty(B, dtype=torch.int32, device=dev)
    need = int(lib().pvlm_spec_accept_workspace_size(B, gamma, V))
    wsb = (ws or _default_ws("accept")).get(need)
    st = lib().pvlm_spec_accept(B, gamma, V, float(temperature), _ptr(draft_logits),
                                _ptr(target_logits), _ptr(draft_tokens), _ptr(u_accept),
                                _ptr(u_sample), _ptr(n_accepted), _ptr(next_token), _ptr(near_tie),
                                _ptr(wsb), wsb.numel(), _ptr(_status(status)), _stream())
    _check(st, "pvlm_spec_accept")
    return n_accepted, next_token, near_tie


__all__ = [
    "LIB_PATH", "EXPORTS", "PvlmError", "Workspace", "lib", "synchronize", "default_status",
    "release_workspaces", "set_stream_cu_budget", "stream_cu_budget",
    "verify_attn", "verify_attn_paged", "verify_attn_noalloc",
    "gather_kv_paged", "rope_append", "rope_append_paged",
    "rope_append_q8", "rope_append_q8_paged", "quantize_kv", "quantize_kv_paged",
    "verify_attn_q8", "verify_attn_q8_paged", "verify_attn_q8_workspace_size",
    "gather_kv_q8", "gather_kv_q8_paged",
    "pages_resize", "slot_map", "Rotary", "rotary_append", "rotary_append_q4", "quantize_kv_q4",
    "quantize_kv_q4_paged", "verify_attn_q4", "verify_attn_q4_paged", "verify_attn_q4_workspace_size",
    "gather_kv_q4", "gather_kv_q4_paged",
    "verify_attn_workspace_size", "uvprune_score_mass", "uvprune_score_cossim",
    "uvprune_criterion_cossim", "prefill_epilogue_cossim", "topk_select", "uvprune_topk_mass", "gather_kv", "spec_accept",
    "PVLM_F32", "PVLM_BF16", "PVLM_E4M3", "PVLM_E2M1", "PVLM_CRIT_MASS", "PVLM_CRIT_COSSIM", "PVLM_DEV_RANGE",
    "PVLM_DEV_TIMEOUT", "PVLM_DEV_PLACEMENT", "PVLM_DEV_NO_PAGES",
]


def speedup(c: float, tau: float, gamma: int) -> dict:
    """pvlm_speedup: the speedup analysis for speed ratio c, acceptance rate
    tau and window gamma (host arithmetic, no GPU)."""
    out = SpeedupModel()
    _check(lib().pvlm_speedup(float(c), float(tau), int(gamma), _c.byref(out)), "speedup")
    return out.as_dict()


def window_size(t_p: float, t_q: float, rounding: str = "down", tau: float = 0.0,
                gamma_max: int = 64):
    """pvlm_window_size: the draft window gamma = T_p / T_q rounded as asked;
    returns (gamma, c)."""
    if rounding not in _ROUNDING:
        raise ValueError(f"rounding must be one of {sorted(_ROUNDING)}")
    g, c = _I(0), _D(0.0)
    _check(lib().pvlm_window_size(float(t_p), float(t_q), _ROUNDING[rounding], float(tau),
                                  int(gamma_max), _c.byref(g), _c.byref(c)), "window_size")
    return g.value, c.value


class Scheduler:
    """The library's parallel decoding scheduler (pvlm_pd_*): host state only.

    ``plan()`` says what the next round runs, ``finish()`` reports the
    target's verdict; tokens are Python ints."""

    def __init__(self, gamma: int, c: float, max_len: int):
        h = _P()
        _check(lib().pvlm_pd_create(int(gamma), float(c), int(max_len), _c.byref(h)),
               "pd_create")
        self._h = h
        self.gamma = int(gamma)

    def close(self):
        if self._h is not None and self._h.value:
            lib().pvlm_pd_destroy(self._h)
        self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @staticmethod
    def _arr(tokens):
        tokens = list(tokens)
        return (_c.c_int32 * max(len(tokens), 1))(*tokens), len(tokens)

    def start(self, startup):
        arr, n = self._arr(startup)
        if n != self.gamma + 1:
            raise ValueError(f"startup needs gamma + 1 = {self.gamma + 1} tokens")
        _check(lib().pvlm_pd_start(self._h, arr), "pd_start")

    def plan(self) -> dict:
        r = PdRound()
        _check(lib().pvlm_pd_plan(self._h, _c.byref(r)), "pd_plan")
        d = {n: getattr(r, n) for n, _ in r._fields_}
        d["mode"] = _PD_MODES[r.mode]
        return d

    def finish(self, drafted, n_accepted: int, target_token=None):
        arr, n = self._arr(drafted)
        tok = -1 if target_token is None else int(target_token)
        _check(lib().pvlm_pd_finish(self._h, arr if n else None, n, int(n_accepted), tok),
               "pd_finish")

    def _tokens(self, fn):
        n = _I(0)
        _check(fn(self._h, None, 0, _c.byref(n)), "pd_tokens")
        buf = (_c.c_int32 * max(n.value, 1))()
        _check(fn(self._h, buf, n.value, _c.byref(n)), "pd_tokens")
        return list(buf[:n.value])

    def output(self):
        return self._tokens(lib().pvlm_pd_output)

    def pending(self):
        return self._tokens(lib().pvlm_pd_pending)

    def stats(self) -> dict:
        st = PdStats()
        _check(lib().pvlm_pd_get_stats(self._h, _c.byref(st)), "pd_stats")
        d = {n: getattr(st, n) for n, _ in st._fields_}
        d["mode"] = _PD_MODES[st.mode]
        return d


def rope_append(q, k_new, v_new, pos, ctx_len, k_cache, v_cache, *, base: float,
                sections=None, q_out=None, status=None):
    """pvlm_rope_append: rotate q and k_new by their positions (1-D RoPE, or
    M-RoPE with ``sections`` = (s0, s1, s2)) and write k_new / v_new into the
    caches at rows ctx_len[b] + t.  q [B][T][Hq][D]; k_new, v_new [B][T][Hkv][D];
    pos [B][T] or [3][B][T] int32; caches [B][Hkv][n_cap][D].  Returns q_out."""
    _need(q, "q")
    dev = q.device
    for t, name in ((k_new, "k_new"), (v_new, "v_new"), (k_cache, "k_cache"),
                    (v_cache, "v_cache")):
        _need(t, name, q.dtype, dev)
    _need(pos, "pos", torch.int32, dev)
    _need(ctx_len, "ctx_len", torch.int32, dev)
    B, T, Hq, D = q.shape
    Hkv = k_new.shape[2]
    n_cap = k_cache.shape[2]
    if tuple(k_new.shape) != (B, T, Hkv, D) or tuple(v_new.shape) != (B, T, Hkv, D):
        raise ValueError("k_new and v_new must be [B][T][Hkv][D]")
    if tuple(k_cache.shape) != (B, Hkv, n_cap, D) or tuple(v_cache.shape) != (B, Hkv, n_cap, D):
        raise ValueError("caches must be [B][Hkv][n_cap][D]")
    want = (B, T) if sections is None else (3, B, T)
    if tuple(pos.shape) != want:
        raise ValueError(f"pos must be {list(want)}")
    if tuple(ctx_len.shape) != (B,):
        raise ValueError("ctx_len must be [B]")
    if q_out is None:
        q_out = torch.empty_like(q)
    else:
        _need(q_out, "q_out", q.dtype, dev)
    sec = None if sections is None else (_c.c_int32 * 3)(*[int(x) for x in sections])
    st = lib().pvlm_rope_append(_dt(q), B, T, Hq, Hkv, D, n_cap, float(base), sec, _ptr(pos),
                                _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(ctx_len), _ptr(q_out),
                                _ptr(k_cache), _ptr(v_cache), _ptr(_status(status)), _stream())
    _check(st, "pvlm_rope_append")
    return q_out


def rope_append_paged(q, k_new, v_new, pos, ctx_len, k_pool, v_pool, page_table, *, base: float,
                      sections=None, q_out=None, status=None):
    """pvlm_rope_append_paged: as ``rope_append``, writing the new rows into
    the pools [n_pages][Hkv][page][D] through page_table [B][max_pages]."""
    _need(q, "q")
    dev = q.device
    for t, name in ((k_new, "k_new"), (v_new, "v_new")):
        _need(t, name, q.dtype, dev)
    n_pages, Hkv, page, Dp = _pool_shape(k_pool, v_pool, page_table, dev, q.dtype)
    _need(pos, "pos", torch.int32, dev)
    _need(ctx_len, "ctx_len", torch.int32, dev)
    B, T, Hq, D = q.shape
    if tuple(k_new.shape) != (B, T, Hkv, D) or tuple(v_new.shape) != (B, T, Hkv, D) or Dp != D:
        raise ValueError("k_new and v_new must be [B][T][Hkv][D] matching the pools")
    if page_table.shape[0] != B or tuple(ctx_len.shape) != (B,):
        raise ValueError("page_table must be [B][max_pages] and ctx_len [B]")
    want = (B, T) if sections is None else (3, B, T)
    if tuple(pos.shape) != want:
        raise ValueError(f"pos must be {list(want)}")
    if q_out is None:
        q_out = torch.empty_like(q)
    else:
        _need(q_out, "q_out", q.dtype, dev)
    sec = None if sections is None else (_c.c_int32 * 3)(*[int(x) for x in sections])
    st = lib().pvlm_rope_append_paged(_dt(q), B, T, Hq, Hkv, D, page, page_table.shape[1], n_pages,
                                      float(base), sec, _ptr(pos), _ptr(q), _ptr(k_new),
                                      _ptr(v_new), _ptr(page_table), _ptr(ctx_len), _ptr(q_out),
                                      _ptr(k_pool), _ptr(v_pool), _ptr(_status(status)),
                                      _stream())
    _check(st, "pvlm_rope_append_paged")
    return q_out


# ------------------------------------------------------------ 8-bit caches --
# Codes are torch.float8_e4m3fn (or the same bytes as torch.uint8), exponents
# torch.uint8: a row stands for code * 2^(exponent - 127).
def _need_q8(k_codes, k_exps, v_codes, v_exps, dev, paged, stacked=None):
    """Check a cache's four tensors; returns the codes' shape.  ``dev`` has to be
    the current device (its stream is the one that a call is enqueued on)."""
    if dev.index != torch.cuda.current_device():
        raise ValueError(f"tensors are on {dev}, but the current device is cuda:{torch.cuda.current_device()}")
    for t, name in ((k_codes, "k_codes"), (v_codes, "v_codes")):
        _need(t, name, None, dev)
        if t.dtype is not torch.float8_e4m3fn and t.dtype is not torch.uint8:
            raise ValueError(f"{name} must be torch.float8_e4m3fn or torch.uint8, got {t.dtype}")
    _need(k_exps, "k_exps", torch.uint8, dev)
    _need(v_exps, "v_exps", torch.uint8, dev)
    shape = k_codes.shape
    if len(shape) != 4 and not (stacked and len(shape) == 5):
        layout = "[n_pages][Hkv][page][D]" if paged else "[B][Hkv][n_cap][D]"
        raise ValueError(f"codes must be {layout}" + (f" or [L]{layout}" if stacked else ""))
    if v_codes.shape != shape or k_exps.shape != shape[:-1] or v_exps.shape != shape[:-1]:
        raise ValueError("k_codes and v_codes must have one shape, k_exps and v_exps that shape without D")
    return shape


def _ws_buffer(kind, ws, nbytes, dev):
    """The buffer of a call whose launches rely on nothing that a workspace held
    before.  A captured call without a workspace of its own takes one of its
    graph's memory, as its temporaries are: graphs captured on one stream may
    be replayed on different ones at once, beside that stream's eager calls."""
    if ws is None and torch.cuda.is_current_stream_capturing():
        return torch.empty(max(nbytes, 1), dtype=torch.uint8, device=dev)
    return (ws or _default_ws(kind)).get(nbytes)


def _need_table(page_table, dev, B):
    _need(page_table, "page_table", torch.int32, dev)
    if page_table.dim() != 2 or page_table.shape[0] != B:
        raise ValueError("page_table must be [B][max_pages]")
    return page_table.shape[1]


def _append_q8(q, k_new, v_new, pos, ctx_len, cache, page_table, base, sections, q_out, status):
    _need(q, "q", torch.bfloat16)
    dev = q.device
    _need(k_new, "k_new", torch.bfloat16, dev)
    _need(v_new, "v_new", torch.bfloat16, dev)
    n0, Hkv, rows, Dc = _need_q8(*cache, dev, page_table is not None)
    _need(pos, "pos", torch.int32, dev)
    _need(ctx_len, "ctx_len", torch.int32, dev)
    if q.dim() != 4:
        raise ValueError("q must be [B][T][Hq][D]")
    B, T, Hq, D = q.shape
    if k_new.shape != (B, T, Hkv, D) or v_new.shape != k_new.shape or Dc != D:
        raise ValueError("k_new and v_new must be [B][T][Hkv][D] matching the cache")
    if ctx_len.shape != (B,):
        raise ValueError("ctx_len must be [B]")
    want = (B, T) if sections is None else (3, B, T)
    if pos.shape != want:
        raise ValueError(f"pos must be {list(want)}")
    if page_table is None and n0 != B:
        raise ValueError("the cache must be [B][Hkv][n_cap][D]")
    geom = (rows,) if page_table is None else (rows, _need_table(page_table, dev, B), n0)
    if q_out is None:
        q_out = torch.empty_like(q)
    else:
        _need(q_out, "q_out", torch.bfloat16, dev)
        if q_out.shape != q.shape:
            raise ValueError("q_out must have q's shape")
    sec = None if sections is None else (_c.c_int32 * 3)(*[int(x) for x in sections])
    name = "pvlm_rope_append_q8" if page_table is None else "pvlm_rope_append_q8_paged"
    rows_in = (q.data_ptr(), k_new.data_ptr(), v_new.data_ptr())
    table = () if page_table is None else (page_table.data_ptr(),)
    st = getattr(lib(), name)(PVLM_BF16, B, T, Hq, Hkv, D, *geom, float(base), sec, pos.data_ptr(), *rows_in,
                              *table, ctx_len.data_ptr(), q_out.data_ptr(), *[t.data_ptr() for t in cache],
                              _ptr(_status(status)), _stream())
    _check(st, name)
    return q_out


def rope_append_q8(q, k_new, v_new, pos, ctx_len, k_codes, k_exps, v_codes, v_exps, *, base: float,
                   sections=None, q_out=None, status=None):
    """pvlm_rope_append_q8: as ``rope_append`` (bf16), writing the new rows in 8
    bits: codes [B][Hkv][n_cap][D] and exponents [B][Hkv][n_cap], n_cap a
    multiple of 32.  Returns q_out."""
    return _append_q8(q, k_new, v_new, pos, ctx_len, (k_codes, k_exps, v_codes, v_exps), None, base,
                      sections, q_out, status)


def rope_append_q8_paged(q, k_new, v_new, pos, ctx_len, k_codes, k_exps, v_codes, v_exps, page_table, *,
                         base: float, sections=None, q_out=None, status=None):
    """pvlm_rope_append_q8_paged: the same into pools [n_pages][Hkv][page][D]
    with exponents [n_pages][Hkv][page], through page_table [B][max_pages]."""
    if page_table is None:
        raise TypeError("page_table must be a torch.Tensor")
    return _append_q8(q, k_new, v_new, pos, ctx_len, (k_codes, k_exps, v_codes, v_exps), page_table, base,
                      sections, q_out, status)


def _quantize(k, v, length, cache, page_table, status):
    _need(k, "k")
    dev = k.device
    _need(v, "v", k.dtype, dev)
    _need(length, "length", torch.int32, dev)
    shape = _need_q8(*cache, dev, page_table is not None, stacked=True)
    if k.dim() != len(shape) or v.shape != k.shape:
        raise ValueError("k and v must be [B][Hkv][src_cap][D], or [L][...] with a stacked cache")
    L = 1 if k.dim() == 4 else k.shape[0]
    B, Hkv, src_cap, D = k.shape[-4:]
    n0, H, rows, Dc = shape[-4:]
    if (H, Dc) != (Hkv, D) or (len(shape) == 5 and shape[0] != L) or (page_table is None and n0 != B):
        raise ValueError("the 8-bit cache does not match k and v")
    if length.shape != (B,):
        raise ValueError("length must be [B]")
    codes = [t.data_ptr() for t in cache]
    if page_table is None:
        st = lib().pvlm_quantize_kv(_dt(k), L, B, Hkv, D, src_cap, k.data_ptr(), v.data_ptr(),
                                    length.data_ptr(), rows, *codes, _ptr(_status(status)), _stream())
        _check(st, "pvlm_quantize_kv")
    else:
        st = lib().pvlm_quantize_kv_paged(_dt(k), L, B, Hkv, D, rows, _need_table(page_table, dev, B), n0,
                                          src_cap, k.data_ptr(), v.data_ptr(), length.data_ptr(),
                                          page_table.data_ptr(), *codes, _ptr(_status(status)), _stream())
        _check(st, "pvlm_quantize_kv_paged")


def quantize_kv(k, v, length, k_codes, k_exps, v_codes, v_exps, *, status=None):
    """pvlm_quantize_kv: rows 0 .. length[b] - 1 of a bf16 or fp32 cache
    [B][Hkv][src_cap][D] (or [L][...]: every layer in one launch) into an 8-bit
    one [B][Hkv][n_cap][D] (or [L][...]); its other rows stay as they are."""
    _quantize(k, v, length, (k_codes, k_exps, v_codes, v_exps), None, status)


def quantize_kv_paged(k, v, length, k_codes, k_exps, v_codes, v_exps, page_table, *, status=None):
    """pvlm_quantize_kv_paged: the same into pools [n_pages][Hkv][page][D] (or
    [L][...]; one page_table [B][max_pages] serves every layer)."""
    if page_table is None:
        raise TypeError("page_table must be a torch.Tensor")
    _quantize(k, v, length, (k_codes, k_exps, v_codes, v_exps), page_table, status)


def verify_attn_q8_workspace_size(B, T, Hq, Hkv, D, n_cap, max_ctx) -> int:
    return int(lib().pvlm_verify_attn_q8_workspace_size(B, T, Hq, Hkv, D, n_cap, max_ctx))


def _verify_q8(q, cache, page_table, ctx_len, scale, max_ctx, out, mass, lse, want_mass, want_lse, ws, status):
    _need(q, "q", torch.bfloat16)
    dev = q.device
    n0, Hkv, rows, Dc = _need_q8(*cache, dev, page_table is not None)
    _need(ctx_len, "ctx_len", torch.int32, dev)
    if q.dim() != 4:
        raise ValueError("q must be [B][T][Hq][D]")
    B, T, Hq, D = q.shape
    if Dc != D or ctx_len.shape != (B,) or (page_table is None and n0 != B):
        raise ValueError("inconsistent verify_attn_q8 shapes")
    if page_table is None:
        n_cap, geom, table = rows, (rows,), ()
    else:
        max_pages = _need_table(page_table, dev, B)
        n_cap, geom, table = max_pages * rows, (rows, max_pages, n0), (page_table.data_ptr(),)
    if max_ctx is None:
        max_ctx = n_cap - T
    if out is None:
        out = torch.empty_like(q)
    elif _need(out, "out", torch.bfloat16, dev).shape != q.shape:
        raise ValueError("out must have q's shape")
    if mass is None:
        mass = torch.empty((B, n_cap), dtype=torch.float32, device=dev) if want_mass else None
    elif _need(mass, "mass", torch.float32, dev).shape != (B, n_cap):
        raise ValueError("mass must be [B][n_cap]")
    if lse is None:
        lse = torch.empty((B, Hq, T), dtype=torch.float32, device=dev) if want_lse else None
    elif _need(lse, "lse", torch.float32, dev).shape != (B, Hq, T):
        raise ValueError("lse must be [B][Hq][T]")
    L = lib()
    wsb = _ws_buffer("verify_q8", ws, L.pvlm_verify_attn_q8_workspace_size(B, T, Hq, Hkv, D, n_cap, max_ctx), dev)
    name = "pvlm_verify_attn_q8" if page_table is None else "pvlm_verify_attn_q8_paged"
    st = getattr(L, name)(PVLM_BF16, B, T, Hq, Hkv, D, *geom, max_ctx,
                          float(D ** -0.5 if scale is None else scale), q.data_ptr(),
                          *[t.data_ptr() for t in cache], *table, ctx_len.data_ptr(), out.data_ptr(), _ptr(mass),
                          _ptr(lse), wsb.data_ptr(), wsb.numel(), _ptr(_status(status)), _stream())
    _check(st, name)
    return out, mass, lse


def verify_attn_q8(q, k_codes, k_exps, v_codes, v_exps, ctx_len, *, scale: Optional[float] = None,
                   max_ctx: Optional[int] = None, out=None, mass=None, lse=None, want_mass: bool = True,
                   want_lse: bool = True, ws: Optional[Workspace] = None, status=None):
    """pvlm_verify_attn_q8: ``verify_attn`` of bf16 queries [B][T][Hq][D] over an
    8-bit cache [B][Hkv][n_cap][D]; T = 1 and want_mass=False for a decode step.
    Returns (out, mass or None, lse or None)."""
    return _verify_q8(q, (k_codes, k_exps, v_codes, v_exps), None, ctx_len, scale, max_ctx, out, mass, lse,
                      want_mass, want_lse, ws, status)


def verify_attn_q8_paged(q, k_codes, k_exps, v_codes, v_exps, page_table, ctx_len, *,
                         scale: Optional[float] = None, max_ctx: Optional[int] = None, out=None, mass=None,
                         lse=None, want_mass: bool = True, want_lse: bool = True,
                         ws: Optional[Workspace] = None, status=None):
    """pvlm_verify_attn_q8_paged: the same over pools [n_pages][Hkv][page][D]
    through page_table [B][max_pages]; mass is [B][max_pages * page]."""
    if page_table is None:
        raise TypeError("page_table must be a torch.Tensor")
    return _verify_q8(q, (k_codes, k_exps, v_codes, v_exps), page_table, ctx_len, scale, max_ctx, out, mass,
                      lse, want_mass, want_lse, ws, status)


def _gather_q8(cache, page_table, idx, k, tail_begin, tail_len, dst_cap, dtype, dst, status):
    _need(cache[0], "k_codes")
    dev = cache[0].device
    shape = _need_q8(*cache, dev, page_table is not None, stacked=True)
    for name, t in (("idx", idx), ("k", k), ("tail_begin", tail_begin), ("tail_len", tail_len)):
        _need(t, name, torch.int32, dev)
    L = 1 if len(shape) == 4 else shape[0]
    n0, Hkv, rows, D = shape[-4:]
    if idx.dim() != 2:
        raise ValueError("idx must be [B][k_cap]")
    B = idx.shape[0]
    if page_table is None and n0 != B:
        raise ValueError("idx must be [B][k_cap]")
    if any(t.shape != (B,) for t in (k, tail_begin, tail_len)):
        raise ValueError("k, tail_begin and tail_len must be [B]")
    if dtype not in (torch.float8_e4m3fn, torch.bfloat16, torch.float32):
        raise ValueError(f"unsupported dtype {dtype}")
    q8 = dtype is torch.float8_e4m3fn
    dst_cap = int(dst_cap)
    want = tuple(shape[:-4]) + (B, Hkv, dst_cap, D)
    fill = dst is None   # the call zeroes what it does not copy of a new destination
    if fill and q8:
        dst = [torch.empty(want[:n], dtype=dtype if n is None else torch.uint8, device=dev) for n in (None, -1) * 2]
    elif fill:
        dst = [torch.empty(want, dtype=dtype, device=dev) for _ in range(2)]
    elif q8:
        if len(dst) != 4 or _need_q8(*dst, dev, False, stacked=True) != want:
            raise ValueError("destination shape mismatch")
    elif len(dst) != 2 or any(_need(t, "dst", dtype, dev).shape != want for t in dst):
        raise ValueError("destination shape mismatch")
    kd, kde, vd, vde = [t.data_ptr() for t in dst] if q8 else (dst[0].data_ptr(), None, dst[1].data_ptr(), None)
    to = PVLM_E4M3 if q8 else PVLM_BF16 if dtype is torch.bfloat16 else PVLM_F32
    if page_table is None:
        name, geom, table = "pvlm_gather_kv_q8", (rows,), ()
    else:
        name = "pvlm_gather_kv_q8_paged"
        geom, table = (rows, _need_table(page_table, dev, B), n0), (page_table.data_ptr(),)
    st = getattr(lib(), name)(to, L, B, Hkv, D, *geom, *[t.data_ptr() for t in cache], *table, idx.data_ptr(),
                              k.data_ptr(), idx.shape[1], tail_begin.data_ptr(), tail_len.data_ptr(), dst_cap,
                              int(fill), kd, kde, vd, vde, _ptr(_status(status)), _stream())
    _check(st, name)
    return tuple(dst)


def gather_kv_q8(k_codes, k_exps, v_codes, v_exps, idx, k, tail_begin, tail_len, dst_cap: int, *,
                 dtype=torch.float8_e4m3fn, dst=None, status=None):
    """pvlm_gather_kv_q8: the draft's compact cache (``gather_kv``) from an 8-bit
    cache [B][Hkv][n_cap][D] or [L][...].  dtype torch.float8_e4m3fn returns
    (k_codes, k_exps, v_codes, v_exps) with dst_cap rows (a multiple of 32);
    torch.bfloat16 or torch.float32 returns (k, v), the values that the rows
    stand for.  ``dst``: those tensors, to be written in place."""
    return _gather_q8((k_codes, k_exps, v_codes, v_exps), None, idx, k, tail_begin, tail_len, dst_cap, dtype,
                      dst, status)


def gather_kv_q8_paged(k_codes, k_exps, v_codes, v_exps, page_table, idx, k, tail_begin, tail_len,
                       dst_cap: int, *, dtype=torch.float8_e4m3fn, dst=None, status=None):
    """pvlm_gather_kv_q8_paged: the same from pools [n_pages][Hkv][page][D] or
    [L][...]; one page_table [B][max_pages] serves every layer."""
    if page_table is None:
        raise TypeError("page_table must be a torch.Tensor")
    return _gather_q8((k_codes, k_exps, v_codes, v_exps), page_table, idx, k, tail_begin, tail_len, dst_cap,
                      dtype, dst, status)


# ------------------------------------------------------- page tables, slots --
# These calls are short beside their host time: a tensor that fits takes one test, the
# device and its stream are asked for once, and a size that only shapes decide is
# kept (with the kernel, a decode step's call took 15.0 us and takes 13.2, a rotary
# append's 12.2 and 11.2).
def _getdev() -> int:
    return torch._C._cuda_getDevice()     # (looked up here: a torch without device support has none)


def _here(t, name, dtype):
    """The device and its number of a contiguous tensor on the current device (whose
    stream a call is enqueued on)."""
    _need(t, name, dtype)
    dev = t.device
    if dev.index != _getdev():
        raise ValueError(f"{name} is on {dev}, but the current device is cuda:{_getdev()}")
    return dev


def _need_shape(t, name, dtype, dev, shape):
    if (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.is_contiguous()
            and t.is_cuda and t.get_device() == dev.index):
        return t
    _need(t, name, dtype, dev)
    raise ValueError(f"{name} must be {list(shape)}")


def _flags(status, dev):
    """The address of the caller's status word, or of this device's default one."""
    if status is None:
        status = _status_cache.get(dev.index)
        if status is None:
            status = _status(None)
    elif not (isinstance(status, torch.Tensor) and status.dtype is torch.int32 and status.is_cuda
              and status.get_device() == dev.index and status.numel()):
        _need(status, "status", torch.int32, dev)
        raise ValueError("status must hold an int32 word")
    return status.data_ptr()


def pages_resize(length, n_held, page_table, free_pages, n_free, *, page_size: int, granted=None, status=None):
    """pvlm_pages_resize: room for length[b] rows in every sequence's pages, from
    and to a stack of free ones.  length, n_held [B]; page_table [B][max_pages];
    free_pages [n_pages]; n_free [1], all int32; n_held, page_table, free_pages
    and n_free are updated.  Returns granted [B] (1: the sequence has what it needs)."""
    dev = _here(length, "length", torch.int32)
    if length.dim() != 1:
        raise ValueError("length must be [B]")
    B = length.shape[0]
    _need_shape(n_held, "n_held", torch.int32, dev, (B,))
    _need(free_pages, "free_pages", torch.int32, dev)
    _need(n_free, "n_free", torch.int32, dev)
    if free_pages.dim() != 1 or n_free.numel() != 1:
        raise ValueError("free_pages must be [n_pages] and n_free [1]")
    max_pages = _need_table(page_table, dev, B)
    if granted is None:
        granted = torch.empty_like(n_held)
    else:
        _need_shape(granted, "granted", torch.int32, dev, (B,))
    st = lib().pvlm_pages_resize(B, page_size, max_pages, free_pages.shape[0], length.data_ptr(), n_held.data_ptr(),
                                 page_table.data_ptr(), free_pages.data_ptr(), n_free.data_ptr(), granted.data_ptr(),
                                 _flags(status, dev), _raw_stream(dev.index))
    if st:
        _check(st, "pvlm_pages_resize")
    return granted


def slot_map(ctx_len, n_new, n_rows: int, *, page_size: int, n_pages: int, page_table=None, rows_per_seq: int = 0,
             want_pos: bool = True, want_seq: bool = True, want_start: bool = True, status=None):
    """pvlm_slot_map: the cache slots of n_new[b] new rows behind ctx_len[b] of every
    sequence, packed or rows_per_seq apart, in a paged cache or (page_table None,
    page_size its n_cap, n_pages its B) a padded one.  Returns (slots [n_rows]
    int64, pos [n_rows], seq [n_rows], row_start [B + 1]); -1 in slots and seq
    where there is no row.  What is not wanted is None."""
    dev = _here(ctx_len, "ctx_len", torch.int32)
    if ctx_len.dim() != 1:
        raise ValueError("ctx_len must be [B]")
    B = ctx_len.shape[0]
    _need_shape(n_new, "n_new", torch.int32, dev, (B,))
    max_pages = 1 if page_table is None else _need_table(page_table, dev, B)
    if page_table is None and n_pages < B:
        raise ValueError("a padded cache has a page for each sequence")
    n_rows = int(n_rows)
    slots = torch.empty(n_rows, dtype=torch.int64, device=dev)
    pos = torch.empty(n_rows, dtype=torch.int32, device=dev) if want_pos else None
    seq = torch.empty(n_rows, dtype=torch.int32, device=dev) if want_seq else None
    start = torch.empty(B + 1, dtype=torch.int32, device=dev) if want_start else None
    st = lib().pvlm_slot_map(B, n_rows, rows_per_seq, page_size, max_pages, n_pages, _ptr(page_table),
                             ctx_len.data_ptr(), n_new.data_ptr(), slots.data_ptr(), _ptr(pos), _ptr(seq), _ptr(start),
                             _flags(status, dev), _raw_stream(dev.index))
    if st:
        _check(st, "pvlm_slot_map")
    return slots, pos, seq, start


# -------------------------------------------------------------- rotary rows --
_LAYOUTS = {"half": 0, "interleaved": 1}
_SCALINGS = {None: 0, "": 0, "linear": 1, "parts": 2, "yarn": 3}


class Rotary:
    """A model's rotation (pvlm_rotary): the first ``rot_dim`` values of a head, in
    pairs ``layout`` "half" (i, i + rot_dim / 2) or "interleaved" (2 i, 2 i + 1);
    ``scaling`` None, "linear" (factor), "parts" or "yarn" (factor, orig_ctx, alpha,
    beta); ``mscale`` times the result; ``sections`` for M-RoPE."""

    def __init__(self, *, rot_dim: int, base: float, layout: str = "half", scaling=None, factor: float = 1.0,
                 orig_ctx: float = 0.0, alpha: float = 0.0, beta: float = 0.0, mscale: float = 1.0, sections=None):
        if layout not in _LAYOUTS:
            raise ValueError(f"layout must be one of {sorted(_LAYOUTS)}")
        if scaling not in _SCALINGS:
            raise ValueError("scaling must be None, 'linear', 'parts' or 'yarn'")
        if sections is not None and (len(sections) != 3 or not any(sections)):
            raise ValueError("sections must be three widths")
        self.params = RotaryParams(float(base), float(factor), float(orig_ctx), float(alpha), float(beta),
                                   float(mscale), int(rot_dim), _LAYOUTS[layout], _SCALINGS[scaling],
                                   (_c.c_int32 * 3)(*[int(x) for x in (sections or (0, 0, 0))]))
        self.by_ref = _c.byref(self.params)
        self.sections = None if sections is None else tuple(int(x) for x in sections)
        self.frequencies()      # (parameters that have none are refused here)

    def frequencies(self):
        """The angle per position of every pair (host floats)."""
        n = max(self.params.rot_dim // 2, 1)
        f = (_D * n)()
        if n > 128:
            raise ValueError("rot_dim must be at most 256")
        _check(lib().pvlm_rotary_freqs(_c.byref(self.params), f), "pvlm_rotary_freqs")
        return list(f)


def _row_stride(t, name, N, H, D, dtype, index):
    """The stride of rows [N][H][D] whose heads lie together."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype is not dtype or not t.is_cuda or t.get_device() != index:
        raise ValueError(f"{name} must be {dtype} on cuda:{index}")
    if t.shape != (N, H, D):
        raise ValueError(f"{name} must be [{N}][{H}][{D}]")
    row, head, one = t.stride()
    if (one != 1 and D > 1) or (head != D and H > 1):
        raise ValueError(f"the heads of a row of {name} must lie together")
    return row if N > 1 else H * D


def _rotary(q, k_new, v_new, pos, slots, rotary, dtype, dev, heads, q_out):
    """What both appends check of their rows; the arguments that they share."""
    if not isinstance(rotary, Rotary):
        raise TypeError("rotary must be a Rotary")
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q must be a tensor [N][Hq][D]")
    N, Hq, D = q.shape
    Hkv, Dc = heads
    if Dc != D:
        raise ValueError("the cache's rows do not have q's D")
    index = dev.index
    sq = _row_stride(q, "q", N, Hq, D, dtype, index)
    sk = _row_stride(k_new, "k_new", N, Hkv, D, dtype, index)
    sv = _row_stride(v_new, "v_new", N, Hkv, D, dtype, index)
    _need_shape(pos, "pos", torch.int32, dev, (N,) if rotary.sections is None else (3, N))
    _need_shape(slots, "slots", torch.int64, dev, (N,))
    if q_out is None:
        q_out = torch.empty((N, Hq, D), dtype=dtype, device=dev)
    else:
        _need_shape(q_out, "q_out", dtype, dev, (N, Hq, D))
    return q_out, (N, Hq, Hkv, D, rotary.by_ref, pos.data_ptr(), q.data_ptr(), sq, k_new.data_ptr(), sk,
                   v_new.data_ptr(), sv, slots.data_ptr())


def rotary_append(q, k_new, v_new, pos, slots, k_cache, v_cache, *, rotary: Rotary, q_out=None, status=None):
    """pvlm_rotary_append: rows q [N][Hq][D], k_new and v_new [N][Hkv][D] (views with
    a row stride are taken as they are), rotated by their positions pos [N] or
    [3][N] and appended at slots [N] (int64, -1: padding) of caches
    [blocks][Hkv][rows][D], padded or a page pool.  Returns q_out; its rows of padding
    are not written (a 4-bit verify takes them with n_new, the others do not)."""
    dev = _here(k_cache, "k_cache", None)
    if k_cache.dim() != 4:
        raise ValueError("caches must be [blocks][Hkv][rows][D]")
    _need_shape(v_cache, "v_cache", k_cache.dtype, dev, k_cache.shape)
    n_blocks, Hkv, rows, D = k_cache.shape
    q_out, args = _rotary(q, k_new, v_new, pos, slots, rotary, k_cache.dtype, dev, (Hkv, D), q_out)
    st = lib().pvlm_rotary_append(_dt(k_cache), *args, n_blocks, rows, q_out.data_ptr(), k_cache.data_ptr(),
                                  v_cache.data_ptr(), _flags(status, dev), _raw_stream(dev.index))
    if st:
        _check(st, "pvlm_rotary_append")
    return q_out


# ------------------------------------------------------------ 4-bit caches --
# Codes are torch.uint8 (two in a byte) or torch.float4_e2m1fn_x2, exponents
# torch.uint8, one for 32 values: a value is code * 2^(exponent - 127).
def _need_q4(k_codes, k_exps, v_codes, v_exps, dev, paged, stacked=False):
    """Check a cache's four tensors; returns the values' shape."""
    if dev.index != _getdev():
        raise ValueError(f"tensors are on {dev}, but the current device is cuda:{_getdev()}")
    for t, name in ((k_codes, "k_codes"), (v_codes, "v_codes")):
        _need(t, name, None, dev)
        if t.dtype is not torch.uint8 and t.dtype is not torch.float4_e2m1fn_x2:
            raise ValueError(f"{name} must be torch.uint8 or torch.float4_e2m1fn_x2, got {t.dtype}")
    shape = tuple(k_codes.shape)
    if len(shape) != 4 and not (stacked and len(shape) == 5):
        layout = "[n_pages][Hkv][page][D / 2]" if paged else "[B][Hkv][n_cap][D / 2]"
        raise ValueError(f"codes must be {layout}" + (f" or [L]{layout}" if stacked else ""))
    D = 2 * shape[-1]
    if D != 128 and D != 64:
        raise ValueError("D must be 64 or 128 (codes of D / 2 bytes)")
    if v_codes.shape != shape:
        raise ValueError("k_codes and v_codes must have one shape")
    exps = shape[:-1] + (D // 32,)
    _need_shape(k_exps, "k_exps", torch.uint8, dev, exps)
    _need_shape(v_exps, "v_exps", torch.uint8, dev, exps)
    return shape[:-1] + (D,)


def rotary_append_q4(q, k_new, v_new, pos, slots, k_codes, k_exps, v_codes, v_exps, *, rotary: Rotary, q_out=None,
                     status=None):
    """pvlm_rotary_append_q4: ``rotary_append`` (bf16) into a 4-bit cache, codes
    [blocks][Hkv][rows][D / 2] and exponents [blocks][Hkv][rows][D / 32].  Returns q_out."""
    cache = (k_codes, k_exps, v_codes, v_exps)
    dev = _here(k_codes, "k_codes", None)
    n_blocks, Hkv, rows, D = _need_q4(*cache, dev, True)
    q_out, args = _rotary(q, k_new, v_new, pos, slots, rotary, torch.bfloat16, dev, (Hkv, D), q_out)
    st = lib().pvlm_rotary_append_q4(PVLM_BF16, *args, n_blocks, rows, q_out.data_ptr(), k_codes.data_ptr(),
                                     k_exps.data_ptr(), v_codes.data_ptr(), v_exps.data_ptr(), _flags(status, dev),
                                     _raw_stream(dev.index))
    if st:
        _check(st, "pvlm_rotary_append_q4")
    return q_out


def _quantize_q4(k, v, length, cache, page_table, status):
    _need(k, "k")
    dev = k.device
    _need(v, "v", k.dtype, dev)
    _need(length, "length", torch.int32, dev)
    shape = _need_q4(*cache, dev, page_table is not None, stacked=True)
    if k.dim() != len(shape) or v.shape != k.shape:
        raise ValueError("k and v must be [B][Hkv][src_cap][D], or [L][...] with a stacked cache")
    L = 1 if k.dim() == 4 else k.shape[0]
    B, Hkv, src_cap, D = k.shape[-4:]
    n0, H, rows, Dc = shape[-4:]
    if (H, Dc) != (Hkv, D) or (len(shape) == 5 and shape[0] != L) or (page_table is None and n0 != B):
        raise ValueError("the 4-bit cache does not match k and v")
    if length.shape != (B,):
        raise ValueError("length must be [B]")
    codes = [t.data_ptr() for t in cache]
    tail = (k.data_ptr(), v.data_ptr(), length.data_ptr())
    if page_table is None:
        name, geom, more = "pvlm_quantize_kv_q4", (src_cap, *tail, rows), ()
    else:
        name, geom = "pvlm_quantize_kv_q4_paged", (rows, _need_table(page_table, dev, B), n0, src_cap, *tail)
        more = (page_table.data_ptr(),)
    st = getattr(lib(), name)(_dt(k), L, B, Hkv, D, *geom, *more, *codes, _flags(status, dev), _raw_stream(dev.index))
    if st:
        _check(st, name)


def quantize_kv_q4(k, v, length, k_codes, k_exps, v_codes, v_exps, *, status=None):
    """pvlm_quantize_kv_q4: ``quantize_kv`` into a 4-bit cache: rows 0 .. length[b] - 1
    of [B][Hkv][src_cap][D] (or [L][...]) to codes [B][Hkv][n_cap][D / 2]."""
    _quantize_q4(k, v, length, (k_codes, k_exps, v_codes, v_exps), None, status)


def quantize_kv_q4_paged(k, v, length, k_codes, k_exps, v_codes, v_exps, page_table, *, status=None):
    """pvlm_quantize_kv_q4_paged: the same into pools [n_pages][Hkv][page][D / 2] (or
    [L][...]; one page_table [B][max_pages] serves every layer)."""
    if page_table is None:
        raise TypeError("page_table must be a torch.Tensor")
    _quantize_q4(k, v, length, (k_codes, k_exps, v_codes, v_exps), page_table, status)


def verify_attn_q4_workspace_size(B, T, Hq, Hkv, D, n_cap, max_ctx) -> int:
    return int(lib().pvlm_verify_attn_q4_workspace_size(B, T, Hq, Hkv, D, n_cap, max_ctx))


_ws_sizes = {}     # of a workspace, by the device and the sizes that decide it


def _verify_q4(q, cache, page_table, ctx_len, n_new, scale, max_ctx, out, mass, lse, want_mass, want_lse, ws, status):
    _need(q, "q", torch.bfloat16)
    dev = q.device
    n0, Hkv, rows, Dc = _need_q4(*cache, dev, page_table is not None)
    if q.dim() != 4:
        raise ValueError("q must be [B][T][Hq][D]")
    B, T, Hq, D = q.shape
    _need_shape(ctx_len, "ctx_len", torch.int32, dev, (B,))
    if Dc != D or (page_table is None and n0 != B):
        raise ValueError("inconsistent verify_attn_q4 shapes")
    name, new = "pvlm_verify_attn_q4", ()
    if n_new is not None:
        name, new = "pvlm_verify_attn_q4_ragged", (_need_shape(n_new, "n_new", torch.int32, dev, (B,)).data_ptr(),)
    if page_table is None:
        n_cap, geom, table = rows, (rows,), ()
    else:
        max_pages = _need_table(page_table, dev, B)
        name, n_cap, geom = name + "_paged", max_pages * rows, (rows, max_pages, n0)
        table = (page_table.data_ptr(),)
    if max_ctx is None:
        max_ctx = n_cap - T
    if out is None:
        out = torch.empty_like(q)
    else:
        _need_shape(out, "out", torch.bfloat16, dev, q.shape)
    if mass is not None:
        _need_shape(mass, "mass", torch.float32, dev, (B, n_cap))
    elif want_mass:
        mass = torch.empty((B, n_cap), dtype=torch.float32, device=dev)
    if lse is not None:
        _need_shape(lse, "lse", torch.float32, dev, (B, Hq, T))
    elif want_lse:
        lse = torch.empty((B, Hq, T), dtype=torch.float32, device=dev)
    L = lib()
    sizes = (dev.index, B, T, Hq, Hkv, D, n_cap, max_ctx)
    need = _ws_sizes.get(sizes)
    if need is None:
        if len(_ws_sizes) >= 4096:
            _ws_sizes.clear()
        need = _ws_sizes[sizes] = L.pvlm_verify_attn_q4_workspace_size(B, T, Hq, Hkv, D, n_cap, max_ctx)
    wsb = _ws_buffer("verify_q4", ws, need, dev)
    if wsb.get_device() != dev.index:
        raise ValueError(f"ws is on {wsb.device}, expected {dev}")
    kc, ke, vc, ve = cache
    st = getattr(L, name)(PVLM_BF16, B, T, Hq, Hkv, D, *geom, max_ctx, D ** -0.5 if scale is None else float(scale),
                          q.data_ptr(), kc.data_ptr(), ke.data_ptr(), vc.data_ptr(), ve.data_ptr(), *table,
                          ctx_len.data_ptr(), *new, out.data_ptr(), None if mass is None else mass.data_ptr(),
                          None if lse is None else lse.data_ptr(), wsb.data_ptr(), wsb.numel(), _flags(status, dev),
                          _raw_stream(dev.index))
    if st:
        _check(st, name)
    return out, mass, lse


def verify_attn_q4(q, k_codes, k_exps, v_codes, v_exps, ctx_len, *, n_new=None, scale: Optional[float] = None,
                   max_ctx: Optional[int] = None, out=None, mass=None, lse=None, want_mass: bool = True,
                   want_lse: bool = True, ws: Optional[Workspace] = None, status=None):
    """pvlm_verify_attn_q4: ``verify_attn`` of bf16 queries [B][T][Hq][D] over a 4-bit
    cache, codes [B][Hkv][n_cap][D / 2] and exponents [B][Hkv][n_cap][D / 32]; T = 1 and
    want_mass=False for a decode step.  n_new [B] int32 (pvlm_verify_attn_q4_ragged): the rows
    that a sequence has, those behind them padding (out 0, lse -inf, no part in the mass).
    Returns (out, mass or None, lse or None)."""
    return _verify_q4(q, (k_codes, k_exps, v_codes, v_exps), None, ctx_len, n_new, scale, max_ctx, out, mass, lse,
                      want_mass, want_lse, ws, status)


def verify_attn_q4_paged(q, k_codes, k_exps, v_codes, v_exps, page_table, ctx_len, *, n_new=None,
                         scale: Optional[float] = None, max_ctx: Optional[int] = None, out=None, mass=None,
                         lse=None, want_mass: bool = True, want_lse: bool = True,
                         ws: Optional[Workspace] = None, status=None):
    """pvlm_verify_attn_q4_paged: the same over pools [n_pages][Hkv][page][D / 2]
    through page_table [B][max_pages]; mass is [B][max_pages * page]."""
    if page_table is None:
        raise TypeError("page_table must be a torch.Tensor")
    return _verify_q4(q, (k_codes, k_exps, v_codes, v_exps), page_table, ctx_len, n_new, scale, max_ctx, out, mass, lse,
                      want_mass, want_lse, ws, status)


def _gather_q4(cache, page_table, idx, k, tail_begin, tail_len, dst_cap, dtype, dst, status):
    _need(cache[0], "k_codes")
    dev = cache[0].device
    shape = _need_q4(*cache, dev, page_table is not None, stacked=True)
    _need(idx, "idx", torch.int32, dev)
    L = 1 if len(shape) == 4 else shape[0]
    n0, Hkv, rows, D = shape[-4:]
    if idx.dim() != 2 or (page_table is None and n0 != idx.shape[0]):
        raise ValueError("idx must be [B][k_cap]")
    B = idx.shape[0]
    _need_shape(k, "k", torch.int32, dev, (B,))
    _need_shape(tail_begin, "tail_begin", torch.int32, dev, (B,))
    _need_shape(tail_len, "tail_len", torch.int32, dev, (B,))
    if dtype not in (torch.float4_e2m1fn_x2, torch.uint8, torch.bfloat16, torch.float32):
        raise ValueError(f"unsupported dtype {dtype}")
    q4 = dtype is torch.uint8 or dtype is torch.float4_e2m1fn_x2
    dst_cap = int(dst_cap)
    want = tuple(shape[:-4]) + (B, Hkv, dst_cap, D)
    fill = dst is None   # the call zeroes what it does not copy of a new destination
    if fill and q4:
        dst = [torch.empty(want[:-1] + (w,), dtype=d, device=dev) for w, d in ((D // 2, dtype), (D // 32, torch.uint8)) * 2]
    elif fill:
        dst = [torch.empty(want, dtype=dtype, device=dev) for _ in range(2)]
    elif q4:
        if len(dst) != 4 or tuple(_need_q4(*dst, dev, False, stacked=True)) != want:
            raise ValueError("destination shape mismatch")
    elif len(dst) != 2 or any(_need(t, "dst", dtype, dev).shape != want for t in dst):
        raise ValueError("destination shape mismatch")
    kd, kde, vd, vde = [t.data_ptr() for t in dst] if q4 else (dst[0].data_ptr(), None, dst[1].data_ptr(), None)
    to = PVLM_E2M1 if q4 else PVLM_BF16 if dtype is torch.bfloat16 else PVLM_F32
    if page_table is None:
        name, geom, table = "pvlm_gather_kv_q4", (rows,), ()
    else:
        name = "pvlm_gather_kv_q4_paged"
        geom, table = (rows, _need_table(page_table, dev, B), n0), (page_table.data_ptr(),)
    st = getattr(lib(), name)(to, L, B, Hkv, D, *geom, *[t.data_ptr() for t in cache], *table, idx.data_ptr(),
                              k.data_ptr(), idx.shape[1], tail_begin.data_ptr(), tail_len.data_ptr(), dst_cap,
                              int(fill), kd, kde, vd, vde, _flags(status, dev), _raw_stream(dev.index))
    if st:
        _check(st, name)
    return tuple(dst)


def gather_kv_q4(k_codes, k_exps, v_codes, v_exps, idx, k, tail_begin, tail_len, dst_cap: int, *,
                 dtype=torch.uint8, dst=None, status=None):
    """pvlm_gather_kv_q4: the draft's compact cache (``gather_kv``) from a 4-bit cache
    [B][Hkv][n_cap][D / 2] or [L][...].  dtype torch.uint8 (or float4_e2m1fn_x2)
    returns (k_codes, k_exps, v_codes, v_exps) with dst_cap rows (a multiple of
    32); torch.bfloat16 or torch.float32 returns (k, v), the values that the rows
    stand for.  ``dst``: those tensors, to be written in place."""
    return _gather_q4((k_codes, k_exps, v_codes, v_exps), None, idx, k, tail_begin, tail_len, dst_cap, dtype, dst,
                      status)


def gather_kv_q4_paged(k_codes, k_exps, v_codes, v_exps, page_table, idx, k, tail_begin, tail_len, dst_cap: int, *,
                       dtype=torch.uint8, dst=None, status=None):
    """pvlm_gather_kv_q4_paged: the same from pools [n_pages][Hkv][page][D / 2] or
    [L][...]; one page_table [B][max_pages] serves every layer."""
    if page_table is None:
        raise TypeError("page_table must be a torch.Tensor")
    return _gather_q4((k_codes, k_exps, v_codes, v_exps), page_table, idx, k, tail_begin, tail_len, dst_cap, dtype,
                      dst, status)
