"""Python binding of libe3.so: argument marshalling only.

Every function has the name and the arguments of the C entry point it calls
(include/e3.h).  Tensors are torch tensors used as device memory; the current
torch stream is handed over as the hipStream_t.  Nothing is computed here, and
there is no fallback: without the built library the import of `lib()` raises.
The calls that a step consists of go through _native (csrc/native_binding.cpp) as long as their
arguments are plain tensors, ints and floats of the right shape; everything else, errors above all,
is treated here.
"""
from __future__ import annotations

import ctypes as C
import importlib.machinery
import importlib.util
import os
from typing import NamedTuple, Optional, Tuple

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libe3.so")
NATIVE_PATH = os.path.join(HERE, "_native.so")

E3_F32, E3_BF16, E3_E4M3 = 0, 1, 2
E3_OK = 0
E3_ERR_SHAPE = -2
E3_TILE_CHUNK, E3_TILE_LANES, E3_TILE_DEPTH = 8, 64, 8
E3_NOALLOC_MAX_ROWS = 1024
E3_MAX_DRAFTS = 63
E3_MAX_AXES = 8
E3_MAX_BEAMS = 32
E3_MAX_KEEP = 64

EXPORTS = ("e3_strerror", "e3_workspace_bytes", "e3_sample_entropy", "e3_sample_entropy_noalloc",
           "e3_sample_restricted", "e3_sample_restricted_ws", "e3_restricted_workspace_bytes",
           "e3_logprob_entropy", "e3_logprob_entropy_advantages",
           "e3_grpo_advantages", "e3_temperature_update", "e3_difficulty_ranks",
           "e3_allocate_budgets", "e3_budget_bounds", "e3_logprob_entropy_gap",
           "e3_temperature_update_gap", "e3_grpo_objective", "e3_cache_append", "e3_cache_read",
           "e3_rotate", "e3_cache_append_rotated", "e3_window_attention", "e3_window_attention_workspace_bytes",
           "e3_beam_workspace_bytes", "e3_beam_select", "e3_beam_reorder", "e3_cache_copy",
           "e3_prefix_attention", "e3_prefix_attention_workspace_bytes", "e3_verify_drafts",
           "e3_verify_workspace_bytes", "e3_read_probe",
           "e3_time_next_launch", "e3_launch_plan", "e3_launch_plan_of")

_NATIVE_CALLS = ("e3_grpo_advantages", "e3_grpo_objective", "e3_workspace_bytes", "e3_sample_entropy",
                 "e3_restricted_workspace_bytes", "e3_sample_restricted_ws", "e3_logprob_entropy_advantages",
                 "e3_logprob_entropy_gap", "e3_temperature_update", "e3_cache_append", "e3_cache_read",
                 "e3_prefix_attention_workspace_bytes", "e3_prefix_attention", "e3_verify_workspace_bytes", "e3_verify_drafts",
                 "e3_rotate", "e3_cache_append_rotated", "e3_window_attention", "e3_window_attention_workspace_bytes",
                 "e3_beam_workspace_bytes", "e3_beam_select", "e3_beam_reorder", "e3_cache_copy")

_lib: Optional[C.CDLL] = None
_native = None                     # the native calls, once they are bound to the loaded library


# A call is one or two launches of a few microseconds, so what surrounds it counts: pointers go over as
# plain integers, the stream as torch's raw handle (no Stream object), and a check asks a tensor
# for as little as it can.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


class E3Error(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {e3_strerror(status)} (status {status})")


def lib() -> C.CDLL:
    """Load libe3.so (built in-tree by paper_2505_18573_amd/build.py)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: run `python -m paper_2505_18573_amd.build` "
                              "(there is no fallback path)")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, u64, f32, f64 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64, C.c_float, C.c_double
        L.e3_strerror.argtypes = [C.c_int]
        L.e3_strerror.restype = C.c_char_p
        L.e3_workspace_bytes.argtypes = [i64, i64]
        L.e3_workspace_bytes.restype = C.c_size_t
        L.e3_sample_entropy.argtypes = [vp, C.c_int, i64, i64, i64, vp, f32, u64, u64,
                                        vp, vp, vp, vp, C.c_size_t, vp]
        L.e3_sample_entropy.restype = C.c_int
        L.e3_sample_entropy_noalloc.argtypes = [vp, C.c_int, i64, i64, i64, vp, f32, u64, u64, vp, vp, vp, vp]
        L.e3_sample_entropy_noalloc.restype = C.c_int
        L.e3_sample_restricted.argtypes = [vp, C.c_int, i64, i64, i64, vp, f32, i32, f32, u64, u64,
                                           vp, vp, vp, vp]
        L.e3_sample_restricted.restype = C.c_int
        L.e3_sample_restricted_ws.argtypes = [vp, C.c_int, i64, i64, i64, vp, f32, i32, f32, u64, u64,
                                              vp, vp, vp, vp, C.c_size_t, vp]
        L.e3_sample_restricted_ws.restype = C.c_int
        L.e3_restricted_workspace_bytes.argtypes = [C.c_int, i64, i64, i32]
        L.e3_restricted_workspace_bytes.restype = C.c_size_t
        L.e3_time_next_launch.argtypes = [vp, vp]
        L.e3_time_next_launch.restype = C.c_int
        L.e3_launch_plan.argtypes = [i64, i64, C.c_int, vp, vp, vp, vp]
        L.e3_launch_plan.restype = C.c_int
        L.e3_launch_plan_of.argtypes = [i64, i64, C.c_int, C.c_int, vp, vp, vp, vp]
        L.e3_launch_plan_of.restype = C.c_int
        L.e3_read_probe.argtypes = [vp, i64, vp, vp]
        L.e3_read_probe.restype = C.c_int
        L.e3_logprob_entropy.argtypes = [vp, C.c_int, i64, i64, i64, vp, vp, vp, f32,
                                         vp, vp, vp, vp, vp, C.c_size_t, vp]
        L.e3_logprob_entropy.restype = C.c_int
        L.e3_logprob_entropy_advantages.argtypes = [vp, C.c_int, i64, i64, i64, vp, vp, vp, f32,
                                                    vp, vp, vp, vp, vp, vp, i32, i32, f32, vp,
                                                    vp, C.c_size_t, vp]
        L.e3_logprob_entropy_advantages.restype = C.c_int
        L.e3_logprob_entropy_gap.argtypes = [vp, C.c_int, i64, i64, i64, vp, vp, vp, f32,
                                             vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
        L.e3_logprob_entropy_gap.restype = C.c_int
        L.e3_temperature_update_gap.argtypes = [f64, f64, f64, f64, i64, i64, i64, f64, f64, f64, vp, vp]
        L.e3_temperature_update_gap.restype = C.c_int
        L.e3_grpo_objective.argtypes = [vp, vp, vp, vp, i32, vp, i32, f32, vp, vp, vp, vp]
        L.e3_grpo_objective.restype = C.c_int
        L.e3_grpo_advantages.argtypes = [vp, vp, i32, i32, f32, vp, vp]
        L.e3_grpo_advantages.restype = C.c_int
        L.e3_temperature_update.argtypes = [f64, f64, f64, i64, i64, i64, i64, f64, f64, f64, vp, vp]
        L.e3_temperature_update.restype = C.c_int
        L.e3_difficulty_ranks.argtypes = [vp, vp, i64, vp]
        L.e3_difficulty_ranks.restype = C.c_int
        L.e3_allocate_budgets.argtypes = [vp, i32, i32, i32, i32, vp, vp]
        L.e3_allocate_budgets.restype = C.c_int
        L.e3_budget_bounds.argtypes = [i32, i32, i32, i32, i32, vp, vp]
        L.e3_budget_bounds.restype = C.c_int
        L.e3_cache_append.argtypes = [vp, vp, vp, C.c_int, i64, i64, i64, i64, i64, vp, vp]
        L.e3_cache_append.restype = C.c_int
        L.e3_cache_read.argtypes = [vp, vp, i64, vp, vp, C.c_int, vp]
        L.e3_cache_read.restype = C.c_int
        L.e3_prefix_attention_workspace_bytes.argtypes = [i64] * 6
        L.e3_prefix_attention_workspace_bytes.restype = C.c_size_t
        L.e3_prefix_attention.argtypes = [vp, vp, i64, i64, i64, i64, i64, i64, vp, i64, vp, i64, vp, vp, i64, vp, f32,
                                          vp, vp, vp, C.c_size_t, vp]
        L.e3_prefix_attention.restype = C.c_int
        L.e3_verify_workspace_bytes.argtypes = [i64, i32, i64]
        L.e3_verify_workspace_bytes.restype = C.c_size_t
        L.e3_verify_drafts.argtypes = [vp, C.c_int, i64, i32, i64, i64, i64, vp, vp, vp, i64, i64, vp, f32, vp, u64, u64,
                                       vp, vp, vp, vp, vp, C.c_size_t, vp]
        L.e3_verify_drafts.restype = C.c_int
        L.e3_rotate.argtypes = [vp, vp, i64, vp, C.c_int, i64, i64, i64, i64, i64, vp, i64, i64, C.c_int, vp]
        L.e3_rotate.restype = C.c_int
        L.e3_cache_append_rotated.argtypes = [vp, vp, vp, i64, vp, vp, vp, C.c_int, i64, i64, i64, i64, i64, i64, i64, i64, vp, vp, i64, i64, vp]
        L.e3_cache_append_rotated.restype = C.c_int
        L.e3_window_attention_workspace_bytes.argtypes = [i64] * 5
        L.e3_window_attention_workspace_bytes.restype = C.c_size_t
        L.e3_window_attention.argtypes = [vp, vp, i64, i64, i64, i64, vp, i64, vp, i64, vp, i64, i64, f32, vp, vp, vp, C.c_size_t, vp]
        L.e3_window_attention.restype = C.c_int
        L.e3_beam_workspace_bytes.argtypes = [i64, i32, i64]
        L.e3_beam_workspace_bytes.restype = C.c_size_t
        L.e3_beam_select.argtypes = [vp, C.c_int, i64, i32, i64, i64, i64, vp, i32, f32, vp, i32, vp, vp, vp, vp, C.c_size_t, vp]
        L.e3_beam_select.restype = C.c_int
        L.e3_beam_reorder.argtypes = [vp, i64, i32, vp, i64, vp, i32, vp, vp, vp, vp, vp, vp]
        L.e3_beam_reorder.restype = C.c_int
        L.e3_cache_copy.argtypes = [vp, vp, vp, vp, i64, vp]
        L.e3_cache_copy.restype = C.c_int
        _bind_native(L)                           # may raise: nothing is loaded then
        _lib = L
    return _lib


def _bind_native(L: C.CDLL) -> None:
    """Loads the native calls (built beside the library) and points them at L's entry points."""
    global _native
    if _raw_stream is None:                       # a torch without the raw stream handle: no native calls
        return
    if not os.path.exists(NATIVE_PATH):
        raise ImportError(f"{NATIVE_PATH} is missing: run `python -m paper_2505_18573_amd.build`")
    loader = importlib.machinery.ExtensionFileLoader("_native", NATIVE_PATH)
    module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_native", loader))
    loader.exec_module(module)
    module.bind({n: C.cast(getattr(L, n), C.c_void_p).value for n in _NATIVE_CALLS}, _raw_stream)
    _native = module


def _ordinary(name: str, *args):
    """The outputs of native call `name` (of the entry point e3_...), or None if its arguments are not ordinary."""
    if _lib is None:
        lib()
    if _native is None:
        return None
    out = getattr(_native, name)(*args)
    if type(out) is int:
        raise E3Error(out, _ENTRY[name])
    return out


_ENTRY = {"advantages": "e3_grpo_advantages", "objective": "e3_grpo_objective", "sample": "e3_sample_entropy",
          "restricted": "e3_sample_restricted", "logprob": "e3_logprob_entropy",
          "logprob_advantages": "e3_logprob_entropy_advantages", "logprob_gap": "e3_logprob_entropy_gap",
          "temperature": "e3_temperature_update", "cache_append": "e3_cache_append", "cache_read": "e3_cache_read",
          "attention": "e3_prefix_attention", "verify": "e3_verify_drafts", "rotate": "e3_rotate",
          "append_rotated": "e3_cache_append_rotated", "window": "e3_window_attention",
          "beam_select": "e3_beam_select", "beam_reorder": "e3_beam_reorder", "cache_copy": "e3_cache_copy"}


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream(device) -> int:
    if _raw_stream is not None and device.index is not None:
        return _raw_stream(device.index)
    return torch.cuda.current_stream(device).cuda_stream


def _logits_meta(logits: torch.Tensor) -> Tuple[int, int, int, int]:
    shape = logits.shape
    if len(shape) != 2:
        raise ValueError("logits must be [rows, V] with unit column stride")
    rows, V = shape
    pitch, step = logits.stride()
    if V > 1 and step != 1:
        raise ValueError("logits must be [rows, V] with unit column stride")
    if not logits.is_cuda:
        raise ValueError("logits must live on the GPU")
    dtype = logits.dtype
    if dtype is torch.bfloat16:
        dt = E3_BF16
    elif dtype is torch.float32:
        dt = E3_F32
    else:
        raise TypeError(f"unsupported logit dtype {dtype}")
    return dt, rows, V, pitch if rows > 1 else max(V, pitch)


def _check(t: Optional[torch.Tensor], dtype, n: int, name: str, device):
    if t is None:
        return
    if t.dtype is not dtype or t.dim() != 1 or t.numel() != n or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of {n} elements on {device}")


def _check_scalar_out(t: Optional[torch.Tensor], dtype, name: str, device):
    """A one-element output that one thread stores once: device memory, or pinned host
    memory (which the device addresses through the same pointer)."""
    if t is not None and t.device.type == "cpu":
        if not t.is_pinned():
            raise ValueError(f"{name}: a host tensor must be pinned")
        device = t.device
    _check(t, dtype, 1, name, device)


def e3_strerror(status: int) -> str:
    return lib().e3_strerror(int(status)).decode()


def e3_workspace_bytes(rows: int, V: int) -> int:
    return int(lib().e3_workspace_bytes(rows, V))


def e3_restricted_workspace_bytes(dtype: int, rows: int, V: int, top_k: int) -> int:
    """Host-only.  dtype: E3_BF16 or E3_F32.  0: e3_sample_restricted has no use for a workspace."""
    return int(lib().e3_restricted_workspace_bytes(dtype, rows, V, top_k))


def new_workspace(rows: int, V: int, device) -> Optional[torch.Tensor]:
    """Allocate a workspace for a [rows, V] problem (None when none is needed)."""
    need = e3_workspace_bytes(rows, V)
    if need == 0:
        return None
    return torch.empty((need + 3) // 4, dtype=torch.int32, device=device)


def _workspace(rows: int, V: int, workspace, device):
    """workspace: a tensor to use, None to allocate one of e3_workspace_bytes(), or False to
    pass NULL (every row then stays in one workgroup)."""
    if workspace is False:
        return None, 0
    if workspace is None:
        workspace = new_workspace(rows, V, device)
    if workspace is None:
        return None, 0
    return workspace, workspace.numel() * workspace.element_size()


def e3_sample_entropy(logits: torch.Tensor, tau_rows: Optional[torch.Tensor], tau_scalar: float,
                      seed: int, row_base: int = 0,
                      token_out: Optional[torch.Tensor] = None,
                      logp_out: Optional[torch.Tensor] = None,
                      entropy_out: Optional[torch.Tensor] = None,
                      workspace=None):
    """Returns (token int32 [rows], logp fp32 [rows], entropy fp32 [rows])."""
    out = _ordinary("sample", logits, tau_rows, tau_scalar, seed, row_base, token_out, logp_out, entropy_out, workspace)
    if out is not None:
        return out
    dt, rows, V, stride = _logits_meta(logits)
    dev = logits.device
    if token_out is None:
        token_out = torch.empty(rows, dtype=torch.int32, device=dev)
    else:
        _check(token_out, torch.int32, rows, "token_out", dev)
    if logp_out is None:
        logp_out = torch.empty(rows, dtype=torch.float32, device=dev)
    else:
        _check(logp_out, torch.float32, rows, "logp_out", dev)
    if entropy_out is None:
        entropy_out = torch.empty(rows, dtype=torch.float32, device=dev)
    else:
        _check(entropy_out, torch.float32, rows, "entropy_out", dev)
    _check(tau_rows, torch.float32, rows, "tau_rows", dev)
    ws, ws_bytes = _workspace(rows, V, workspace, dev)
    rc = lib().e3_sample_entropy(_ptr(logits), dt, rows, V, stride, _ptr(tau_rows),
                                 float(tau_scalar), int(seed), int(row_base),
                                 _ptr(token_out), _ptr(logp_out), _ptr(entropy_out),
                                 _ptr(ws), ws_bytes, _stream(dev))
    if rc != E3_OK:
        raise E3Error(rc, "e3_sample_entropy")
    return token_out, logp_out, entropy_out


def e3_sample_entropy_noalloc(logits: torch.Tensor, tau_rows: Optional[torch.Tensor], tau_scalar: float,
                              seed: int, row_base: int, token_out: torch.Tensor,
                              logp_out: Optional[torch.Tensor], entropy_out: Optional[torch.Tensor]):
    """The allocation-free entry point: the caller passes every output (nothing is allocated
    here either).  Returns (token_out, logp_out, entropy_out)."""
    dt, rows, V, stride = _logits_meta(logits)
    dev = logits.device
    _check(tau_rows, torch.float32, rows, "tau_rows", dev)
    _check(token_out, torch.int32, rows, "token_out", dev)
    _check(logp_out, torch.float32, rows, "logp_out", dev)
    _check(entropy_out, torch.float32, rows, "entropy_out", dev)
    rc = lib().e3_sample_entropy_noalloc(_ptr(logits), dt, rows, V, stride, _ptr(tau_rows),
                                         float(tau_scalar), int(seed), int(row_base),
                                         _ptr(token_out), _ptr(logp_out), _ptr(entropy_out), _stream(dev))
    if rc != E3_OK:
        raise E3Error(rc, "e3_sample_entropy_noalloc")
    return token_out, logp_out, entropy_out


def e3_sample_restricted(logits: torch.Tensor, tau_rows: Optional[torch.Tensor], tau_scalar: float,
                         top_k: int, top_p: float, seed: int, row_base: int = 0,
                         token_out: Optional[torch.Tensor] = None,
                         logp_out: Optional[torch.Tensor] = None,
                         kept_out: Optional[torch.Tensor] = None,
                         workspace=None):
    """Returns (token int32 [rows], logp fp32 [rows], kept int32 [rows]).  bf16 rows: any
    top_k / top_p; fp32 rows: 1 <= top_k <= 256 (E3_ERR_VALUE otherwise).

    workspace: a tensor of e3_restricted_workspace_bytes() to use, with which few wide rows are spread over
    workgroups, or False for none (a row then stays in one workgroup).  None: a call that allocates outputs allocates it
    too, if there is memory; a call that is given all of its outputs allocates nothing."""
    out = _ordinary("restricted", logits, tau_rows, tau_scalar, top_k, top_p, seed, row_base, token_out, logp_out, kept_out,
                    workspace)
    if out is not None:
        return out
    dt, rows, V, stride = _logits_meta(logits)
    dev = logits.device
    may_allocate = token_out is None or logp_out is None or kept_out is None
    if token_out is None:
        token_out = torch.empty(rows, dtype=torch.int32, device=dev)
    else:
        _check(token_out, torch.int32, rows, "token_out", dev)
    if logp_out is None:
        logp_out = torch.empty(rows, dtype=torch.float32, device=dev)
    else:
        _check(logp_out, torch.float32, rows, "logp_out", dev)
    if kept_out is None:
        kept_out = torch.empty(rows, dtype=torch.int32, device=dev)
    else:
        _check(kept_out, torch.int32, rows, "kept_out", dev)
    _check(tau_rows, torch.float32, rows, "tau_rows", dev)
    L, top_k = lib(), int(top_k)
    if workspace is None and may_allocate:
        need = L.e3_restricted_workspace_bytes(dt, rows, V, top_k)
        try:
            workspace = torch.empty(need, dtype=torch.uint8, device=dev) if need else False
        except torch.OutOfMemoryError:
            workspace = False
    elif workspace is None:
        workspace = False
    elif workspace is not False and (workspace.device != dev or not workspace.is_contiguous()):
        raise ValueError(f"workspace must be a contiguous tensor on {dev}")
    ws, ws_bytes = _workspace(rows, V, workspace, dev)
    rc = L.e3_sample_restricted_ws(_ptr(logits), dt, rows, V, stride, _ptr(tau_rows),
                                   float(tau_scalar), top_k, float(top_p), int(seed),
                                   int(row_base), _ptr(token_out), _ptr(logp_out), _ptr(kept_out),
                                   _ptr(ws), ws_bytes, _stream(dev))
    if rc != E3_OK:
        raise E3Error(rc, "e3_sample_restricted")
    return token_out, logp_out, kept_out


E3_READ_PROBE_SUMS = 2048


def e3_time_next_launch(start_event: Optional[int], stop_event: Optional[int]) -> None:
    """start_event / stop_event: hipEvent_t handles as integers (or None)."""
    lib().e3_time_next_launch(C.c_void_p(start_event), C.c_void_p(stop_event))


def e3_launch_plan(rows: int, V: int, sample: bool = True, dtype: torch.dtype = torch.bfloat16) -> Tuple[bool, int, int, int]:
    """Host-only: how a [rows, V] batch is launched: (cut, if the caller brings the workspace for it;
    waves and rows per workgroup and number of workgroups of the launch of whole rows)."""
    cut, waves, rows_per_group, workgroups = C.c_int32(), C.c_int32(), C.c_int32(), C.c_int64()
    rc = lib().e3_launch_plan_of(rows, V, {torch.bfloat16: E3_BF16, torch.float32: E3_F32}[dtype], int(sample), C.byref(cut), C.byref(waves), C.byref(rows_per_group),
                                 C.byref(workgroups))
    if rc != E3_OK:
        raise E3Error(rc, "e3_launch_plan")
    return bool(cut.value), waves.value, rows_per_group.value, workgroups.value


def e3_read_probe(buf: torch.Tensor, sums_out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Reads the (contiguous) tensor once; returns the E3_READ_PROBE_SUMS xor checksums (int32)."""
    if not buf.is_cuda or not buf.is_contiguous():
        raise ValueError("buf must be a contiguous GPU tensor")
    dev = buf.device
    if sums_out is None:
        sums_out = torch.empty(E3_READ_PROBE_SUMS, dtype=torch.int32, device=dev)
    _check(sums_out, torch.int32, E3_READ_PROBE_SUMS, "sums_out", dev)
    rc = lib().e3_read_probe(_ptr(buf), buf.numel() * buf.element_size(), _ptr(sums_out), _stream(dev))
    if rc != E3_OK:
        raise E3Error(rc, "e3_read_probe")
    return sums_out


def e3_logprob_entropy(logits: torch.Tensor, target_ids: Optional[torch.Tensor],
                       row_mask: Optional[torch.Tensor], tau_rows: Optional[torch.Tensor],
                       tau_scalar: float,
                       logp_out: Optional[torch.Tensor] = None,
                       entropy_out: Optional[torch.Tensor] = None,
                       entropy_sum_out: Optional[torch.Tensor] = None,
                       entropy_count_out: Optional[torch.Tensor] = None,
                       workspace=None, want_sum: bool = True):
    """Returns (logp fp32 [rows] or None, entropy fp32 [rows], entropy_sum fp64 [1] or None,
    entropy_count int64 [1] or None); the sum and count stay on the device unless pinned host
    tensors are passed for them."""
    out = _ordinary("logprob", logits, target_ids, row_mask, tau_rows, tau_scalar, None, None, 0, 0.0, logp_out,
                    entropy_out, entropy_sum_out, entropy_count_out, None, workspace, want_sum)
    if out is not None:
        return out
    dt, rows, V, stride = _logits_meta(logits)
    dev = logits.device
    if logp_out is not None:
        _check(logp_out, torch.float32, rows, "logp_out", dev)
    elif target_ids is not None:
        logp_out = torch.empty(rows, dtype=torch.float32, device=dev)
    if entropy_out is None:
        entropy_out = torch.empty(rows, dtype=torch.float32, device=dev)
    else:
        _check(entropy_out, torch.float32, rows, "entropy_out", dev)
    if want_sum and entropy_sum_out is None:
        entropy_sum_out = torch.empty(1, dtype=torch.float64, device=dev)
    if want_sum and entropy_count_out is None:
        entropy_count_out = torch.empty(1, dtype=torch.int64, device=dev)
    _check(target_ids, torch.int32, rows, "target_ids", dev)
    _check(row_mask, torch.uint8, rows, "row_mask", dev)
    _check(tau_rows, torch.float32, rows, "tau_rows", dev)
    _check_scalar_out(entropy_sum_out, torch.float64, "entropy_sum_out", dev)
    _check_scalar_out(entropy_count_out, torch.int64, "entropy_count_out", dev)
    ws, ws_bytes = _workspace(rows, V, workspace, dev)
    rc = lib().e3_logprob_entropy(_ptr(logits), dt, rows, V, stride, _ptr(target_ids),
                                  _ptr(row_mask), _ptr(tau_rows), float(tau_scalar),
                                  _ptr(logp_out), _ptr(entropy_out),
                                  _ptr(entropy_sum_out), _ptr(entropy_count_out),
                                  _ptr(ws), ws_bytes, _stream(dev))
    if rc != E3_OK:
        raise E3Error(rc, "e3_logprob_entropy")
    return logp_out, entropy_out, entropy_sum_out, entropy_count_out


def e3_logprob_entropy_advantages(logits: torch.Tensor, target_ids: Optional[torch.Tensor],
                                  row_mask: Optional[torch.Tensor], tau_rows: Optional[torch.Tensor],
                                  tau_scalar: float, rewards: torch.Tensor, group_offsets: torch.Tensor,
                                  ddof: int = 0, eps: float = 0.0,
                                  logp_out: Optional[torch.Tensor] = None,
                                  entropy_out: Optional[torch.Tensor] = None,
                                  entropy_sum_out: Optional[torch.Tensor] = None,
                                  entropy_count_out: Optional[torch.Tensor] = None,
                                  adv_out: Optional[torch.Tensor] = None,
                                  workspace=None, want_sum: bool = True):
    """e3_logprob_entropy and e3_grpo_advantages in one call.  Returns (logp, entropy,
    entropy_sum, entropy_count, adv)."""
    if rewards is not None:
        out = _ordinary("logprob_advantages", logits, target_ids, row_mask, tau_rows, tau_scalar, rewards, group_offsets, ddof,
                        eps, logp_out, entropy_out, entropy_sum_out, entropy_count_out, adv_out, workspace, want_sum)
        if out is not None:
            return out
    dt, rows, V, stride = _logits_meta(logits)
    dev = logits.device
    n = rewards.shape[0]
    num_groups = group_offsets.shape[0] - 1
    if logp_out is not None:
        _check(logp_out, torch.float32, rows, "logp_out", dev)
    elif target_ids is not None:
        logp_out = torch.empty(rows, dtype=torch.float32, device=dev)
    if entropy_out is None:
        entropy_out = torch.empty(rows, dtype=torch.float32, device=dev)
    else:
        _check(entropy_out, torch.float32, rows, "entropy_out", dev)
    if want_sum and entropy_sum_out is None:
        entropy_sum_out = torch.empty(1, dtype=torch.float64, device=dev)
    if want_sum and entropy_count_out is None:
        entropy_count_out = torch.empty(1, dtype=torch.int64, device=dev)
    if adv_out is None:
        adv_out = torch.empty(n, dtype=torch.float32, device=dev)
    else:
        _check(adv_out, torch.float32, n, "adv_out", dev)
    _check(target_ids, torch.int32, rows, "target_ids", dev)
    _check(row_mask, torch.uint8, rows, "row_mask", dev)
    _check(tau_rows, torch.float32, rows, "tau_rows", dev)
    _check_scalar_out(entropy_sum_out, torch.float64, "entropy_sum_out", dev)
    _check_scalar_out(entropy_count_out, torch.int64, "entropy_count_out", dev)
    _check(rewards, torch.float32, n, "rewards", dev)
    _check(group_offsets, torch.int32, num_groups + 1, "group_offsets", dev)
    ws, ws_bytes = _workspace(rows, V, workspace, dev)
    rc = lib().e3_logprob_entropy_advantages(_ptr(logits), dt, rows, V, stride, _ptr(target_ids),
                                             _ptr(row_mask), _ptr(tau_rows), float(tau_scalar),
                                             _ptr(logp_out), _ptr(entropy_out),
                                             _ptr(entropy_sum_out), _ptr(entropy_count_out),
                                             _ptr(rewards), _ptr(group_offsets), num_groups, int(ddof),
                                             float(eps), _ptr(adv_out), _ptr(ws), ws_bytes, _stream(dev))
    if rc != E3_OK:
        raise E3Error(rc, "e3_logprob_entropy_advantages")
    return logp_out, entropy_out, entropy_sum_out, entropy_count_out, adv_out


def e3_grpo_advantages(rewards: torch.Tensor, group_offsets: torch.Tensor, ddof: int = 0,
                       eps: float = 0.0, adv_out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Returns adv fp32 [N].  group_offsets is int32 [B+1] on the same device."""
    out = _ordinary("advantages", rewards, group_offsets, ddof, eps, adv_out)
    if out is not None:
        return out
    dev = rewards.device
    if not rewards.is_cuda:
        raise ValueError("rewards must live on the GPU")
    n = rewards.shape[0]
    num_groups = group_offsets.shape[0] - 1
    _check(rewards, torch.float32, n, "rewards", dev)
    _check(group_offsets, torch.int32, num_groups + 1, "group_offsets", dev)
    if adv_out is None:
        adv_out = torch.empty(n, dtype=torch.float32, device=dev)
    else:
        _check(adv_out, torch.float32, n, "adv_out", dev)
    rc = lib().e3_grpo_advantages(_ptr(rewards), _ptr(group_offsets), num_groups, int(ddof),
                                  float(eps), _ptr(adv_out), _stream(dev))
    if rc != E3_OK:
        raise E3Error(rc, "e3_grpo_advantages")
    return adv_out


def e3_temperature_update(tau_t: float, H_t: float, H_init: float, vocab: int, t: int = 0,
                          t_anneal: int = -1, t_max: int = 0, eta: float = 1.0,
                          tau_min: float = 0.0, tau_max: float = float("inf")):
    """Host-only scheduler step.  Returns (tau_next, H_target)."""
    out = _ordinary("temperature", tau_t, H_t, H_init, vocab, t, t_anneal, t_max, eta, tau_min, tau_max)
    if out is not None:
        return out
    nxt, tgt = C.c_double(float("nan")), C.c_double(float("nan"))
    rc = lib().e3_temperature_update(float(tau_t), float(H_t), float(H_init), int(vocab), int(t),
                                     int(t_anneal), int(t_max), float(eta), float(tau_min),
                                     float(tau_max), C.addressof(nxt), C.addressof(tgt))
    if rc != E3_OK:
        raise E3Error(rc, "e3_temperature_update")
    return nxt.value, tgt.value


def e3_difficulty_ranks(cum_reward, cum_rollouts):
    """Host-only.  Returns k (numpy float64 [num_questions])."""
    import numpy as np
    r = np.ascontiguousarray(cum_reward, dtype=np.float64)
    n = np.ascontiguousarray(cum_rollouts, dtype=np.int64)
    if r.shape != n.shape or r.ndim != 1:
        raise ValueError("cum_reward and cum_rollouts must be 1-D and of equal length")
    k = np.empty(r.shape[0], dtype=np.float64)
    rc = lib().e3_difficulty_ranks(r.ctypes.data, n.ctypes.data, r.shape[0], k.ctypes.data)
    if rc != E3_OK:
        raise E3Error(rc, "e3_difficulty_ranks")
    return k


def e3_allocate_budgets(k, G: int, G_min: int, G_max: int):
    """Host-only.  Returns (G_i int32 [B], offsets int32 [B+1]) as numpy arrays."""
    import numpy as np
    k = np.ascontiguousarray(k, dtype=np.float64)
    B = k.shape[0]
    g = np.empty(B, dtype=np.int32)
    off = np.empty(B + 1, dtype=np.int32)
    rc = lib().e3_allocate_budgets(k.ctypes.data, B, int(G), int(G_min), int(G_max),
                                   g.ctypes.data, off.ctypes.data)
    if rc != E3_OK:
        raise E3Error(rc, "e3_allocate_budgets")
    return g, off


def e3_budget_bounds(G: int, passes_done: int, step: int, G_min_limit: int, G_max_limit: int):
    """Host-only.  Returns (G_min, G_max)."""
    lo, hi = C.c_int32(-1), C.c_int32(-1)
    rc = lib().e3_budget_bounds(int(G), int(passes_done), int(step), int(G_min_limit),
                                int(G_max_limit), C.addressof(lo), C.addressof(hi))
    if rc != E3_OK:
        raise E3Error(rc, "e3_budget_bounds")
    return lo.value, hi.value


def e3_logprob_entropy_gap(logits: torch.Tensor, target_ids: Optional[torch.Tensor],
                           row_mask: Optional[torch.Tensor], tau_rows: Optional[torch.Tensor],
                           tau_scalar: float, workspace=None):
    """Returns (logp or None, entropy, gap, entropy_sum fp64 [1], gap_sum fp64 [1], count int64 [1]),
    all on the device."""
    out = _ordinary("logprob_gap", logits, target_ids, row_mask, tau_rows, tau_scalar, workspace)
    if out is not None:
        return out
    dt, rows, V, stride = _logits_meta(logits)
    dev = logits.device
    logp = torch.empty(rows, dtype=torch.float32, device=dev) if target_ids is not None else None
    ent = torch.empty(rows, dtype=torch.float32, device=dev)
    gap = torch.empty(rows, dtype=torch.float32, device=dev)
    hs = torch.empty(1, dtype=torch.float64, device=dev)
    gs = torch.empty(1, dtype=torch.float64, device=dev)
    cnt = torch.empty(1, dtype=torch.int64, device=dev)
    _check(target_ids, torch.int32, rows, "target_ids", dev)
    _check(row_mask, torch.uint8, rows, "row_mask", dev)
    _check(tau_rows, torch.float32, rows, "tau_rows", dev)
    ws, ws_bytes = _workspace(rows, V, workspace, dev)
    rc = lib().e3_logprob_entropy_gap(_ptr(logits), dt, rows, V, stride, _ptr(target_ids),
                                      _ptr(row_mask), _ptr(tau_rows), float(tau_scalar),
                                      _ptr(logp), _ptr(ent), _ptr(gap), _ptr(hs), _ptr(gs), _ptr(cnt),
                                      _ptr(ws), ws_bytes, _stream(dev))
    if rc != E3_OK:
        raise E3Error(rc, "e3_logprob_entropy_gap")
    return logp, ent, gap, hs, gs, cnt


def e3_temperature_update_gap(tau_t: float, H_t: float, H_init: float, gap: float, t: int = 0,
                              t_anneal: int = -1, t_max: int = 0, eta: float = 1.0,
                              tau_min: float = 0.0, tau_max: float = float("inf")):
    """Host-only scheduler step with a measured gap.  Returns (tau_next, H_target)."""
    nxt, tgt = C.c_double(float("nan")), C.c_double(float("nan"))
    rc = lib().e3_temperature_update_gap(float(tau_t), float(H_t), float(H_init), float(gap), int(t),
                                         int(t_anneal), int(t_max), float(eta), float(tau_min),
                                         float(tau_max), C.addressof(nxt), C.addressof(tgt))
    if rc != E3_OK:
        raise E3Error(rc, "e3_temperature_update_gap")
    return nxt.value, tgt.value


def e3_grpo_objective(logp_new: torch.Tensor, logp_old: torch.Tensor, seq_offsets: torch.Tensor,
                      adv: torch.Tensor, group_offsets: torch.Tensor, clip_eps: float,
                      want_token_terms: bool = False):
    """Returns (objective fp64 [1], seq_mean fp64 [N], token_terms fp32 [T] or None), on the device."""
    out = _ordinary("objective", logp_new, logp_old, seq_offsets, adv, group_offsets, clip_eps, want_token_terms)
    if out is not None:
        return out
    dev = logp_new.device
    if not logp_new.is_cuda:
        raise ValueError("logp_new must live on the GPU")
    T = logp_new.shape[0]
    N = adv.shape[0]
    B = group_offsets.shape[0] - 1
    _check(logp_new, torch.float32, T, "logp_new", dev)
    _check(logp_old, torch.float32, T, "logp_old", dev)
    _check(seq_offsets, torch.int32, N + 1, "seq_offsets", dev)
    _check(adv, torch.float32, N, "adv", dev)
    _check(group_offsets, torch.int32, B + 1, "group_offsets", dev)
    terms = torch.empty(T, dtype=torch.float32, device=dev) if want_token_terms else None
    seq_mean = torch.empty(N, dtype=torch.float64, device=dev)
    J = torch.empty(1, dtype=torch.float64, device=dev)
    rc = lib().e3_grpo_objective(_ptr(logp_new), _ptr(logp_old), _ptr(seq_offsets), _ptr(adv), N,
                                 _ptr(group_offsets), B, float(clip_eps), _ptr(terms),
                                 _ptr(seq_mean), _ptr(J), _stream(dev))
    if rc != E3_OK:
        raise E3Error(rc, "e3_grpo_objective")
    return J, seq_mean, terms


class E3Cache(NamedTuple):
    """A paged cache of keys and values (e3_cache in include/e3.h): k [pages, heads, page, D], v [pages, heads, page / 8, D, 8]
    of torch.bfloat16, or of torch.float8_e4m3fn with the exponent bytes k_scale, v_scale [pages, heads, page]."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: Optional[torch.Tensor] = None
    v_scale: Optional[torch.Tensor] = None


class _CacheStruct(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("num_pages", C.c_int64), ("page_size", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("dtype", C.c_int32)]


def new_cache(num_pages: int, page_size: int, kv_heads: int, head_dim: int, dtype: torch.dtype = torch.float8_e4m3fn,
              device="cuda") -> E3Cache:
    """Allocate an empty cache.  dtype: torch.float8_e4m3fn (8 bits, quantised as it is written) or torch.bfloat16."""
    if dtype not in (torch.float8_e4m3fn, torch.bfloat16):
        raise TypeError(f"unsupported cache dtype {dtype}")
    if page_size < 32 or page_size & (page_size - 1):
        raise ValueError("page_size must be a power of two of at least 32")
    k = torch.zeros((num_pages, kv_heads, page_size, head_dim), dtype=dtype, device=device)
    v = torch.zeros((num_pages, kv_heads, page_size // 8, head_dim, 8), dtype=dtype, device=device)
    if dtype is torch.bfloat16:
        return E3Cache(k, v)
    scales = [torch.zeros((num_pages, kv_heads, page_size), dtype=torch.uint8, device=device) for _ in range(2)]
    return E3Cache(k, v, *scales)


def _cache(cache) -> _CacheStruct:
    k, v, ks, vs = cache
    if k.dim() != 4 or not k.is_cuda:
        raise ValueError("a cache's keys must be [pages, heads, page, D] on the GPU")
    pages, heads, page, D = k.shape
    dev = k.device
    if k.dtype is torch.bfloat16:
        dt = E3_BF16
    elif k.dtype is torch.float8_e4m3fn:
        dt = E3_E4M3
    else:
        raise TypeError(f"unsupported cache dtype {k.dtype}")
    if v.dtype is not k.dtype or v.device != dev or v.shape != (pages, heads, page // 8, D, 8):
        raise ValueError("a cache's values must be [pages, heads, page / 8, D, 8] of the keys' type and device")
    if not k.is_contiguous() or not v.is_contiguous():
        raise ValueError("a cache's tensors must be contiguous")
    for t, name in ((ks, "k_scale"), (vs, "v_scale")):
        if (t is None) != (dt == E3_BF16):
            raise ValueError(f"{name} belongs to an 8-bit cache, and to no other")
        if t is not None and (t.dtype is not torch.uint8 or t.shape != (pages, heads, page) or t.device != dev
                              or not t.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous uint8 tensor [pages, heads, page] on {dev}")
    return _CacheStruct(_ptr(k), _ptr(v), _ptr(ks), _ptr(vs), pages, page, heads, D, dt)


_FLOATS = {torch.bfloat16: E3_BF16, torch.float32: E3_F32}


def _float_type(dtype) -> int:
    if dtype not in _FLOATS:
        raise TypeError(f"unsupported dtype {dtype}")
    return _FLOATS[dtype]


def _step(t: torch.Tensor, dim: int) -> int:
    """A dimension's stride; one of a single element has none of its own (torch may report anything)."""
    return t.stride(dim) if t.shape[dim] > 1 else 0


def e3_cache_append(cache: E3Cache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor) -> None:
    """Write keys and values [tokens, heads, D] (bf16 or fp32, any strides with columns next to each other) to the slots
    (int64 [tokens]; negative: skipped) of the cache."""
    if _ordinary("cache_append", cache, k, v, slots) is not None:
        return
    c = _cache(cache)
    dev = cache[0].device
    dt = _float_type(k.dtype)
    n = slots.shape[0]
    for t, name in ((k, "k"), (v, "v")):
        if t.dtype is not k.dtype or t.shape != (n, c.kv_heads, c.head_dim) or t.device != dev or (n and t.stride(2) != 1):
            raise ValueError(f"{name} must be a {k.dtype} tensor [{n}, {c.kv_heads}, {c.head_dim}] with unit column stride on {dev}")
    _check(slots, torch.int64, n, "slots", dev)
    rc = lib().e3_cache_append(C.byref(c), _ptr(k), _ptr(v), dt, n, _step(k, 0), _step(k, 1), _step(v, 0), _step(v, 1),
                               _ptr(slots), _stream(dev))
    if rc != E3_OK:
        raise E3Error(rc, "e3_cache_append")


def e3_cache_read(cache: E3Cache, slots: torch.Tensor, dtype: torch.dtype = torch.bfloat16,
                  k_out: Optional[torch.Tensor] = None, v_out: Optional[torch.Tensor] = None):
    """Returns (k, v) [tokens, heads, D] of the slots (int64 [tokens]; outside the cache: zeros) in bf16 or fp32."""
    if dtype is torch.bfloat16 or dtype is torch.float32:
        out = _ordinary("cache_read", cache, slots, dtype is torch.bfloat16, k_out, v_out)
        if out is not None:
            return out
    c = _cache(cache)
    dev = cache[0].device
    n = slots.shape[0]
    _check(slots, torch.int64, n, "slots", dev)
    outs = []
    for t, name in ((k_out, "k_out"), (v_out, "v_out")):
        if t is None:
            t = torch.empty((n, c.kv_heads, c.head_dim), dtype=dtype, device=dev)
        elif t.dtype is not dtype or t.shape != (n, c.kv_heads, c.head_dim) or t.device != dev or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous {dtype} tensor [{n}, {c.kv_heads}, {c.head_dim}] on {dev}")
        outs.append(t)
    rc = lib().e3_cache_read(C.byref(c), _ptr(slots), n, _ptr(outs[0]), _ptr(outs[1]), _float_type(dtype), _stream(dev))
    if rc != E3_OK:
        raise E3Error(rc, "e3_cache_read")
    return outs[0], outs[1]


def _integer(v, bits: int, name: str) -> int:
    """An int that C takes in so many bits (ctypes would cut it)."""
    v = int(v)
    if not -(1 << (bits - 1)) <= v < 1 << (bits - 1):
        raise ValueError(f"{name} must fit {bits} bits")
    return v


def _int32(v, name: str) -> int:
    return _integer(v, 32, name)


def _int64(v, name: str) -> int:
    return _integer(v, 64, name)


class E3Rotary(NamedTuple):
    """Rotary positions (e3_rotary in include/e3.h): freqs fp64 [pairs], radians per position; axis uint8 [pairs] or None (one axis);
    neighbours: pairs of columns (2 i, 2 i + 1) instead of (i, i + pairs)."""
    freqs: torch.Tensor
    axis: Optional[torch.Tensor] = None
    neighbours: bool = False


class _RotaryStruct(C.Structure):
    _fields_ = [("freqs", C.c_void_p), ("axis", C.c_void_p), ("rot_dim", C.c_int32), ("axes", C.c_int32), ("neighbours", C.c_int32)]


def new_rotary(rot_dim: int, base: float = 10000.0, sections=None, neighbours: bool = False, device="cuda") -> E3Rotary:
    """Frequencies base^(-2 i / rot_dim) for the rot_dim / 2 pairs.  sections: how many pairs, in order, go by each axis."""
    if rot_dim < 16 or rot_dim % 16:
        raise ValueError("rot_dim must be a multiple of 16")
    pairs = rot_dim // 2
    freqs = torch.tensor([float(base) ** (-2.0 * i / rot_dim) for i in range(pairs)], dtype=torch.float64)
    axis = None
    if sections is not None:
        if sum(sections) != pairs or min(sections) < 0 or len(sections) > E3_MAX_AXES:
            raise ValueError(f"sections must be at most {E3_MAX_AXES} numbers of pairs that add up to {pairs}")
        axis = torch.tensor([a for a, n in enumerate(sections) for _ in range(n)], dtype=torch.uint8).to(device)
    return E3Rotary(freqs.to(device), axis, neighbours)


def _rotary(rotary, positions: torch.Tensor, tokens: int, device) -> Tuple[_RotaryStruct, int]:
    """The struct, and the stride of the positions' rows."""
    freqs, axis, neighbours = rotary
    if freqs.dtype is not torch.float64 or freqs.dim() != 1 or not freqs.is_contiguous() or freqs.device != device:
        raise ValueError(f"freqs must be a contiguous fp64 vector on {device}")
    pairs = freqs.shape[0]
    _check(axis, torch.uint8, pairs, "axis", device)
    if positions.dtype is not torch.int64 or positions.dim() not in (1, 2) or positions.shape[-1] != tokens or positions.device != device \
            or (tokens > 1 and positions.stride(-1) != 1):
        raise ValueError(f"positions must be an int64 tensor [axes, {tokens}] (or [{tokens}]) with unit stride on {device}")
    axes = positions.shape[0] if positions.dim() == 2 else 1
    if axis is None and axes != 1:
        raise ValueError("positions on several axes need the rotary's axis")
    return _RotaryStruct(_ptr(freqs), _ptr(axis), 2 * pairs, axes, int(bool(neighbours))), positions.stride(0) if axes > 1 else 0


def _heads(t: torch.Tensor, name: str, dtype, shape, device) -> None:
    if t.dtype is not dtype or tuple(t.shape) != tuple(shape) or t.device != device or (t.numel() and t.shape[2] > 1 and t.stride(2) != 1):
        raise ValueError(f"{name} must be a {dtype} tensor {list(shape)} with unit column stride on {device}")


def e3_rotate(x: torch.Tensor, rotary: E3Rotary, positions: torch.Tensor, out: Optional[torch.Tensor] = None,
              inverse: bool = False) -> torch.Tensor:
    """Turn x [tokens, heads, D] (bf16 or fp32, any strides with columns next to each other) by its tokens' positions (int64 [axes,
    tokens], or [tokens]); inverse: by the opposite angles, which takes a gradient back.  out: like x, x itself allowed."""
    res = _ordinary("rotate", x, rotary, positions, out, inverse)
    if res is not None:
        return res
    if x.dim() != 3 or not x.is_cuda:
        raise ValueError("x must be [tokens, heads, D] on the GPU")
    dt, dev = _float_type(x.dtype), x.device
    _heads(x, "x", x.dtype, x.shape, dev)
    n, H, D = x.shape
    r, stride = _rotary(rotary, positions, n, dev)
    if out is None:
        out = torch.empty((n, H, D), dtype=x.dtype, device=dev)
    else:
        _heads(out, "out", x.dtype, x.shape, dev)
    rc = lib().e3_rotate(C.byref(r), _ptr(positions), stride, _ptr(x), dt, n, H, D, _step(x, 0), _step(x, 1), _ptr(out), _step(out, 0),
                         _step(out, 1), int(bool(inverse)), _stream(dev))
    if rc != E3_OK:
        raise E3Error(rc, "e3_rotate")
    return out


def e3_cache_append_rotated(cache: E3Cache, q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, rotary: E3Rotary,
                            positions: torch.Tensor, slots: torch.Tensor, q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
    """e3_cache_append with the keys turned by their positions (int64 [axes, tokens], or [tokens]) on the way.  Returns the queries q [tokens,
    q_heads, D] turned as well (in q_out if given, which may be q), or None without queries."""
    res = _ordinary("append_rotated", cache, q, k, v, rotary, positions, slots, q_out)
    if res is not None:
        return None if res is True else res
    c = _cache(cache)
    dev = cache[0].device
    dt = _float_type(k.dtype)
    n = slots.shape[0]
    for t, name in ((k, "k"), (v, "v")):
        _heads(t, name, k.dtype, (n, c.kv_heads, c.head_dim), dev)
    _check(slots, torch.int64, n, "slots", dev)
    r, stride = _rotary(rotary, positions, n, dev)
    q_heads, strides, out_strides = 0, (0, 0), (0, 0)
    if q is not None:
        if q.dim() != 3:
            raise ValueError(f"q must be [{n}, q_heads, {c.head_dim}]")
        q_heads = q.shape[1]
        _heads(q, "q", k.dtype, (n, q_heads, c.head_dim), dev)
        if q_out is None:
            q_out = torch.empty((n, q_heads, c.head_dim), dtype=k.dtype, device=dev)
        else:
            _heads(q_out, "q_out", k.dtype, (n, q_heads, c.head_dim), dev)
        strides, out_strides = (_step(q, 0), _step(q, 1)), (_step(q_out, 0), _step(q_out, 1))
    elif q_out is not None:
        raise ValueError("q_out belongs to q")
    rc = lib().e3_cache_append_rotated(C.byref(c), C.byref(r), _ptr(positions), stride, _ptr(q), _ptr(k), _ptr(v), dt, n, q_heads, *strides,
                                       _step(k, 0), _step(k, 1), _step(v, 0), _step(v, 1), _ptr(slots), _ptr(q_out), *out_strides, _stream(dev))
    if rc != E3_OK:
        raise E3Error(rc, "e3_cache_append_rotated")
    return q_out


def e3_prefix_attention_workspace_bytes(rows: int, queries: int, q_heads: int, kv_heads: int, head_dim: int, num_groups: int) -> int:
    """Host-only; 0 for a shape that is not served."""
    return int(lib().e3_prefix_attention_workspace_bytes(rows, queries, q_heads, kv_heads, head_dim, num_groups))


def _table(t: torch.Tensor, n: int, name: str, device) -> int:
    if t.dtype is not torch.int32 or t.dim() != 2 or t.shape[0] != n or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{name} must be a contiguous int32 tensor [{n}, pages] on {device}")
    return t.shape[1]


def e3_prefix_attention(q: torch.Tensor, cache: E3Cache, group_offsets: Optional[torch.Tensor],
                        prefix_pages: Optional[torch.Tensor], prefix_lens: Optional[torch.Tensor],
                        row_pages: torch.Tensor, row_lens: torch.Tensor, scale: float,
                        out: Optional[torch.Tensor] = None, lse_out: Optional[torch.Tensor] = None,
                        workspace: Optional[torch.Tensor] = None, want_lse: bool = True):
    """Attention of a decode step: q bf16 [rows, queries, q_heads, D]; row r of group g (group_offsets int32 [groups + 1], None:
    no prefixes) sees the group's prefix (prefix_pages int32 [groups, width], prefix_lens int32 [groups]) and its own
    tokens (row_pages, row_lens), query t all but its last queries - 1 - t.  Returns (out bf16 like q, lse fp32 [rows, queries,
    q_heads] or None).  workspace: a tensor of e3_prefix_attention_workspace_bytes(), or None to allocate one."""
    res = _ordinary("attention", q, cache, group_offsets, prefix_pages, prefix_lens, row_pages, row_lens, scale, out, lse_out,
                    workspace, want_lse)
    if res is not None:
        return res
    c = _cache(cache)
    dev = cache[0].device
    if q.dim() != 4 or q.dtype is not torch.bfloat16 or q.device != dev or q.shape[3] != c.head_dim or (q.numel() and q.stride(3) != 1):
        raise ValueError(f"q must be a bf16 tensor [rows, queries, q_heads, {c.head_dim}] with unit column stride on {dev}")
    rows, T, q_heads, D = q.shape
    groups = 0 if group_offsets is None else group_offsets.shape[0] - 1
    prefix_width = 0
    if group_offsets is not None:
        _check(group_offsets, torch.int32, groups + 1, "group_offsets", dev)
        if prefix_pages is None or prefix_lens is None:
            raise ValueError("groups need prefix_pages and prefix_lens")
        prefix_width = _table(prefix_pages, groups, "prefix_pages", dev)
        _check(prefix_lens, torch.int32, groups, "prefix_lens", dev)
    row_width = _table(row_pages, rows, "row_pages", dev)
    _check(row_lens, torch.int32, rows, "row_lens", dev)
    if out is None:
        out = torch.empty((rows, T, q_heads, D), dtype=torch.bfloat16, device=dev)
    elif out.dtype is not torch.bfloat16 or out.shape != q.shape or out.device != dev or not out.is_contiguous():
        raise ValueError(f"out must be a contiguous bf16 tensor {tuple(q.shape)} on {dev}")
    if lse_out is None:
        lse_out = torch.empty((rows, T, q_heads), dtype=torch.float32, device=dev) if want_lse else None
    elif lse_out.dtype is not torch.float32 or lse_out.shape != q.shape[:3] or lse_out.device != dev or not lse_out.is_contiguous():
        raise ValueError(f"lse_out must be a contiguous fp32 tensor {tuple(q.shape[:3])} on {dev}")
    if workspace is None:
        need = e3_prefix_attention_workspace_bytes(rows, T, q_heads, c.kv_heads, D, groups)
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    elif workspace.device != dev or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on {dev}")
    rc = lib().e3_prefix_attention(C.byref(c), _ptr(q), rows, T, q_heads, _step(q, 0), _step(q, 1), _step(q, 2),
                                   _ptr(group_offsets) if groups else None, groups, _ptr(prefix_pages), prefix_width,
                                   _ptr(prefix_lens), _ptr(row_pages), row_width, _ptr(row_lens), float(scale),
                                   _ptr(out), _ptr(lse_out), _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(dev))
    if rc != E3_OK:
        raise E3Error(rc, "e3_prefix_attention")
    return out, lse_out


def e3_window_attention_workspace_bytes(rows: int, tokens: int, q_heads: int, kv_heads: int, head_dim: int) -> int:
    """Host-only; 0 for a shape that is not served."""
    return int(lib().e3_window_attention_workspace_bytes(rows, tokens, q_heads, kv_heads, head_dim))


def e3_window_attention(q: torch.Tensor, cache: E3Cache, query_offsets: torch.Tensor, row_pages: torch.Tensor, row_lens: torch.Tensor,
                        window: int, sinks: int, scale: float, out: Optional[torch.Tensor] = None, lse_out: Optional[torch.Tensor] = None,
                        workspace: Optional[torch.Tensor] = None, want_lse: bool = True):
    """Attention with a sliding window over the cache: q bf16 [tokens, q_heads, D]; row r brings queries query_offsets[r] ..
    query_offsets[r + 1] - 1 (int32 [rows + 1]), the last ones of its row_lens[r] tokens (int32 [rows], in pages row_pages int32 [rows, width]); the
    one at position p sees the tokens j <= p with j > p - window or j < sinks.  Returns (out bf16 like q, lse fp32 [tokens, q_heads] or
    None).  workspace: a tensor of e3_window_attention_workspace_bytes(), or None to allocate one."""
    res = _ordinary("window", q, cache, query_offsets, row_pages, row_lens, window, sinks, scale, out, lse_out, workspace, want_lse)
    if res is not None:
        return res
    c = _cache(cache)
    dev = cache[0].device
    window, sinks = _int64(window, "window"), _int64(sinks, "sinks")
    if q.dim() != 3:
        raise ValueError(f"q must be [tokens, q_heads, {c.head_dim}]")
    tokens, q_heads, D = q.shape
    _heads(q, "q", torch.bfloat16, (tokens, q_heads, c.head_dim), dev)
    rows = query_offsets.shape[0] - 1
    _check(query_offsets, torch.int32, rows + 1, "query_offsets", dev)
    row_width = _table(row_pages, rows, "row_pages", dev)
    _check(row_lens, torch.int32, rows, "row_lens", dev)
    if out is None:
        out = torch.empty((tokens, q_heads, D), dtype=torch.bfloat16, device=dev)
    elif out.dtype is not torch.bfloat16 or out.shape != q.shape or out.device != dev or not out.is_contiguous():
        raise ValueError(f"out must be a contiguous bf16 tensor {tuple(q.shape)} on {dev}")
    if lse_out is None:
        lse_out = torch.empty((tokens, q_heads), dtype=torch.float32, device=dev) if want_lse else None
    elif lse_out.dtype is not torch.float32 or lse_out.shape != q.shape[:2] or lse_out.device != dev or not lse_out.is_contiguous():
        raise ValueError(f"lse_out must be a contiguous fp32 tensor {tuple(q.shape[:2])} on {dev}")
    if workspace is None:
        workspace = torch.empty(e3_window_attention_workspace_bytes(rows, tokens, q_heads, c.kv_heads, D), dtype=torch.uint8, device=dev)
    elif workspace.device != dev or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on {dev}")
    rc = lib().e3_window_attention(C.byref(c), _ptr(q), tokens, q_heads, _step(q, 0), _step(q, 1), _ptr(query_offsets), rows, _ptr(row_pages),
                                   row_width, _ptr(row_lens), window, sinks, float(scale), _ptr(out), _ptr(lse_out), _ptr(workspace),
                                   workspace.numel() * workspace.element_size(), _stream(dev))
    if rc != E3_OK:
        raise E3Error(rc, "e3_window_attention")
    return out, lse_out


def e3_verify_workspace_bytes(rows: int, drafts: int, V: int) -> int:
    """Host-only; 0 for a shape that is not served."""
    return int(lib().e3_verify_workspace_bytes(rows, drafts, V))


def _positions(t: torch.Tensor, name: str, dtype, shape, device) -> Tuple[int, int]:
    if t.dtype is not dtype or t.dim() != 3 or tuple(t.shape) != tuple(shape) or t.device != device or (t.shape[2] > 1 and t.stride(2) != 1):
        raise ValueError(f"{name} must be a {dtype} tensor {list(shape)} with unit column stride on {device}")
    # a dimension of one has no stride of its own: torch may report anything
    V = t.shape[2]
    pitch = t.stride(1) if t.shape[1] > 1 else -(-V // 8) * 8
    return (t.stride(0) if t.shape[0] > 1 else pitch * t.shape[1]), pitch


def e3_verify_drafts(logits: torch.Tensor, draft_tokens: Optional[torch.Tensor], draft_logits: Optional[torch.Tensor],
                     draft_lens: Optional[torch.Tensor], tau_rows: Optional[torch.Tensor], tau_scalar: float,
                     seed: int, row_base: int = 0, draft_tau_rows: Optional[torch.Tensor] = None,
                     accepted_out: Optional[torch.Tensor] = None, token_out: Optional[torch.Tensor] = None,
                     logp_out: Optional[torch.Tensor] = None, entropy_out: Optional[torch.Tensor] = None,
                     workspace: Optional[torch.Tensor] = None):
    """Verify drafted tokens: logits [rows, drafts + 1, V], draft_tokens int32 [rows, drafts], draft_logits [rows, drafts, V] or None
    (drafts without a distribution).  Returns (accepted int32 [rows], token int32 [rows, drafts + 1], logp fp32, entropy fp32 of the
    same shape).  workspace: a tensor of e3_verify_workspace_bytes(), or None to allocate one."""
    res = _ordinary("verify", logits, draft_tokens, draft_logits, draft_lens, tau_rows, tau_scalar, seed, row_base, draft_tau_rows,
                    accepted_out, token_out, logp_out, entropy_out, workspace)
    if res is not None:
        return res
    if logits.dim() != 3 or not logits.is_cuda:
        raise ValueError("logits must be [rows, drafts + 1, V] on the GPU")
    dt = _float_type(logits.dtype)
    rows, positions, V = logits.shape
    drafts, dev = positions - 1, logits.device
    row_stride, position_stride = _positions(logits, "logits", logits.dtype, (rows, positions, V), dev)
    draft_strides = (0, 0)
    if draft_logits is not None:                # (without drafts an empty tensor, whose strides say nothing)
        draft_strides = _positions(draft_logits, "draft_logits", logits.dtype, (rows, drafts, V), dev) if drafts else (0, 0)
    if draft_tokens is not None or drafts > 0:
        if (draft_tokens is None or draft_tokens.dtype is not torch.int32 or tuple(draft_tokens.shape) != (rows, drafts)
                or not draft_tokens.is_contiguous() or draft_tokens.device != dev):
            raise ValueError(f"draft_tokens must be a contiguous int32 tensor [{rows}, {drafts}] on {dev}")
    _check(draft_lens, torch.int32, rows, "draft_lens", dev)
    _check(tau_rows, torch.float32, rows, "tau_rows", dev)
    _check(draft_tau_rows, torch.float32, rows, "draft_tau_rows", dev)
    if accepted_out is None:
        accepted_out = torch.empty(rows, dtype=torch.int32, device=dev)
    else:
        _check(accepted_out, torch.int32, rows, "accepted_out", dev)
    outs = []
    for t, dtype, name in ((token_out, torch.int32, "token_out"), (logp_out, torch.float32, "logp_out"), (entropy_out, torch.float32, "entropy_out")):
        if t is None:
            t = torch.empty((rows, positions), dtype=dtype, device=dev)
        elif t.dtype is not dtype or tuple(t.shape) != (rows, positions) or t.device != dev or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous {dtype} tensor [{rows}, {positions}] on {dev}")
        outs.append(t)
    if workspace is None:
        workspace = torch.empty(e3_verify_workspace_bytes(rows, drafts, V), dtype=torch.uint8, device=dev)
    elif workspace.device != dev or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on {dev}")
    rc = lib().e3_verify_drafts(_ptr(logits), dt, rows, drafts, V, row_stride, position_stride, _ptr(draft_tokens), _ptr(draft_lens),
                                _ptr(draft_logits), *draft_strides, _ptr(tau_rows), float(tau_scalar), _ptr(draft_tau_rows),
                                int(seed), int(row_base), _ptr(accepted_out), *(_ptr(t) for t in outs), _ptr(workspace),
                                workspace.numel() * workspace.element_size(), _stream(dev))
    if rc != E3_OK:
        raise E3Error(rc, "e3_verify_drafts")
    return (accepted_out, *outs)


def e3_beam_workspace_bytes(seqs: int, beams: int, V: int) -> int:
    """Host-only; 0 for a shape that is not served."""
    return int(lib().e3_beam_workspace_bytes(seqs, beams, V))


def e3_beam_select(logits: torch.Tensor, scores: torch.Tensor, keep: int, tau: float = 1.0, finished: Optional[torch.Tensor] = None,
                   eos_token: int = -1, parent_out: Optional[torch.Tensor] = None, token_out: Optional[torch.Tensor] = None,
                   score_out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """The `keep` best continuations of every sequence: logits [seqs, beams, V], scores fp32 [seqs, beams] (sums of log-probs; -inf: none),
    finished uint8 [seqs, beams] or None (with eos_token).  Returns (parent int32, token int32, score fp32), [seqs, keep] each.
    workspace: a tensor of e3_beam_workspace_bytes(), or None to allocate one."""
    res = _ordinary("beam_select", logits, scores, keep, tau, finished, eos_token, parent_out, token_out, score_out, workspace)
    if res is not None:
        return res
    if logits.dim() != 3 or not logits.is_cuda:
        raise ValueError("logits must be [seqs, beams, V] on the GPU")
    dt, dev = _float_type(logits.dtype), logits.device
    seqs, beams, V = logits.shape
    keep, eos_token = _int32(keep, "keep"), _int32(eos_token, "eos_token")
    if keep < 1 or keep > E3_MAX_KEEP:                             # (before outputs of that size are allocated)
        raise E3Error(E3_ERR_SHAPE, "e3_beam_select")
    seq_stride, beam_stride = _positions(logits, "logits", logits.dtype, (seqs, beams, V), dev)
    for t, dtype, name in ((scores, torch.float32, "scores"), (finished, torch.uint8, "finished")):
        if t is not None and (t.dtype is not dtype or tuple(t.shape) != (seqs, beams) or t.device != dev or not t.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous {dtype} tensor [{seqs}, {beams}] on {dev}")
    outs = []
    for t, dtype, name in ((parent_out, torch.int32, "parent_out"), (token_out, torch.int32, "token_out"), (score_out, torch.float32, "score_out")):
        if t is None:
            t = torch.empty((seqs, keep), dtype=dtype, device=dev)
        elif t.dtype is not dtype or tuple(t.shape) != (seqs, keep) or t.device != dev or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous {dtype} tensor [{seqs}, {keep}] on {dev}")
        outs.append(t)
    if workspace is None:
        workspace = torch.empty(e3_beam_workspace_bytes(seqs, beams, V), dtype=torch.uint8, device=dev)
    elif workspace.device != dev or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on {dev}")
    rc = lib().e3_beam_select(_ptr(logits), dt, seqs, beams, V, seq_stride, beam_stride, _ptr(scores), keep, float(tau), _ptr(finished),
                              eos_token, *(_ptr(t) for t in outs), _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(dev))
    if rc != E3_OK:
        raise E3Error(rc, "e3_beam_select")
    return tuple(outs)


def e3_beam_reorder(parent: torch.Tensor, row_pages: torch.Tensor, row_lens: torch.Tensor, page_size: int,
                    pages_out: Optional[torch.Tensor] = None, lens_out: Optional[torch.Tensor] = None, src_out: Optional[torch.Tensor] = None,
                    dst_out: Optional[torch.Tensor] = None, counts_out: Optional[torch.Tensor] = None):
    """The beams' page tables after a selection: parent int32 [seqs, beams], row_pages int32 [seqs * beams, width], row_lens int32
    [seqs * beams].  Returns (row_pages, row_lens, src, dst, counts), the last three (int32 [seqs * beams]) for e3_cache_copy.  Entries behind
    the page of a row's next token are its parent's, the same in all of the parent's children: set them anew where tables are filled ahead."""
    res = _ordinary("beam_reorder", parent, row_pages, row_lens, page_size, pages_out, lens_out, src_out, dst_out, counts_out)
    if res is not None:
        return res
    dev = parent.device
    if parent.dtype is not torch.int32 or parent.dim() != 2 or not parent.is_contiguous() or not parent.is_cuda:
        raise ValueError("parent must be a contiguous int32 tensor [seqs, beams] on the GPU")
    seqs, beams = parent.shape
    rows, page_size = seqs * beams, _int32(page_size, "page_size")
    width = _table(row_pages, rows, "row_pages", dev)
    _check(row_lens, torch.int32, rows, "row_lens", dev)
    if pages_out is None:
        pages_out = torch.empty((rows, width), dtype=torch.int32, device=dev)
    elif _table(pages_out, rows, "pages_out", dev) != width:
        raise ValueError(f"pages_out must be [{rows}, {width}]")
    outs = []
    for t, name in ((lens_out, "lens_out"), (src_out, "src_out"), (dst_out, "dst_out"), (counts_out, "counts_out")):
        if t is None:
            t = torch.empty(rows, dtype=torch.int32, device=dev)
        else:
            _check(t, torch.int32, rows, name, dev)
        outs.append(t)
    rc = lib().e3_beam_reorder(_ptr(parent), seqs, beams, _ptr(row_pages), width, _ptr(row_lens), page_size, _ptr(pages_out),
                               *(_ptr(t) for t in outs), _stream(dev))
    if rc != E3_OK:
        raise E3Error(rc, "e3_beam_reorder")
    return (pages_out, *outs)


def e3_cache_copy(cache: E3Cache, src_pages: torch.Tensor, dst_pages: torch.Tensor, counts: torch.Tensor) -> None:
    """Copy the first counts[i] tokens (rounded up to a multiple of eight) of page src_pages[i] to page dst_pages[i], int32 [n] each; pages that
    are not in the cache: nothing."""
    if _ordinary("cache_copy", cache, src_pages, dst_pages, counts) is not None:
        return
    c = _cache(cache)
    dev = cache[0].device
    n = src_pages.shape[0]
    for t, name in ((src_pages, "src_pages"), (dst_pages, "dst_pages"), (counts, "counts")):
        if t is None:
            raise ValueError(f"{name} must be given")
        _check(t, torch.int32, n, name, dev)
    rc = lib().e3_cache_copy(C.byref(c), _ptr(src_pages), _ptr(dst_pages), _ptr(counts), n, _stream(dev))
    if rc != E3_OK:
        raise E3Error(rc, "e3_cache_copy")
