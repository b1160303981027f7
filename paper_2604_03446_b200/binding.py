"""ctypes binding of libmmee.so: the same entry points as include/mmee.h, argument marshalling only.

PyTorch supplies device memory (uint8 CUDA tensors hold the result records) and the stream.
Every step of the search runs in the library's CUDA kernels; if the shared object cannot be
loaded this module raises -- there is no other implementation to fall back to.
"""
from __future__ import annotations

import ctypes as C
import os
import struct

from . import build as _build

OBJ_ENERGY, OBJ_LATENCY, OBJ_EDP, OBJ_ENERGY_LCAP, OBJ_LATENCY_ECAP = 0, 1, 2, 3, 4
TILE_POW2, TILE_ALL_DIVISORS = 0, 1
ORD_NORECOMP2, ORD_ALL6 = 0, 1
FUSE_FUSED, FUSE_SOFTMAX_IN_OP1, FUSE_SEPARATE = 1, 2, 4
F16, BF16 = 0, 1
ACT_SILU, ACT_GELU, ACT_RELU, ACT_SIGMOID = range(4)
MAX_TOPK = 16
NO_INDEX = 2 ** 64 - 1
OK, ERR_ARG, ERR_OVERFLOW, ERR_QUANTUM, ERR_NO_FEASIBLE, ERR_CUDA, ERR_TIMEOUT, ERR_RANGE, ERR_CHECK = range(9)

EXPORTS = ("mmee_create", "mmee_search", "mmee_search_host", "mmee_destroy", "mmee_trim", "mmee_search_static", "mmee_num_candidates", "mmee_num_tilings",
           "mmee_num_rows", "mmee_strerror", "mmee_last_cuda_error", "mmee_eval", "mmee_decode", "mmee_dump_keys", "mmee_filter_flags", "mmee_solve_host", "mmee_pareto_front", "mmee_pareto_front_bs_da", "mmee_search_shapes",
           "mmee_query_vector", "mmee_recompute_flag", "mmee_row_pruning_keep", "mmee_last_search_stats", "mmee_kernel_timing",
           "mmee_alu_peak", "mmee_gated_ffn", "mmee_gated_ffn_backward", "mmee_gated_ffn_workspace",
           "mmee_attention", "mmee_attention_workspace", "mmee_attention_backward", "mmee_attention_backward_workspace",
           "mmee_chain_status", "mmee_chain_wait_limit")


class Workload(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in
                ("batch", "q_heads", "kv_heads", "seq_q", "seq_kv", "d_qk", "d_v", "word_bytes")]


class Arch(C.Structure):
    _fields_ = [("pe_rows", C.c_uint32), ("pe_cols", C.c_uint32), ("n_arrays", C.c_uint32),
                ("gb_bytes", C.c_uint64), ("rf_bytes", C.c_uint64),
                ("dram_words_per_cycle", C.c_uint32),
                ("e_dram_pj", C.c_double), ("e_gb_pj", C.c_double), ("e_rf_pj", C.c_double),
                ("e_mac_pj", C.c_double), ("c_softmax", C.c_double),
                ("energy_quantum_pj", C.c_double)]


class Objective(C.Structure):
    _fields_ = [("objective", C.c_uint32), ("topk", C.c_uint32), ("tiling_set", C.c_uint32),
                ("order_set", C.c_uint32), ("fuse_mask", C.c_uint32), ("row_pruning", C.c_uint32),
                ("t_begin", C.c_uint64), ("t_end", C.c_uint64), ("key_cap", C.c_int64),
                ("stationary_mask", C.c_uint32), ("rf_tiling", C.c_uint32)]


class Result(C.Structure):
    _fields_ = [("idx", C.c_uint64), ("t", C.c_uint64), ("row", C.c_uint32),
                ("bound", C.c_uint32 * 8),
                ("phi", C.c_uint8), ("pi", C.c_uint8), ("beta", C.c_uint8 * 5), ("sm", C.c_uint8 * 2),
                ("recompute", C.c_uint8), ("feasible", C.c_uint8), ("reserved", C.c_uint8 * 5),
                ("status", C.c_int32),
                ("bs_x", C.c_int64 * 5), ("bs_op1", C.c_int64), ("bs_op2", C.c_int64), ("bs", C.c_int64),
                ("da_x", C.c_int64 * 5), ("da_sm", C.c_int64),
                ("br", C.c_int64), ("cyc1", C.c_int64), ("cyc2", C.c_int64),
                ("n", C.c_int64 * 5), ("e_key", C.c_int64), ("l_key", C.c_int64),
                ("edp_key", C.c_double), ("energy_pj", C.c_double), ("latency_cycles", C.c_double),
                ("n_total", C.c_uint64), ("n_feasible", C.c_uint64),
                ("rf_block", C.c_uint32 * 6), ("reserved2", C.c_uint32 * 2)]


class LaunchStats(C.Structure):
    _fields_ = [("kernels_launched", C.c_uint32), ("grid", C.c_uint32), ("block", C.c_uint32),
                ("smem_bytes", C.c_uint32), ("tasks", C.c_uint64),
                ("search_ms", C.c_float), ("finalize_ms", C.c_float),
                ("rows_per_tiling", C.c_uint32), ("rows_evaluated_per_tiling", C.c_uint32),
                ("exact_path_visits", C.c_uint64), ("create_ms", C.c_float), ("reserved", C.c_uint32),
                ("rows_tested", C.c_uint64)]


class Attention(C.Structure):
    _fields_ = [("dtype", C.c_uint32), ("scale", C.c_float), ("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p),
                ("o", C.c_void_p), ("q_stride", C.c_int64 * 3), ("k_stride", C.c_int64 * 3), ("v_stride", C.c_int64 * 3),
                ("o_stride", C.c_int64 * 3), ("lse", C.c_void_p), ("o_rest", C.c_void_p), ("kv_len", C.c_void_p), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_uint64)]


class AttentionGrad(C.Structure):
    _fields_ = [("d_o", C.c_void_p), ("d_q", C.c_void_p), ("d_k", C.c_void_p), ("d_v", C.c_void_p),
                ("d_o_stride", C.c_int64 * 3), ("d_q_stride", C.c_int64 * 3), ("d_k_stride", C.c_int64 * 3),
                ("d_v_stride", C.c_int64 * 3), ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64)]


class GatedFfn(C.Structure):
    _fields_ = [("dtype", C.c_uint32), ("activation", C.c_uint32),
                ("x", C.c_void_p), ("w_gate", C.c_void_p), ("w_up", C.c_void_p), ("w_down", C.c_void_p),
                ("x_stride", C.c_int64), ("w_gate_stride", C.c_int64), ("w_up_stride", C.c_int64),
                ("w_down_stride", C.c_int64), ("hidden", C.c_void_p), ("kept", C.c_void_p), ("y", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64)]


class GatedFfnGrad(C.Structure):
    _fields_ = [("d_y", C.c_void_p), ("d_y_stride", C.c_int64), ("d_x", C.c_void_p), ("d_w_gate", C.c_void_p),
                ("d_w_up", C.c_void_p), ("d_w_down", C.c_void_p)]


RESULT_BYTES = C.sizeof(Result)


class MmeeError(RuntimeError):
    def __init__(self, code: int, where: str):
        msg = library().mmee_strerror(code).decode() if _lib is not None else "status %d" % code
        if code == ERR_CUDA and _lib is not None:
            msg += ": " + library().mmee_last_cuda_error().decode()
        super().__init__("%s: %s (status %d)" % (where, msg, code))
        self.code = code


_lib = None


def library():
    """Load libmmee.so (building it first when its sources are newer and nvcc is present)."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.LIB
    try:
        if _build.is_stale():
            _build.build_library()
    except Exception:
        if not os.path.exists(path):
            raise
    L = C.CDLL(path)
    H = C.c_void_p
    L.mmee_create.argtypes = [C.POINTER(Workload), C.POINTER(Arch), C.POINTER(Objective), C.POINTER(H)]
    L.mmee_search.argtypes = [H, C.c_void_p, C.c_void_p, C.c_void_p]
    L.mmee_search_host.argtypes = [H, C.POINTER(Result), C.POINTER(Result)]
    L.mmee_destroy.argtypes = [H]
    L.mmee_trim.argtypes = []
    L.mmee_search_static.argtypes = [C.POINTER(Workload), C.POINTER(Arch), C.POINTER(Objective),
                                     C.c_void_p, C.c_void_p, C.c_void_p]
    for name in ("mmee_num_candidates", "mmee_num_tilings", "mmee_num_rows"):
        getattr(L, name).argtypes = [H]
        getattr(L, name).restype = C.c_uint64
    L.mmee_strerror.argtypes = [C.c_int]
    L.mmee_strerror.restype = C.c_char_p
    L.mmee_last_cuda_error.argtypes = []
    L.mmee_last_cuda_error.restype = C.c_char_p
    L.mmee_eval.argtypes = [H, C.c_void_p, C.c_uint64, C.c_uint64, C.c_void_p]
    L.mmee_decode.argtypes = [H, C.c_uint64, C.POINTER(Result)]
    L.mmee_dump_keys.argtypes = [H, C.c_void_p, C.c_void_p]
    L.mmee_filter_flags.argtypes = [H, C.c_void_p, C.c_int64, C.c_void_p]
    L.mmee_solve_host.argtypes = [C.POINTER(Workload), C.POINTER(Arch), C.POINTER(Objective),
                                  C.POINTER(Result), C.POINTER(Result),
                                  C.POINTER(C.c_uint64), C.POINTER(C.c_uint64)]
    L.mmee_pareto_front.argtypes = [C.POINTER(Workload), C.POINTER(Arch), C.POINTER(Objective),
                                    C.POINTER(Result), C.c_uint32, C.POINTER(C.c_uint32)]
    L.mmee_pareto_front_bs_da.argtypes = L.mmee_pareto_front.argtypes
    L.mmee_search_shapes.argtypes = [C.POINTER(Workload), C.POINTER(Arch), C.POINTER(Objective),
                                     C.POINTER(C.c_uint32), C.c_uint32, C.POINTER(Result), C.POINTER(C.c_uint32)]
    L.mmee_query_vector.argtypes = [C.c_uint32] * 6 + [C.POINTER(C.c_uint8)]
    L.mmee_recompute_flag.argtypes = [C.c_uint32, C.c_uint32, C.POINTER(C.c_uint32)]
    L.mmee_row_pruning_keep.argtypes = [C.POINTER(Objective), C.POINTER(C.c_uint8), C.c_uint32,
                                        C.POINTER(C.c_uint32)]
    L.mmee_last_search_stats.argtypes = [H, C.POINTER(LaunchStats)]
    L.mmee_kernel_timing.argtypes = [H, C.c_int]
    L.mmee_alu_peak.argtypes = [C.POINTER(C.c_double)]
    L.mmee_gated_ffn.argtypes = [C.POINTER(Workload), C.POINTER(GatedFfn), C.c_void_p]
    L.mmee_gated_ffn_backward.argtypes = [C.POINTER(Workload), C.POINTER(GatedFfn), C.POINTER(GatedFfnGrad), C.c_void_p]
    L.mmee_gated_ffn_workspace.argtypes = [C.POINTER(Workload), C.c_uint32, C.POINTER(C.c_uint64)]
    L.mmee_attention.argtypes = [C.POINTER(Workload), C.POINTER(Attention), C.c_void_p]
    L.mmee_attention_workspace.argtypes = [C.POINTER(Workload), C.POINTER(C.c_uint64)]
    L.mmee_attention_backward.argtypes = [C.POINTER(Workload), C.POINTER(Attention), C.POINTER(AttentionGrad), C.c_void_p]
    L.mmee_attention_backward_workspace.argtypes = [C.POINTER(Workload), C.POINTER(C.c_uint64)]
    L.mmee_chain_status.argtypes = []
    L.mmee_chain_wait_limit.argtypes = [C.c_uint64]
    _lib = L
    return L


def _fill(struct, values: dict):
    struct.__init__(**values)
    return struct


def _inputs(workload: dict, arch: dict, objective: dict):
    return Workload(**workload), Arch(**arch), Objective(**objective)


def _record_space(n: int):
    """Uninitialised host memory for n result records (a ctypes array would be zeroed: 30 us for 4096 records)."""
    import numpy as np
    return np.empty(n * RESULT_BYTES, dtype=np.uint8)


def _records(space, n: int) -> list:
    return list((Result * n).from_buffer_copy(space))


def _check(code: int, where: str):
    if code != OK:
        raise MmeeError(code, where)


def _current_stream():
    """The current stream of the current device as an address; afterwards without the stream object that torch makes for it
    (1.5 us a call)."""
    global _current_stream
    import torch
    ptr = torch.cuda.current_stream().cuda_stream
    device, raw = getattr(torch._C, "_cuda_getDevice", None), getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if device and raw:
        _current_stream = lambda: raw(device())
    return ptr


def _stream_ptr(stream):
    return _current_stream() if stream is None else stream.cuda_stream


def mmee_create(workload: dict, arch: dict, objective: dict) -> C.c_void_p:
    h = C.c_void_p()
    _check(library().mmee_create(_fill(Workload(), workload), _fill(Arch(), arch),
                                 _fill(Objective(), objective), C.byref(h)), "mmee_create")
    return h


def mmee_destroy(handle) -> None:
    _check(library().mmee_destroy(handle), "mmee_destroy")


def mmee_trim() -> None:
    """Free the device scratch and pinned host memory that the library keeps of released handles."""
    _check(library().mmee_trim(), "mmee_trim")


def mmee_num_candidates(handle) -> int:
    return library().mmee_num_candidates(handle)


def mmee_num_tilings(handle) -> int:
    return library().mmee_num_tilings(handle)


def mmee_num_rows(handle) -> int:
    return library().mmee_num_rows(handle)


def result_buffer(n: int, device="cuda"):
    """Uninitialised device buffer for n result records."""
    import torch
    return torch.empty(n * RESULT_BYTES, dtype=torch.uint8, device=device)


def mmee_search(handle, out_best, out_topk=None, stream=None) -> None:
    """Asynchronous: out_best / out_topk are uint8 CUDA tensors from result_buffer()."""
    code = (_lib or library()).mmee_search(handle, _stream_ptr(stream), out_best.data_ptr(),
                                           out_topk.data_ptr() if out_topk is not None else None)
    if code:
        _check(code, "mmee_search")


def mmee_search_host(handle, want_topk: bool = False, topk: int = 0):
    """Search through a planned handle with the records copied to host structs: (best, list of top-k or None)."""
    best = Result()
    arr = (Result * topk)() if want_topk else None
    _check(library().mmee_search_host(handle, C.byref(best), arr), "mmee_search_host")
    return best, (list(arr) if want_topk else None)


def mmee_search_static(workload: dict, arch: dict, objective: dict, out_best, out_topk=None, stream=None) -> None:
    """Search without device allocation: plans on the host, uses the library's fixed scratch.
    Asynchronous; out_best / out_topk are caller-owned uint8 CUDA tensors (result_buffer())."""
    _check(library().mmee_search_static(_fill(Workload(), workload), _fill(Arch(), arch),
                                        _fill(Objective(), objective), _stream_ptr(stream),
                                        C.c_void_p(out_best.data_ptr()),
                                        C.c_void_p(out_topk.data_ptr()) if out_topk is not None else None),
           "mmee_search_static")


def mmee_eval(handle, idx_begin: int, count: int, out, stream=None) -> None:
    _check(library().mmee_eval(handle, _stream_ptr(stream), idx_begin, count, C.c_void_p(out.data_ptr())),
           "mmee_eval")


def mmee_decode(handle, idx: int) -> Result:
    """The mapping behind one candidate index with its full evaluation, as a host record (synchronous)."""
    r = Result()
    _check(library().mmee_decode(handle, idx, C.byref(r)), "mmee_decode")
    return r


def mmee_dump_keys(handle, out_keys, stream=None) -> None:
    """out_keys: int64 CUDA tensor with one entry per candidate of the handle's tiling range."""
    _check(library().mmee_dump_keys(handle, _stream_ptr(stream), C.c_void_p(out_keys.data_ptr())),
           "mmee_dump_keys")


def mmee_filter_flags(handle, threshold_key: int, out_flags, stream=None) -> None:
    """out_flags: uint8 CUDA tensor with 25 entries per task of the handle's tiling range (1 = group flagged)."""
    _check(library().mmee_filter_flags(handle, _stream_ptr(stream), threshold_key, C.c_void_p(out_flags.data_ptr())),
           "mmee_filter_flags")


def mmee_solve_host(workload: dict, arch: dict, objective: dict):
    """(best, topk list, h2d bytes, d2h bytes) with host buffers."""
    k = objective["topk"]
    best, topk = Result(), (Result * k)()
    h2d, d2h = C.c_uint64(), C.c_uint64()
    code = (_lib or library()).mmee_solve_host(*_inputs(workload, arch, objective), best, topk, h2d, d2h)
    if code:
        _check(code, "mmee_solve_host")
    return best, list(topk), h2d.value, d2h.value


def mmee_pareto_front(workload: dict, arch: dict, objective: dict, capacity: int = 256):
    """Energy-latency Pareto front of the whole mapping space: list of Result, by increasing energy."""
    pts = _record_space(capacity)
    n = C.c_uint32()
    _check(library().mmee_pareto_front(*_inputs(workload, arch, objective), C.cast(pts.ctypes.data, C.POINTER(Result)), capacity, n),
           "mmee_pareto_front")
    return _records(pts, n.value)


def mmee_pareto_front_bs_da(workload: dict, arch: dict, objective: dict, capacity: int = 1024):
    """Buffer-size / DRAM-traffic Pareto front of the whole mapping space: list of Result, by decreasing buffer size."""
    pts = _record_space(capacity)
    n = C.c_uint32()
    _check(library().mmee_pareto_front_bs_da(*_inputs(workload, arch, objective), C.cast(pts.ctypes.data, C.POINTER(Result)), capacity,
                                             n),
           "mmee_pareto_front_bs_da")
    return _records(pts, n.value)


def mmee_search_shapes(workload: dict, arch: dict, objective: dict, shapes):
    """One search per logical array shape (rows, cols): (list of Result per shape, index of the best shape or None)."""
    n = len(shapes)
    flat = (C.c_uint32 * (2 * n))(*[v for rc in shapes for v in rc])
    out = (Result * n)()
    best = C.c_uint32()
    _check(library().mmee_search_shapes(*_inputs(workload, arch, objective), flat, n, out, best), "mmee_search_shapes")
    return list(out), (None if best.value == 2 ** 32 - 1 else best.value)


def mmee_query_vector(metric: int, phi: int, pi: int, operand: int, beta: int, recompute: int = 0):
    q = (C.c_uint8 * 8)()
    _check(library().mmee_query_vector(metric, phi, pi, operand, beta, recompute, q), "mmee_query_vector")
    return list(q)


def mmee_row_pruning_keep(objective: dict):
    """List of 0/1 per row of a tiling: the rows evaluated under objective.row_pruning = 1."""
    rows = C.c_uint32()
    buf = (C.c_uint8 * 26250)()
    _check(library().mmee_row_pruning_keep(_fill(Objective(), objective), buf, 26250, C.byref(rows)),
           "mmee_row_pruning_keep")
    return list(buf[:rows.value])


def mmee_recompute_flag(pi: int, beta_c: int) -> int:
    f = C.c_uint32()
    _check(library().mmee_recompute_flag(pi, beta_c, C.byref(f)), "mmee_recompute_flag")
    return f.value


def mmee_last_search_stats(handle) -> LaunchStats:
    s = LaunchStats()
    _check(library().mmee_last_search_stats(handle, C.byref(s)), "mmee_last_search_stats")
    return s


def mmee_kernel_timing(handle, enable: bool) -> None:
    _check(library().mmee_kernel_timing(handle, int(enable)), "mmee_kernel_timing")


def mmee_alu_peak():
    out = (C.c_double * 4)()
    _check(library().mmee_alu_peak(out), "mmee_alu_peak")
    return list(out)


def _refuse(where: str, why: str):
    raise MmeeError(ERR_ARG, "%s: %s" % (where, why))


_torch = _forward_mode = None
_type_codes = {}


def _no_graph(where, tensors):
    """Refuses tensors that autograd, or a forward-mode level, would carry on from: the call's results would silently drop out."""
    recorded = _torch.is_grad_enabled() and any(t.requires_grad for t in tensors)
    if recorded or (_forward_mode._current_level >= 0 and any(_forward_mode.unpack_dual(t).tangent is not None for t in tensors)):
        _refuse(where, "tensors that want a gradient: automatic differentiation does not see this call (under torch.no_grad(), or on "
                       "detached tensors, call it and its _backward yourself)")


def _chain_code(where: str, rank: int, *tensors):
    """The type code that the tensors of one call share: CUDA tensors of one 16-bit type on one device, of `rank` dimensions with
    the last one contiguous, none of which takes part in an automatic differentiation."""
    global _torch, _forward_mode
    if _torch is None:
        import torch
        import torch.autograd.forward_ad
        _forward_mode = torch.autograd.forward_ad
        _type_codes.update({torch.bfloat16: BF16, torch.float16: F16})
        _torch = torch                                 # (last: another thread's first call goes by it)
    try:
        dtype, at = tensors[0].dtype, tensors[0].get_device()
        code, graph = _type_codes[dtype], False
        for t in tensors:
            steps = t.stride()
            graph = graph or t.requires_grad
            if t.dtype is not dtype or t.get_device() != at or len(steps) != rank or (steps[-1] != 1 and t.shape[-1] > 1):
                break
        else:
            if graph or _forward_mode._current_level >= 0:
                _no_graph(where, tensors)
            if at >= 0:
                return code
    except (AttributeError, KeyError, TypeError):
        pass
    _refuse(where, "tensors of %d dimensions, the last one contiguous, of bfloat16 or float16 all, on one CUDA device are wanted" % rank)


def _current_device():
    """The current device's number; afterwards without torch's own wrapper around the question (1 us a call)."""
    global _current_device
    import torch
    n = torch.cuda.current_device()
    _current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    return n


def _there(where, t, stream):
    """Makes the tensor's device and the stream current: launches and the memory that a call takes are theirs."""
    if stream is None:
        return _torch.cuda.device(t.device)
    if stream.device != t.device:
        _refuse(where, "a stream of the tensors' device is wanted")
    return _torch.cuda.stream(stream)


# The call structs as bytes, in the layouts of Workload, Attention, AttentionGrad, GatedFfn and GatedFfnGrad: filling a
# ctypes struct field by field takes several times as long (the calls below are made once per layer and token).
_WORKLOAD, _ATTENTION, _ATTENTION_GRAD = struct.Struct("=8I").pack, struct.Struct("=If4Q12q5Q").pack, struct.Struct("=4Q12q2Q").pack
_FFN, _FFN_GRAD = struct.Struct("=2I4Q4q5Q").pack, struct.Struct("=Qq4Q").pack


class _ChainCalls:
    """The library's chain calls with structs given as bytes."""

    def __init__(self):
        L = library()
        for name, n in (("attention", 2), ("attention_backward", 3), ("gated_ffn", 2), ("gated_ffn_backward", 3)):
            f = L["mmee_" + name]
            f.argtypes = [C.c_char_p] * n + [C.c_void_p]
            setattr(self, name, f)
        for name in ("attention_workspace", "attention_backward_workspace", "gated_ffn_workspace"):
            f = L["mmee_" + name]
            f.argtypes = [C.c_char_p] + [C.c_uint32] * (name == "gated_ffn_workspace") + [C.c_void_p]
            setattr(self, name, f)


_chain_calls = None


def _chain():
    global _chain_calls
    if _chain_calls is None:
        _chain_calls = _ChainCalls()
    return _chain_calls


def _space(ask, like, where, *args):
    """Workspace for one call (None: it needs none) and its size."""
    need = C.c_uint64()
    code = ask(*args, C.addressof(need))
    if code:
        _check(code, where)
    return (like.new_empty(need.value, dtype=_torch.uint8) if need.value else None), need.value


def _attention_sizes(where, q, k, v, kv_len):
    """(batch, q_heads, kv_heads, seq_q, seq_kv, d_qk, d_v) of tensors that fit each other."""
    (batch, seq_q, q_heads, d_qk), (b, seq_kv, kv_heads, d) = q.shape, k.shape
    bv, sv, hv, d_v = v.shape
    if b != batch or bv != batch or sv != seq_kv or hv != kv_heads or d != d_qk:
        _refuse(where, "q is (batch, tokens, heads, d), k and v have one batch, length and number of heads, q and k one width")
    if kv_len is not None:
        if not (isinstance(kv_len, _torch.Tensor) and kv_len.dtype is _torch.int32 and kv_len.shape == (batch,) and
                kv_len.get_device() == q.get_device() and kv_len.is_contiguous()):
            _refuse(where, "kv_len is a contiguous int32 tensor, one entry per sequence, on the tensors' device")
    return batch, q_heads, kv_heads, seq_q, seq_kv, d_qk, d_v


def mmee_attention(q, k, v, kv_len=None, scale=None, stream=None):
    """softmax(scale q k^T) v over each sequence's first kv_len keys: (o, saved).  q: (batch, tokens, q_heads, d_qk), k: (batch, keys,
    kv_heads, d_qk), v: (batch, keys, kv_heads, d_v), bfloat16 or float16; kv_len: int32 tensor with an entry per sequence, None: all keys;
    scale: d_qk ** -0.5 unless given.  saved: what mmee_attention_backward needs; attention_lse(saved, o) is the part of it that is
    of use elsewhere.  Not recorded by autograd: tensors that require a gradient are refused unless under torch.no_grad().  Asynchronous."""
    where = "mmee_attention"
    code = _chain_code(where, 4, q, k, v)
    if stream is not None or _current_device() != q.get_device():
        with _there(where, q, stream):
            return mmee_attention(q, k, v, kv_len, scale)
    batch, q_heads, kv_heads, seq_q, seq_kv, d_qk, d_v = _attention_sizes(where, q, k, v, kv_len)
    try:
        calls = _chain()
        w = _WORKLOAD(batch, q_heads, kv_heads, seq_q, seq_kv, d_qk, d_v, 2)
        space, need = _space(calls.attention_workspace, q, where, w)
        o = q.new_empty((batch, seq_q, q_heads, d_v))
        rows = batch * seq_q * q_heads
        ahead = (rows + 3) // 4 * 4                        # (what follows the rows' sums starts on sixteen bytes)
        saved = q.new_empty(ahead + rows * d_v // 2, dtype=_torch.float32)
        at = saved.data_ptr()
        a = _ATTENTION(code, (d_qk or 1) ** -0.5 if scale is None else scale, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                       *q.stride()[:3], *k.stride()[:3], *v.stride()[:3], seq_q * q_heads * d_v, q_heads * d_v, d_v, at, at + 4 * ahead,
                       0 if kv_len is None else kv_len.data_ptr(), space.data_ptr() if need else 0, need)
        code = calls.attention(w, a, _current_stream())
    except (struct.error, OverflowError) as e:
        _refuse(where, "an argument is no number that the call holds (%s)" % e)
    if code:
        _check(code, where)
    return o, saved


def attention_lse(saved, o):
    """log sum exp(scale q k^T) of every row, float32 (batch, q_heads, tokens), out of what mmee_attention returned beside o."""
    batch, seq_q, q_heads, _ = o.shape
    return saved[:batch * q_heads * seq_q].view(batch, q_heads, seq_q)


def mmee_attention_backward(d_o, q, k, v, o, saved, kv_len=None, scale=None, stream=None):
    """The gradients (d_q, d_k, d_v) of mmee_attention for a gradient d_o of o; o and saved are what the forward call with the same
    tensors returned.  Keys behind a sequence's end get zeros.  Asynchronous."""
    where = "mmee_attention_backward"
    code = _chain_code(where, 4, q, k, v, o, d_o)
    if stream is not None or _current_device() != q.get_device():
        with _there(where, q, stream):
            return mmee_attention_backward(d_o, q, k, v, o, saved, kv_len, scale)
    batch, q_heads, kv_heads, seq_q, seq_kv, d_qk, d_v = _attention_sizes(where, q, k, v, kv_len)
    if o.shape != (batch, seq_q, q_heads, d_v) or d_o.shape != o.shape:
        _refuse(where, "o and d_o are (batch, tokens, q_heads, d_v)")
    rows = batch * seq_q * q_heads
    ahead = (rows + 3) // 4 * 4
    if not (isinstance(saved, _torch.Tensor) and saved.shape == (ahead + rows * d_v // 2,) and saved.dtype is _torch.float32 and
            saved.get_device() == q.get_device() and saved.is_contiguous()):
        _refuse(where, "saved is what the forward call for these tensors returned")
    at = saved.data_ptr()
    try:
        calls = _chain()
        w = _WORKLOAD(batch, q_heads, kv_heads, seq_q, seq_kv, d_qk, d_v, 2)
        space, need = _space(calls.attention_backward_workspace, q, where, w)
        d_q, d_k, d_v_ = q.new_empty(q.shape), q.new_empty(k.shape), q.new_empty(v.shape)
        a = _ATTENTION(code, (d_qk or 1) ** -0.5 if scale is None else scale, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                       *q.stride()[:3], *k.stride()[:3], *v.stride()[:3], *o.stride()[:3], at, at + 4 * ahead,
                       0 if kv_len is None else kv_len.data_ptr(), 0, 0)
        g = _ATTENTION_GRAD(d_o.data_ptr(), d_q.data_ptr(), d_k.data_ptr(), d_v_.data_ptr(), *d_o.stride()[:3], *d_q.stride()[:3],
                            *d_k.stride()[:3], *d_v_.stride()[:3], space.data_ptr(), need)
        code = calls.attention_backward(w, a, g, _current_stream())
    except (struct.error, OverflowError) as e:
        _refuse(where, "an argument is no number that the call holds (%s)" % e)
    if code:
        _check(code, where)
    return d_q, d_k, d_v_


def _ffn_sizes(where, x, w_gate, w_up, w_down):
    """(tokens, inner, in, out) of tensors that fit each other."""
    (tokens, d_in), (d_ff, d), (d_out, inner) = x.shape, w_gate.shape, w_down.shape
    if d != d_in or w_up.shape != (d_ff, d_in) or inner != d_ff:
        _refuse(where, "w_gate and w_up are (inner, in), w_down is (out, inner), x is (tokens, in)")
    return tokens, d_ff, d_in, d_out


def mmee_gated_ffn(x, w_gate, w_up, w_down, activation: int = ACT_SILU, save: bool = False, stream=None):
    """y = (act(x w_gate^T) * (x w_up^T)) w_down^T: (y, saved).  x: (tokens, in), w_gate and w_up: (inner, in), w_down: (out, inner),
    bfloat16 or float16.  saved: what mmee_gated_ffn_backward needs where `save`, otherwise None.  Not recorded by autograd, as
    mmee_attention.  Asynchronous."""
    where = "mmee_gated_ffn"
    code = _chain_code(where, 2, x, w_gate, w_up, w_down)
    if stream is not None or _current_device() != x.get_device():
        with _there(where, x, stream):
            return mmee_gated_ffn(x, w_gate, w_up, w_down, activation, save)
    tokens, d_ff, d_in, d_out = _ffn_sizes(where, x, w_gate, w_up, w_down)
    try:
        calls = _chain()
        w = _WORKLOAD(1, 1, 1, tokens, d_ff, d_in, d_out, 2)
        hidden, y = x.new_empty((tokens, d_ff)), x.new_empty((tokens, d_out))
        kept = x.new_empty((2, tokens, d_ff), dtype=_torch.float32) if save else None
        space, need = _space(calls.gated_ffn_workspace, x, where, w, 0)
        f = _FFN(code, activation, x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr(), x.stride(0), w_gate.stride(0),
                 w_up.stride(0), w_down.stride(0), hidden.data_ptr(), kept.data_ptr() if save else 0, y.data_ptr(), space.data_ptr() if need else 0, need)
        code = calls.gated_ffn(w, f, _current_stream())
    except (struct.error, OverflowError) as e:
        _refuse(where, "an argument is no number that the call holds (%s)" % e)
    if code:
        _check(code, where)
    return y, ((hidden, kept) if save else None)


def mmee_gated_ffn_backward(d_y, x, w_gate, w_up, w_down, saved, activation: int = ACT_SILU, stream=None):
    """The gradients (d_x, d_w_gate, d_w_up, d_w_down) of mmee_gated_ffn for a gradient d_y of y; `saved` is what the forward call
    with the same x, weights and activation returned.  Asynchronous."""
    where = "mmee_gated_ffn_backward"
    if not isinstance(saved, tuple) or len(saved) != 2:
        _refuse(where, "saved is what the forward call with save=True returned")
    code = _chain_code(where, 2, x, w_gate, w_up, w_down, d_y, saved[0])
    if stream is not None or _current_device() != x.get_device():
        with _there(where, x, stream):
            return mmee_gated_ffn_backward(d_y, x, w_gate, w_up, w_down, saved, activation)
    tokens, d_ff, d_in, d_out = _ffn_sizes(where, x, w_gate, w_up, w_down)
    hidden, kept = saved
    if d_y.shape != (tokens, d_out):
        _refuse(where, "d_y is (tokens, out)")
    if (hidden.shape != (tokens, d_ff) or not hidden.is_contiguous() or getattr(kept, "shape", None) != (2, tokens, d_ff) or
            kept.dtype is not _torch.float32 or not kept.is_contiguous() or kept.get_device() != x.get_device()):
        _refuse(where, "saved is not what the forward call for these tensors returned")
    try:
        calls = _chain()
        w = _WORKLOAD(1, 1, 1, tokens, d_ff, d_in, d_out, 2)
        space, need = _space(calls.gated_ffn_workspace, x, where, w, 1)
        grads = tuple([x.new_empty(t.shape) for t in (x, w_gate, w_up, w_down)])
        f = _FFN(code, activation, x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr(), x.stride(0), w_gate.stride(0),
                 w_up.stride(0), w_down.stride(0), hidden.data_ptr(), kept.data_ptr(), 0,
                 space.data_ptr() if need else 0, need)
        g = _FFN_GRAD(d_y.data_ptr(), d_y.stride(0), *[t.data_ptr() for t in grads])
        code = calls.gated_ffn_backward(w, f, g, _current_stream())
    except (struct.error, OverflowError) as e:
        _refuse(where, "an argument is no number that the call holds (%s)" % e)
    if code:
        _check(code, where)
    return grads


def mmee_chain_status() -> None:
    """Raises once after a wait inside a chain's kernel ran out (its outputs are not a result).  Waits for the device."""
    _check(library().mmee_chain_status(), "mmee_chain_status")


def mmee_chain_wait_limit(seconds: float = 4.0) -> None:
    """How long a wait for a barrier in the chains' kernels on the current device may last.  Waits for the device."""
    if not 0 <= seconds < 2 ** 32:
        _refuse("mmee_chain_wait_limit", "seconds from nothing to 2^32 are wanted")
    _check(library().mmee_chain_wait_limit(int(seconds * 1e9)), "mmee_chain_wait_limit")


def read_results(buf, n: int):
    """Copy n records from a device buffer to host Result structs (synchronises)."""
    raw = bytes(buf.cpu().numpy().tobytes())
    return [Result.from_buffer_copy(raw[i * RESULT_BYTES:(i + 1) * RESULT_BYTES]) for i in range(n)]
