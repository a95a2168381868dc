"""Thin ctypes binding over libgrouter.so: argument marshalling only.

Every function mirrors the C entry point of the same name in include/grouter.h and takes torch tensors
that already live on the GPU (PyTorch is used for device memory and streams, nothing else).  There is
no fallback: if the HIP library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgrouter.so")
_lib = None

OK, ERR_INVALID_ARG, ERR_WORKSPACE_TOO_SMALL, ERR_INDEX_OUT_OF_RANGE, ERR_HIP = 0, -1, -2, -3, -4
IDX_INT32, IDX_UINT8 = 0, 1
PHASES = ("plan", "permute", "gateup", "down", "combine", "dO", "dH", "dW2", "dW13", "dXp", "dX_reduce", "affinity",
          "placement", "coactivation", "fold", "sample_stats", "route", "route_bwd", "balance", "gate_bwd", "adamw")
FP32, BF16, FP16 = 0, 1, 2
GATE_SOFTMAX_SELECTED, GATE_SOFTMAX_ALL, GATE_SIGMOID, GATE_SIGMOID_NORMALISED = 0, 1, 2, 3
ADAMW_FP32, ADAMW_MASTER, ADAMW_BF16 = 0, 1, 2

EXPORTS = (
    "grouter_strerror", "grouter_last_hip_error", "grouter_plan_bytes", "grouter_ctx_bytes",
    "grouter_bwd_scratch_bytes", "grouter_plan_build", "grouter_plan_views", "grouter_plan_status",
    "grouter_permute", "grouter_combine", "grouter_moe_fwd", "grouter_moe_bwd", "grouter_timing_enable",
    "grouter_timing_read", "grouter_phase_name", "grouter_fwd_only_bytes", "grouter_moe_fwd_only", "grouter_affinity", "grouter_sample_placement",
    "grouter_coactivation", "grouter_fold_groups", "grouter_fold_weights", "grouter_static_ws_bytes",
    "grouter_moe_fwd_only_static", "grouter_sample_stats", "grouter_plan_set_gates", "grouter_mfma_probe",
    "grouter_route", "grouter_route_bwd", "grouter_balance_bytes", "grouter_balance", "grouter_gate_bwd", "grouter_moe_gate_bwd",
    "grouter_adamw_hyper_set", "grouter_adamw",
)


class GrouterError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = lib().grouter_strerror(code).decode()
        if code == ERR_HIP:
            msg += f" (hipError_t {lib().grouter_last_hip_error()})"
        super().__init__(f"{where}: {msg}")


class AdamWHyper(ctypes.Structure):
    """One step's numbers (grouter_adamw_hyper), made by grouter_adamw_hyper."""

    _fields_ = [(n, ctypes.c_float) for n in ("beta1", "one_minus_beta1", "beta2", "one_minus_beta2", "inv_root_correction", "eps",
                                              "step_size", "decay", "grad_scale")] + [("seed", ctypes.c_uint32), ("reserved", ctypes.c_uint32 * 2)]

    def tensor(self):
        """The same as a uint8 CPU tensor of 48 bytes, to be copied into the device buffer of a captured step."""
        import torch

        return torch.frombuffer(bytearray(bytes(self)), dtype=torch.uint8)


class _AdamWTensor(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("param", "master", "grad", "m", "v", "m_exp", "v_exp")] + [("n", ctypes.c_int64)]


def lib():
    """Load libgrouter.so (built in-tree by paper_2603_06626_amd.build); raises if it is absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -c 'import __graft_entry__ as g; g.build()'` "
                               "(there is no non-HIP fallback)")
        L = ctypes.CDLL(LIB_PATH)
        i64, i32, vp, sz = ctypes.c_int64, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t
        L.grouter_strerror.argtypes = [i32]
        L.grouter_strerror.restype = ctypes.c_char_p
        L.grouter_phase_name.argtypes = [i32]
        L.grouter_phase_name.restype = ctypes.c_char_p
        L.grouter_last_hip_error.restype = i32
        L.grouter_plan_bytes.argtypes = [i64, i32, i32]
        L.grouter_plan_bytes.restype = sz
        L.grouter_ctx_bytes.argtypes = [i64, i32, i32, i32]
        L.grouter_ctx_bytes.restype = sz
        L.grouter_bwd_scratch_bytes.argtypes = [i64, i32, i32, i32]
        L.grouter_bwd_scratch_bytes.restype = sz
        L.grouter_plan_build.argtypes = [vp, i32, i64, i32, i32, vp, sz, vp]
        L.grouter_plan_set_gates.argtypes = [vp, i64, i32, i32, vp, vp]
        L.grouter_plan_set_gates.restype = i32
        L.grouter_plan_views.argtypes = [vp, i64, i32, i32] + [ctypes.POINTER(vp)] * 4
        L.grouter_plan_status.argtypes = [vp, vp]
        L.grouter_permute.argtypes = [vp, i64, i32, i32, i32, vp, vp, vp, vp]
        L.grouter_combine.argtypes = [vp, i64, i32, i32, i32, vp, vp, vp, vp]
        L.grouter_moe_fwd.argtypes = [vp, i64, i32, i32, i32, i32] + [vp] * 7 + [sz, vp]
        L.grouter_fwd_only_bytes.argtypes = [i64, i32, i32, i32]
        L.grouter_fwd_only_bytes.restype = sz
        L.grouter_moe_fwd_only.argtypes = [vp, i64, i32, i32, i32, i32] + [vp] * 7 + [sz, vp]
        L.grouter_moe_fwd_only.restype = i32
        L.grouter_static_ws_bytes.argtypes = []
        L.grouter_static_ws_bytes.restype = sz
        L.grouter_moe_fwd_only_static.argtypes = [vp, i64, i32, i32, i32, i32] + [vp] * 6 + [vp]
        L.grouter_moe_fwd_only_static.restype = i32
        L.grouter_moe_bwd.argtypes = [vp, i64, i32, i32, i32, i32] + [vp] * 7 + [sz] + [vp] * 5 + [sz, vp]
        L.grouter_timing_enable.argtypes = [i32]
        L.grouter_timing_read.argtypes = [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(i64)]
        L.grouter_affinity.argtypes = [vp, i32, i64, i32, i32, i32, vp, vp, vp, vp, vp]
        L.grouter_sample_placement.argtypes = [vp, i32, i64, i32, i32, i32, vp, i32, vp, vp, vp]
        L.grouter_sample_stats.argtypes = [vp, i32, i64, i32, i32, i32, vp, vp, vp, vp, vp, i32, vp, vp, vp]
        L.grouter_sample_stats.restype = i32
        L.grouter_coactivation.argtypes = [vp, i32, i64, i32, i32, vp, vp]
        L.grouter_fold_groups.argtypes = [vp, i32, i32, vp, vp]
        L.grouter_mfma_probe.argtypes = [i32, i32, i32, vp, sz, vp]
        L.grouter_fold_weights.argtypes = [vp, vp, i32, i32, i32, vp, vp]
        f32, f64, u32 = ctypes.c_float, ctypes.c_double, ctypes.c_uint32
        L.grouter_route.argtypes = [vp, i32, i64, i64, i32, i32, i32, vp, vp, i32, vp, vp]
        L.grouter_route_bwd.argtypes = [vp, i32, i64, i64, i32, i32, vp, vp, i32, i32, vp, vp, i64, vp, vp, i32, i64, vp]
        L.grouter_balance_bytes.argtypes = [i64, i32, i64]
        L.grouter_balance_bytes.restype = sz
        L.grouter_balance.argtypes = [vp, i32, i64, i64, i32, i32, i32, vp, vp, i32, vp, i64, f32, vp, vp, vp, vp, vp, sz, vp]
        L.grouter_gate_bwd.argtypes = [vp, i64, i32, i32, i32, vp, vp, vp, vp]
        L.grouter_moe_gate_bwd.argtypes = [vp, i64, i32, i32, i32, i32, vp, vp, sz, vp, vp]
        L.grouter_adamw_hyper_set.argtypes = [f64, f64, f64, f64, f64, i64, f64, u32, ctypes.POINTER(AdamWHyper)]
        L.grouter_adamw.argtypes = [ctypes.POINTER(_AdamWTensor), i32, i32, i32, i32, ctypes.POINTER(AdamWHyper), vp, vp, vp]
        for name in ("grouter_route", "grouter_route_bwd", "grouter_balance", "grouter_gate_bwd", "grouter_moe_gate_bwd",
                     "grouter_adamw_hyper_set", "grouter_adamw"):
            getattr(L, name).restype = i32
        for name in ("grouter_plan_build", "grouter_plan_views", "grouter_plan_status", "grouter_permute",
                     "grouter_combine", "grouter_moe_fwd", "grouter_moe_bwd", "grouter_timing_enable",
                     "grouter_timing_read", "grouter_affinity", "grouter_sample_placement", "grouter_coactivation",
                     "grouter_fold_groups", "grouter_fold_weights"):
            getattr(L, name).restype = i32
        _lib = L
    return _lib


def _check(code: int, where: str):
    if code != OK:
        raise GrouterError(code, where)


def _p(t):
    return None if t is None else t.data_ptr()     # (the argument types make a pointer of it)


def _find_raw_stream():
    """How to get the current stream's handle: from torch itself, since building a torch.cuda.Stream for it on every call costs
    about as much as a kernel launch."""
    import torch

    get, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), torch.cuda.current_device   # (the latter initialises torch.cuda)
    if get is None:
        return lambda: torch.cuda.current_stream().cuda_stream
    return lambda: get(device())


_raw_stream = None


def _stream(stream=None):
    global _raw_stream
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        _raw_stream = _find_raw_stream()
    return _raw_stream()


def _find_current():
    """(the current device, the handle of a device's current stream), from torch itself where it has them: its public functions look
    after initialisation on every call, which a tensor on the GPU stands for."""
    import torch

    device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    handle = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda d: torch.cuda.current_stream(d).cuda_stream)
    return device, handle


_current = None


def _stream_for(t, stream=None):
    """The stream to enqueue on: the given one, or the current one of the current device, which has to be the one that t is on."""
    global _current
    at = t.get_device()
    if stream is not None:
        device, handle = stream.device.index, stream.cuda_stream
    else:
        if _current is None:
            _current = _find_current()
        device = _current[0]()
        handle = _current[1](device)
    if at != device:
        raise ValueError(f"the tensors are on device {at}, the stream is device {device}'s")
    return handle


def _dev(t, name, dtype=None):
    if not (t.is_cuda and t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous GPU tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must have dtype {dtype}")
    return t


def grouter_plan_bytes(T, k, E) -> int:
    return int(lib().grouter_plan_bytes(T, k, E))


def grouter_ctx_bytes(T, k, d, f) -> int:
    return int(lib().grouter_ctx_bytes(T, k, d, f))


def grouter_bwd_scratch_bytes(T, k, d, f) -> int:
    return int(lib().grouter_bwd_scratch_bytes(T, k, d, f))


def grouter_plan_build(topk_idx, E, plan_ws, stream=None):
    """topk_idx: [T,k] int32 or uint8 GPU tensor; plan_ws: uint8 GPU tensor of >= grouter_plan_bytes."""
    import torch

    _dev(topk_idx, "topk_idx")
    if topk_idx.dtype == torch.int32:
        dt = IDX_INT32
    elif topk_idx.dtype == torch.uint8:
        dt = IDX_UINT8
    else:
        raise ValueError("topk_idx must be int32 or uint8")
    T, k = topk_idx.shape
    _check(lib().grouter_plan_build(_p(topk_idx), dt, T, k, E, _p(_dev(plan_ws, "plan_ws")), plan_ws.numel(),
                                    _stream(stream)), "grouter_plan_build")


def grouter_plan_set_gates(plan_ws, E, gate_w, stream=None):
    """Lay the gate weights [T,k] (bf16) out in the plan; the layer calls then take gate_w=None and k."""
    import torch

    T, k = gate_w.shape
    _dev(gate_w, "gate_w", torch.bfloat16)
    _check(lib().grouter_plan_set_gates(_p(_dev(plan_ws, "plan_ws")), T, k, E, _p(gate_w), _stream(stream)),
           "grouter_plan_set_gates")


def grouter_plan_views(plan_ws, T, k, E):
    """(counts[E], offsets[E+1], row_to_src[N], src_to_row[N]) as int32 GPU tensors aliasing plan_ws."""
    import torch

    ptrs = [ctypes.c_void_p() for _ in range(4)]
    _check(lib().grouter_plan_views(_p(plan_ws), T, k, E, *[ctypes.byref(p) for p in ptrs]), "grouter_plan_views")
    base = plan_ws.data_ptr()
    as_i32 = plan_ws.view(torch.int32)
    out = []
    for p, n in zip(ptrs, (E, E + 1, T * k, T * k)):
        off = (p.value - base) // 4
        out.append(as_i32[off:off + n])
    return tuple(out)


def grouter_plan_status(plan_ws, stream=None):
    _check(lib().grouter_plan_status(_p(plan_ws), _stream(stream)), "grouter_plan_status")


def grouter_permute(plan_ws, T, k, E, inp, gate_w, out, stream=None):
    d = inp.shape[1]
    _check(lib().grouter_permute(_p(plan_ws), T, k, E, d, _p(_dev(inp, "in")), _p(gate_w), _p(_dev(out, "out")),
                                 _stream(stream)), "grouter_permute")


def grouter_combine(plan_ws, T, k, E, inp, gate_w, out, stream=None):
    d = inp.shape[1]
    _check(lib().grouter_combine(_p(plan_ws), T, k, E, d, _p(_dev(inp, "in")), _p(gate_w), _p(_dev(out, "out")),
                                 _stream(stream)), "grouter_combine")


def grouter_moe_fwd(plan_ws, x, gate_w, W1, W3, W2, y, ctx_ws, stream=None, k=None):
    """gate_w=None: use the gates attached to the plan with grouter_plan_set_gates (k must then be given)."""
    import torch

    bf = torch.bfloat16
    T, d = x.shape
    k = gate_w.shape[1] if gate_w is not None else int(k)
    E, d1, f = W1.shape
    if d1 != d or W3.shape != (E, d, f) or W2.shape != (E, f, d) or y.shape != (T, d):
        raise ValueError("shape mismatch")
    for t, n in ((x, "x"), (gate_w, "gate_w"), (W1, "W1"), (W3, "W3"), (W2, "W2"), (y, "y")):
        if t is not None:
            _dev(t, n, bf)
    _check(lib().grouter_moe_fwd(_p(plan_ws), T, k, E, d, f, _p(x), _p(gate_w), _p(W1), _p(W3), _p(W2), _p(y),
                                 _p(_dev(ctx_ws, "ctx_ws")), ctx_ws.numel(), _stream(stream)), "grouter_moe_fwd")


def grouter_fwd_only_bytes(T, k, d, f) -> int:
    return int(lib().grouter_fwd_only_bytes(T, k, d, f))


def grouter_moe_fwd_only(plan_ws, x, gate_w, W1, W3, W2, y, ws, stream=None, k=None):
    import torch

    bf = torch.bfloat16
    T, d = x.shape
    k = gate_w.shape[1] if gate_w is not None else int(k)
    E, d1, f = W1.shape
    if d1 != d or W3.shape != (E, d, f) or W2.shape != (E, f, d) or y.shape != (T, d):
        raise ValueError("shape mismatch")
    for t, n in ((x, "x"), (gate_w, "gate_w"), (W1, "W1"), (W3, "W3"), (W2, "W2"), (y, "y")):
        if t is not None:
            _dev(t, n, bf)
    _check(lib().grouter_moe_fwd_only(_p(plan_ws), T, k, E, d, f, _p(x), _p(gate_w), _p(W1), _p(W3), _p(W2), _p(y),
                                      _p(_dev(ws, "ws")), ws.numel(), _stream(stream)), "grouter_moe_fwd_only")


def grouter_static_ws_bytes() -> int:
    return int(lib().grouter_static_ws_bytes())


def grouter_moe_fwd_only_static(plan_ws, x, gate_w, W1, W3, W2, y, stream=None, k=None):
    """grouter_moe_fwd_only with the library's static device array as workspace (allocates nothing)."""
    import torch

    bf = torch.bfloat16
    T, d = x.shape
    k = gate_w.shape[1] if gate_w is not None else int(k)
    E, d1, f = W1.shape
    if d1 != d or W3.shape != (E, d, f) or W2.shape != (E, f, d) or y.shape != (T, d):
        raise ValueError("shape mismatch")
    for t, n in ((x, "x"), (gate_w, "gate_w"), (W1, "W1"), (W3, "W3"), (W2, "W2"), (y, "y")):
        if t is not None:
            _dev(t, n, bf)
    _check(lib().grouter_moe_fwd_only_static(_p(plan_ws), T, k, E, d, f, _p(x), _p(gate_w), _p(W1), _p(W3), _p(W2),
                                             _p(y), _stream(stream)), "grouter_moe_fwd_only_static")


def grouter_moe_bwd(plan_ws, x, gate_w, W1, W3, W2, dY, ctx_ws, dX, dW1, dW3, dW2, scratch_ws, stream=None, k=None):
    import torch

    bf = torch.bfloat16
    T, d = x.shape
    k = gate_w.shape[1] if gate_w is not None else int(k)
    E, _, f = W1.shape
    if (dY.shape != (T, d) or dX.shape != (T, d) or dW1.shape != (E, d, f)
            or dW3.shape != (E, d, f) or dW2.shape != (E, f, d)):
        raise ValueError("shape mismatch")
    for t, n in ((x, "x"), (gate_w, "gate_w"), (W1, "W1"), (W3, "W3"), (W2, "W2"), (dY, "dY"), (dX, "dX"),
                 (dW1, "dW1"), (dW3, "dW3"), (dW2, "dW2")):
        if t is not None:
            _dev(t, n, bf)
    _check(lib().grouter_moe_bwd(_p(plan_ws), T, k, E, d, f, _p(x), _p(gate_w), _p(W1), _p(W3), _p(W2), _p(dY),
                                 _p(_dev(ctx_ws, "ctx_ws")), ctx_ws.numel(), _p(dX), _p(dW1), _p(dW3), _p(dW2),
                                 _p(_dev(scratch_ws, "scratch_ws")), scratch_ws.numel(), _stream(stream)),
           "grouter_moe_bwd")


def _idx_dtype(t):
    import torch

    if t.dtype == torch.int32:
        return IDX_INT32
    if t.dtype == torch.uint8:
        return IDX_UINT8
    raise ValueError("topk_idx must be int32 or uint8")


def grouter_affinity(topk_idx, E, counts, entropy_bits, loads, maxvio, stream=None):
    """topk_idx [S,L,k]; counts int32 [S,E]; entropy_bits float64 [S]; loads int64 [E]; maxvio float64 [1]."""
    import torch

    S, L, k = topk_idx.shape
    _dev(topk_idx, "topk_idx")
    _dev(counts, "counts", torch.int32)
    _dev(entropy_bits, "entropy_bits", torch.float64)
    _dev(loads, "loads", torch.int64)
    _dev(maxvio, "maxvio", torch.float64)
    if counts.shape != (S, E) or entropy_bits.numel() != S or loads.numel() != E or maxvio.numel() != 1:
        raise ValueError("shape mismatch")
    _check(lib().grouter_affinity(_p(topk_idx), _idx_dtype(topk_idx), S, L, k, E, _p(counts), _p(entropy_bits),
                                  _p(loads), _p(maxvio), _stream(stream)), "grouter_affinity")


def grouter_sample_placement(topk_idx, E, expert_nodes, n_nodes, comm, best_node, stream=None):
    """topk_idx [S,L,k]; expert_nodes int64 [E] (bit n = expert on node n); comm int32 [S,n_nodes]; best_node int32 [S]."""
    import torch

    S, L, k = topk_idx.shape
    _dev(topk_idx, "topk_idx")
    _dev(expert_nodes, "expert_nodes", torch.int64)
    _dev(comm, "comm", torch.int32)
    _dev(best_node, "best_node", torch.int32)
    if expert_nodes.numel() != E or comm.shape != (S, n_nodes) or best_node.numel() != S:
        raise ValueError("shape mismatch")
    _check(lib().grouter_sample_placement(_p(topk_idx), _idx_dtype(topk_idx), S, L, k, E, _p(expert_nodes), n_nodes,
                                          _p(comm), _p(best_node), _stream(stream)), "grouter_sample_placement")


def grouter_sample_stats(topk_idx, E, counts, entropy_bits, loads, maxvio, expert_nodes, n_nodes, comm, best_node,
                         stream=None):
    """grouter_affinity and grouter_sample_placement in one pass over topk_idx [S,L,k]."""
    import torch

    S, L, k = topk_idx.shape
    _dev(topk_idx, "topk_idx")
    _dev(counts, "counts", torch.int32)
    _dev(entropy_bits, "entropy_bits", torch.float64)
    _dev(loads, "loads", torch.int64)
    _dev(maxvio, "maxvio", torch.float64)
    _dev(expert_nodes, "expert_nodes", torch.int64)
    _dev(comm, "comm", torch.int32)
    _dev(best_node, "best_node", torch.int32)
    if (counts.shape != (S, E) or entropy_bits.numel() != S or loads.numel() != E or maxvio.numel() != 1
            or expert_nodes.numel() != E or comm.shape != (S, n_nodes) or best_node.numel() != S):
        raise ValueError("shape mismatch")
    _check(lib().grouter_sample_stats(_p(topk_idx), _idx_dtype(topk_idx), S, L, k, E, _p(counts), _p(entropy_bits),
                                      _p(loads), _p(maxvio), _p(expert_nodes), n_nodes, _p(comm), _p(best_node),
                                      _stream(stream)), "grouter_sample_stats")


def grouter_coactivation(topk_idx, E, P, stream=None):
    """topk_idx [T,k]; P int64 [E,E]."""
    import torch

    T, k = topk_idx.shape
    _dev(topk_idx, "topk_idx")
    _dev(P, "P", torch.int64)
    if P.shape != (E, E):
        raise ValueError("shape mismatch")
    _check(lib().grouter_coactivation(_p(topk_idx), _idx_dtype(topk_idx), T, k, E, _p(P), _stream(stream)),
           "grouter_coactivation")


def grouter_fold_groups(P, E_T, group_of, stream=None):
    """P int64 [E_S,E_S]; group_of int32 [E_S]."""
    import torch

    E_S = P.shape[0]
    _dev(P, "P", torch.int64)
    _dev(group_of, "group_of", torch.int32)
    if P.shape != (E_S, E_S) or group_of.numel() != E_S:
        raise ValueError("shape mismatch")
    _check(lib().grouter_fold_groups(_p(P), E_S, E_T, _p(group_of), _stream(stream)), "grouter_fold_groups")


def grouter_mfma_probe(mode, iters, workgroups, out, stream=None):
    """out float32, at least workgroups*256 elements (a checksum only); returns the FLOP count of the launch."""
    import torch

    _dev(out, "out", torch.float32)
    _check(lib().grouter_mfma_probe(mode, iters, workgroups, _p(out), out.numel(), _stream(stream)), "grouter_mfma_probe")
    return workgroups * 4 * iters * 8 * 32768


def grouter_fold_weights(W_s, group_of, E_T, out, stream=None):
    """W_s float32 [d,E_S]; group_of int32 [E_S]; out float32 [d,E_T]."""
    import torch

    d, E_S = W_s.shape
    _dev(W_s, "W_s", torch.float32)
    _dev(group_of, "group_of", torch.int32)
    _dev(out, "out", torch.float32)
    if group_of.numel() != E_S or out.shape != (d, E_T):
        raise ValueError("shape mismatch")
    _check(lib().grouter_fold_weights(_p(W_s), _p(group_of), d, E_S, E_T, _p(out), _stream(stream)),
           "grouter_fold_weights")


_FLOATS = {}     # torch dtype -> GROUTER_FP32 ..., filled when first asked


def _float_dtype(t, name, allowed=(FP32, BF16, FP16)):
    if not _FLOATS:
        import torch

        _FLOATS.update({torch.float32: FP32, torch.bfloat16: BF16, torch.float16: FP16})
    dt = _FLOATS.get(t.dtype)
    if dt not in allowed:
        raise ValueError(f"{name} has an unsupported dtype ({t.dtype})")
    return dt


def _matrix(t, name, at=None):
    """How far apart the rows of a GPU matrix are; a row is contiguous, its neighbours may be further off than its width."""
    if (t.is_cuda if at is None else t.get_device() == at) and t.dim() == 2:
        E = t.shape[1]
        if t.is_contiguous():
            return E
        rows, columns = t.stride()
        if columns == 1 and rows >= E:
            return rows
        if E == 1 and rows >= 1:
            return rows
    raise ValueError(f"{name} must be a matrix with contiguous rows on {_place(at)}")


def _place(at):
    return "the GPU" if at is None else f"device {at}, as the call's other tensors"


def _beside(t, name, at, dtype=None):
    """A contiguous tensor on device `at` (None: any GPU), which a CPU tensor's -1 never is."""
    if not (t.is_cuda if at is None else t.get_device() == at) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous tensor on {_place(at)}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must have dtype {dtype}")
    return t


def _device_of(t, name):
    at = t.get_device()
    if at < 0:
        raise ValueError(f"{name} must be on the GPU")
    return at


def _mask(token_mask, T, at):
    import torch

    if token_mask is None:
        return None
    _beside(token_mask, "token_mask", at)
    if token_mask.dtype not in (torch.uint8, torch.bool) or token_mask.numel() != T:
        raise ValueError("token_mask must be uint8 or bool [T]")
    return token_mask.data_ptr()


def _sequences(seq_offsets, at):
    import torch

    if seq_offsets is None:
        return None, 1
    _beside(seq_offsets, "seq_offsets", at, torch.int64)
    if seq_offsets.dim() != 1 or seq_offsets.numel() < 2:
        raise ValueError("seq_offsets must be int64 [S+1]")
    return seq_offsets.data_ptr(), seq_offsets.numel() - 1


def _address(t, name, dtype, shape, at):
    """The address of a contiguous tensor of that type and shape on device `at`."""
    if t.get_device() != at or not t.is_contiguous() or t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{name} must be a contiguous tensor of {dtype} {tuple(shape)} on {_place(at)}")
    return t.data_ptr()


def _ids(topk_idx, T, k, at):
    """The address and the type of expert ids [T,k]."""
    kind = _idx_dtype(topk_idx)
    return _address(topk_idx, "topk_idx", topk_idx.dtype, (T, k), at), kind


def grouter_route(scores, k, gating, topk_idx, gate_w, token_mask=None, stream=None):
    """scores [T,E] fp32/bf16/fp16 (rows may be apart); topk_idx [T,k] int32/uint8 and gate_w [T,k] bf16 are written."""
    import torch

    ld = _matrix(scores, "scores")
    T, E = scores.shape
    at = scores.get_device()
    ids, kind = _ids(topk_idx, T, k, at)
    gates = _address(gate_w, "gate_w", torch.bfloat16, (T, k), at)
    _check(lib().grouter_route(scores.data_ptr(), _float_dtype(scores, "scores"), ld, T, E, k, gating, _mask(token_mask, T, at), ids, kind, gates,
                               _stream_for(scores, stream)), "grouter_route")


def grouter_route_bwd(scores, gating, dscores, topk_idx=None, dlog_gate=None, token_mask=None, seq_offsets=None, coef=None, stream=None):
    """dscores [T,E] = gradient out of dlog_gate fp32 [T,k] at topk_idx and/or of the balance loss whose coef fp32 [S,E] is given."""
    import torch

    ld, at = _matrix(scores, "scores"), scores.get_device()
    dld = _matrix(dscores, "dscores", at)
    T, E = shape = scores.shape
    if dscores.shape != shape:
        raise ValueError("shape mismatch")
    off = ids = dlog = weights = None
    S, k, kind = 1, 0, 0
    if coef is not None:
        off, S = _sequences(seq_offsets, at)
        weights = _address(coef, "coef", torch.float32, (S, E), at)
    if dlog_gate is not None:
        if topk_idx is None:
            raise ValueError("dlog_gate comes with the topk_idx that it belongs to")
        k = dlog_gate.shape[-1]
        ids, kind = _ids(topk_idx, T, k, at)
        dlog = _address(dlog_gate, "dlog_gate", torch.float32, (T, k), at)
    _check(lib().grouter_route_bwd(scores.data_ptr(), _float_dtype(scores, "scores"), ld, T, E, gating, _mask(token_mask, T, at), ids, kind, k, dlog, off, S,
                                   weights, dscores.data_ptr(), _float_dtype(dscores, "dscores"), dld, _stream_for(scores, stream)), "grouter_route_bwd")


def grouter_balance_bytes(T, E, S) -> int:
    return int(lib().grouter_balance_bytes(T, E, S))


def grouter_balance(scores, gating, topk_idx, alpha, counts, prob, coef, loss, ws, token_mask=None, seq_offsets=None, stream=None):
    """scores [T,E], topk_idx [T,k], seq_offsets int64 [S+1] or None (S = 1); written: counts int32, prob and coef fp32 [S,E], loss fp32 [1]."""
    import torch

    ld = _matrix(scores, "scores")
    T, E = scores.shape
    at = scores.get_device()
    off, S = _sequences(seq_offsets, at)
    k = topk_idx.shape[-1]
    ids, kind = _ids(topk_idx, T, k, at)
    fp32, per_sequence = torch.float32, (S, E)
    if not loss.numel() == 1:
        raise ValueError("loss must have one element")
    _check(lib().grouter_balance(scores.data_ptr(), _float_dtype(scores, "scores"), ld, T, E, k, gating, _mask(token_mask, T, at), ids, kind, off, S, alpha,
                                 _address(counts, "counts", torch.int32, per_sequence, at), _address(prob, "prob", fp32, per_sequence, at),
                                 _address(coef, "coef", fp32, per_sequence, at), _beside(loss, "loss", at, fp32).data_ptr(),
                                 _beside(ws, "ws", at).data_ptr(),
                                 ws.numel() * ws.element_size(), _stream_for(scores, stream)), "grouter_balance")


def grouter_gate_bwd(plan_ws, T, k, E, dY, inp, dlog_gate, stream=None):
    """dlog_gate fp32 [T,k] from dY bf16 [T,d] and rows inp bf16 [T*k,d] in expert-sorted order."""
    import torch

    bf, d = torch.bfloat16, dY.shape[-1]
    at = _device_of(dY, "dY")
    if _beside(plan_ws, "plan_ws", at).numel() < grouter_plan_bytes(T, k, E):
        raise ValueError("plan_ws is smaller than a plan of this size")
    _check(lib().grouter_gate_bwd(plan_ws.data_ptr(), T, k, E, d, _address(dY, "dY", bf, (T, d), at), _address(inp, "in", bf, (T * k, d), at),
                                  _address(dlog_gate, "dlog_gate", torch.float32, (T, k), at), _stream_for(dY, stream)), "grouter_gate_bwd")


def grouter_moe_gate_bwd(plan_ws, E, f, dY, ctx_ws, dlog_gate, stream=None):
    """The same on the rows that grouter_moe_fwd kept in ctx_ws."""
    import torch

    T, k = dlog_gate.shape
    d = dY.shape[-1]
    at = _device_of(dY, "dY")
    if _beside(plan_ws, "plan_ws", at).numel() < grouter_plan_bytes(T, k, E):
        raise ValueError("plan_ws is smaller than a plan of this size")
    _check(lib().grouter_moe_gate_bwd(plan_ws.data_ptr(), T, k, E, d, f, _address(dY, "dY", torch.bfloat16, (T, d), at),
                                      _beside(ctx_ws, "ctx_ws", at).data_ptr(), ctx_ws.numel(),
                                      _address(dlog_gate, "dlog_gate", torch.float32, (T, k), at), _stream_for(dY, stream)),
           "grouter_moe_gate_bwd")


def grouter_adamw_hyper(lr, beta1, beta2, eps, weight_decay, step, grad_scale=1.0, seed=0) -> AdamWHyper:
    h = AdamWHyper()
    _check(lib().grouter_adamw_hyper_set(lr, beta1, beta2, eps, weight_decay, step, grad_scale, seed & 0xffffffff, ctypes.byref(h)),
           "grouter_adamw_hyper_set")
    return h


class AdamWTensors:
    """The tensors of an optimizer step, looked over once: lists of parameters, gradients and moments of one type each.

    param fp32, or bf16, alone or with fp32 `master` copies; grad fp32 or bf16; m and v fp32, or uint8 codes with uint8 exponents
    m_exp and v_exp of ceil(n/32) elements.  The object holds the tensors; a gradient that moves needs a new one, which costs the host about
    5 us per tensor (12 tensors 60 us, 75 330, 300 1300), more than most steps: keep gradients in place, as this library's own calls do
    and as autograd does after zero_grad(set_to_none=False).
    """

    def __init__(self, param, grad, m, v, master=None, m_exp=None, v_exp=None):
        import torch

        param, grad, m, v = list(param), list(grad), list(m), list(v)
        none = [None] * len(param)
        master, m_exp, v_exp = (none if x is None else list(x) for x in (master, m_exp, v_exp))
        self._held = (param, grad, m, v, master, m_exp, v_exp)
        if any(len(x) != len(param) for x in self._held):
            raise ValueError("lists of different lengths")
        self.count, self.device = len(param), param[0].device if param else None
        first = param[0] if param else None
        if first is not None and first.dtype not in (torch.float32, torch.bfloat16):
            raise ValueError("param must be fp32 or bf16")
        if master is not none and first is not None and first.dtype != torch.bfloat16:
            raise ValueError("master copies belong to bf16 parameters")
        self.kind = ADAMW_FP32 if first is None or first.dtype == torch.float32 else ADAMW_BF16 if master is none else ADAMW_MASTER
        self.grad_dtype = _float_dtype(grad[0], "grad", (FP32, BF16)) if grad else FP32
        self.bits = 8 if m and m[0].dtype == torch.uint8 else 32
        if (self.bits == 8) != (m_exp is not none) or (self.bits == 8) != (v_exp is not none):
            if first is not None:
                raise ValueError("8-bit moments come with exponents, 32-bit ones without")
        state = torch.uint8 if self.bits == 8 else torch.float32
        self._array = (_AdamWTensor * max(1, self.count))()
        spans = []
        for i, (p, g, a, b, w, ea, eb) in enumerate(zip(*self._held)):
            n = p.numel()
            for t, name, dtype, size in ((p, "param", first.dtype, n), (g, "grad", grad[0].dtype, n), (a, "m", state, n), (b, "v", state, n),
                                         (w, "master", torch.float32, n), (ea, "m_exp", torch.uint8, -(-n // 32)),
                                         (eb, "v_exp", torch.uint8, -(-n // 32))):
                if t is None:
                    continue
                if _dev(t, name, dtype).numel() != size or t.device != self.device:
                    raise ValueError(f"{name} {i}: wrong size or device")
                if size and name not in ("m_exp", "v_exp") and t.data_ptr() % 16:
                    raise ValueError(f"{name} {i} must be aligned to 16 bytes")
                if size:
                    spans.append((t.data_ptr(), t.data_ptr() + size * t.element_size()))
            self._array[i] = _AdamWTensor(*(_p(t) for t in (p, w, g, a, b, ea, eb)), n)
        spans.sort()
        if any(y[0] < x[1] for x, y in zip(spans, spans[1:])):
            raise ValueError("tensors overlap")


def grouter_adamw(tensors, hyper, grad_scale=None, stream=None):
    """One step over an AdamWTensors; hyper an AdamWHyper, or a GPU uint8 tensor holding one; grad_scale fp32 [1] on the GPU or None."""
    import torch

    host = isinstance(hyper, AdamWHyper)
    at = tensors._held[0][0].get_device() if tensors.count else None
    if not host and _beside(hyper, "hyper", at, torch.uint8).numel() < ctypes.sizeof(AdamWHyper):
        raise ValueError("hyper must hold 48 bytes")
    if grad_scale is not None and _beside(grad_scale, "grad_scale", at, torch.float32).numel() != 1:
        raise ValueError("grad_scale must have one element")
    if not tensors.count:
        return
    _check(lib().grouter_adamw(tensors._array, tensors.count, tensors.kind, tensors.grad_dtype, tensors.bits,
                               ctypes.byref(hyper) if host else None, None if host else _p(hyper), _p(grad_scale), _stream_for(tensors._held[0][0], stream)),
           "grouter_adamw")


def grouter_timing_enable(on: bool):
    _check(lib().grouter_timing_enable(1 if on else 0), "grouter_timing_enable")


def grouter_timing_read():
    """{phase: (milliseconds, launches)} accumulated since the previous read; waits for the recorded events."""
    n = len(PHASES)
    ms = (ctypes.c_double * n)()
    cnt = (ctypes.c_int64 * n)()
    _check(lib().grouter_timing_read(ms, cnt), "grouter_timing_read")
    return {PHASES[i]: (float(ms[i]), int(cnt[i])) for i in range(n)}
