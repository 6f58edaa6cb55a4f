"""ctypes binding of libskrull_attn.so: same names as the C ABI, argument
marshalling only.  Tensors are torch CUDA(HIP) tensors used purely as device
memory; every step of the path runs in the library's kernels.  There is no CPU
fallback: a missing library raises."""
from __future__ import annotations

import ctypes
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libskrull_attn.so")

SKRULL_OK, SKRULL_EINVAL, SKRULL_ENOMEM, SKRULL_EHIP, SKRULL_EUNSUPPORTED, SKRULL_ESCHED = 0, -1, -2, -3, -4, -5
(ARRAY_CU_Q, ARRAY_CU_K, ARRAY_Q_BEGIN, ARRAY_Q_LEN, ARRAY_KV_LEN, ARRAY_FWD_ITEMS, ARRAY_DKV_ITEMS,
 ARRAY_SHARES_KV) = range(8)
CUT_CONTIGUOUS, CUT_TWO_CHUNKS = 0, 1
ROTARY_HALF, ROTARY_INTERLEAVED = 0, 1
ROTARY_PLAIN, ROTARY_LINEAR, ROTARY_NTK, ROTARY_PARTS = range(4)
ROWS_Q, ROWS_K = 0, 1
NORM_RMS, NORM_LAYER = 0, 1
TYPE_BF16, TYPE_FP32 = 0, 1

EXPORTED_SYMBOLS = ("skrull_attn_plan", "skrull_attn_plan_info", "skrull_attn_plan_export",
                    "skrull_attn_fwd", "skrull_attn_bwd", "skrull_attn_bwd_static", "skrull_attn_plan_destroy",
                    "skrull_attn_strerror", "skrull_attn_profile", "skrull_attn_profile_read",
                    "skrull_attn_mfma_ceiling", "skrull_attn_trace", "skrull_attn_trace_layout",
                    "skrull_dacp_schedule", "skrull_dacp_rank_batch",
                    "skrull_gds_binpack", "skrull_gds_schedule", "skrull_gds_micro_batch")
# the operators around attention (skrull_rotary.h, skrull_norm.h, skrull_loss.h)
OPERATOR_SYMBOLS = ("skrull_rotary_check", "skrull_rotary", "skrull_norm_fwd", "skrull_norm_workspace", "skrull_norm_bwd",
                    "skrull_loss_workspace", "skrull_loss_fwd", "skrull_loss_bwd")


class Problem(ctypes.Structure):
    _fields_ = [("num_seqs", ctypes.c_int32),
                ("seq_len", ctypes.POINTER(ctypes.c_int32)),
                ("shard_degree", ctypes.POINTER(ctypes.c_int32)),
                ("shard_index", ctypes.POINTER(ctypes.c_int32)),
                ("num_q_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float),
                ("block_m", ctypes.c_int32),
                ("block_n", ctypes.c_int32),
                ("shard_cut", ctypes.POINTER(ctypes.c_int32)),
                ("head_split", ctypes.c_int32), ("wg_query_rows", ctypes.c_int32)]


class PlanInfo(ctypes.Structure):
    _fields_ = [("num_seqs", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("block_m", ctypes.c_int32), ("block_n", ctypes.c_int32),
                ("total_q", ctypes.c_int32), ("total_k", ctypes.c_int32),
                ("n_fwd_items", ctypes.c_int32), ("n_dkv_items", ctypes.c_int32),
                ("attended_pairs", ctypes.c_int64), ("useful_flops_fwd", ctypes.c_int64),
                ("useful_flops_bwd", ctypes.c_int64), ("bwd_workspace_bytes", ctypes.c_int64),
                ("num_segments", ctypes.c_int32), ("head_split", ctypes.c_int32),
                ("wg_query_rows", ctypes.c_int32), ("shapes", ctypes.c_int32)]

    @property
    def fwd_waves(self):
        """Wavefronts of a forward workgroup that runs."""
        return self.shapes & 255

    @property
    def dq_waves(self):
        """Wavefronts of a dQ workgroup where dQ is a launch of its own."""
        return self.shapes >> 8 & 255

    @property
    def dq_pipelined(self):
        return bool(self.shapes >> 16 & 1)


class FlopsModel(ctypes.Structure):
    _fields_ = [("hidden", ctypes.c_int64), ("hidden_kv", ctypes.c_int64), ("batch", ctypes.c_int64)]


class Rotary(ctypes.Structure):
    _fields_ = [("head_dim", ctypes.c_int32), ("rotary_dim", ctypes.c_int32), ("layout", ctypes.c_int32),
                ("scaling", ctypes.c_int32), ("base", ctypes.c_double), ("factor", ctypes.c_double),
                ("original_length", ctypes.c_double), ("low_turns", ctypes.c_double), ("high_turns", ctypes.c_double),
                ("amplitude", ctypes.c_double)]


class RotaryTensor(ctypes.Structure):
    _fields_ = [("in_", ctypes.c_void_p), ("out", ctypes.c_void_p), ("in_stride", ctypes.c_int64),
                ("out_stride", ctypes.c_int64), ("heads", ctypes.c_int32), ("rows", ctypes.c_int32)]


class Norm(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int32), ("kind", ctypes.c_int32), ("type", ctypes.c_int32),
                ("weight_type", ctypes.c_int32), ("eps", ctypes.c_float), ("x_stride", ctypes.c_int64),
                ("y_stride", ctypes.c_int64), ("dy_stride", ctypes.c_int64), ("dx_stride", ctypes.c_int64)]


class Loss(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("hidden", ctypes.c_int32), ("vocab", ctypes.c_int32),
                ("x_stride", ctypes.c_int64)]


class SkrullError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"skrull_attn error {code}: {msg}")
        self.code = code


_lib = None


def lib():
    """Load the in-tree HIP library; raise loudly if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run __graft_entry__.build() "
                               "(python -m paper_2505_19609_amd.build); there is no fallback path")
        # PyTorch ships its own HIP runtime; loading it first lets this library's
        # libamdhip64 dependency resolve to that same copy, so device pointers and
        # streams made by torch are valid in our calls (two runtimes in one process
        # do not see each other's devices).
        import torch  # noqa: F401
        L = ctypes.CDLL(LIB_PATH)
        vp = ctypes.c_void_p
        L.skrull_attn_plan.argtypes = [ctypes.POINTER(Problem), vp, ctypes.POINTER(vp)]
        L.skrull_attn_plan.restype = ctypes.c_int
        L.skrull_attn_plan_info.argtypes = [vp, ctypes.POINTER(PlanInfo)]
        L.skrull_attn_plan_info.restype = ctypes.c_int
        L.skrull_attn_plan_export.argtypes = [vp, ctypes.c_int, vp, ctypes.c_size_t]
        L.skrull_attn_plan_export.restype = ctypes.c_int
        L.skrull_attn_fwd.argtypes = [vp] * 7
        L.skrull_attn_fwd.restype = ctypes.c_int
        L.skrull_attn_bwd.argtypes = [vp] * 11 + [ctypes.c_size_t, vp]
        L.skrull_attn_bwd.restype = ctypes.c_int
        L.skrull_attn_bwd_static.argtypes = [vp] * 11
        L.skrull_attn_bwd_static.restype = ctypes.c_int
        L.skrull_attn_plan_destroy.argtypes = [vp]
        L.skrull_attn_plan_destroy.restype = None
        L.skrull_attn_strerror.argtypes = [ctypes.c_int]
        L.skrull_attn_strerror.restype = ctypes.c_char_p
        L.skrull_attn_profile.argtypes = [ctypes.c_int]
        L.skrull_attn_profile.restype = ctypes.c_int
        L.skrull_attn_profile_read.argtypes = [ctypes.POINTER(ctypes.c_float)]
        L.skrull_attn_profile_read.restype = ctypes.c_int
        L.skrull_attn_mfma_ceiling.argtypes = [vp, ctypes.POINTER(ctypes.c_float)]
        L.skrull_attn_mfma_ceiling.restype = ctypes.c_int
        i32p = ctypes.POINTER(ctypes.c_int32)
        L.skrull_attn_trace.argtypes = [vp, ctypes.c_size_t]
        L.skrull_attn_trace.restype = ctypes.c_int
        L.skrull_attn_trace_layout.argtypes = [vp, i32p, i32p]
        L.skrull_attn_trace_layout.restype = ctypes.c_int
        L.skrull_dacp_schedule.argtypes = [ctypes.c_int32, i32p, ctypes.c_int64, ctypes.c_int32,
                                           ctypes.POINTER(FlopsModel), i32p]
        L.skrull_dacp_schedule.restype = ctypes.c_int
        L.skrull_dacp_rank_batch.argtypes = [ctypes.c_int32, i32p, i32p, ctypes.c_int32, ctypes.c_int32,
                                             i32p, i32p, i32p, i32p, i32p]
        L.skrull_dacp_rank_batch.restype = ctypes.c_int
        L.skrull_gds_binpack.argtypes = [ctypes.c_int32, i32p, ctypes.c_int32, ctypes.POINTER(FlopsModel), i32p]
        L.skrull_gds_binpack.restype = ctypes.c_int
        L.skrull_gds_schedule.argtypes = [ctypes.c_int32, i32p, ctypes.c_int64, ctypes.c_int32, ctypes.c_int32,
                                          ctypes.c_int32, ctypes.POINTER(FlopsModel), i32p, i32p, i32p, i32p]
        L.skrull_gds_schedule.restype = ctypes.c_int
        L.skrull_gds_micro_batch.argtypes = [ctypes.c_int32, i32p, i32p, ctypes.c_int32, i32p, i32p]
        L.skrull_gds_micro_batch.restype = ctypes.c_int
        L.skrull_rotary_check.argtypes = [ctypes.POINTER(Rotary)]
        L.skrull_rotary.argtypes = [vp, ctypes.POINTER(Rotary), ctypes.POINTER(RotaryTensor), ctypes.POINTER(RotaryTensor),
                                    ctypes.c_int, vp]
        norm, loss = ctypes.POINTER(Norm), ctypes.POINTER(Loss)
        L.skrull_norm_fwd.argtypes = [norm] + [vp] * 7
        L.skrull_norm_workspace.argtypes = [norm]
        L.skrull_norm_bwd.argtypes = [norm] + [vp] * 9 + [ctypes.c_size_t, vp]
        L.skrull_loss_workspace.argtypes = [loss, ctypes.c_int]
        L.skrull_loss_fwd.argtypes = [loss] + [vp] * 6 + [ctypes.c_size_t, vp]
        L.skrull_loss_bwd.argtypes = [loss] + [vp] * 8 + [ctypes.c_size_t, vp]
        for name in OPERATOR_SYMBOLS:
            getattr(L, name).restype = ctypes.c_int64 if name.endswith("workspace") else ctypes.c_int
        _lib = L
    return _lib


def skrull_attn_strerror(code: int) -> str:
    return lib().skrull_attn_strerror(code).decode()


def _check(rc: int):
    if rc != SKRULL_OK:
        raise SkrullError(rc, skrull_attn_strerror(rc))


def _stream_ptr(stream):
    """The hipStream_t of `stream`, or of torch's current one, as an integer.  (The current stream is asked
    for as a raw pointer: torch.cuda.current_stream() builds a Stream object, 3 us of the 7 that a
    forward call cost the host.  That function is private to torch, so it may be missing.)"""
    if stream is None:
        import torch
        if torch.cuda.is_initialized():
            try:
                raw = torch._C._cuda_getCurrentRawStream
            except AttributeError:
                pass
            else:
                return raw(torch.cuda.current_device())
        stream = torch.cuda.current_stream()
    return int(getattr(stream, "cuda_stream", stream))


class Plan:
    """Owner of a ``skrull_attn_plan_t*``."""

    def __init__(self, handle, info: PlanInfo):
        self.handle = handle
        self.info = info

    def __getattr__(self, name):
        return getattr(self.info, name)

    def destroy(self):
        if self.handle:
            lib().skrull_attn_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def skrull_attn_plan(seq_len, shard_degree, shard_index, num_q_heads, num_kv_heads, head_dim,
                     softmax_scale, block_m=0, block_n=0, stream=None, raw_stream=None,
                     shard_cut=None, head_split=0, wg_query_rows=0) -> Plan:
    S = np.ascontiguousarray(seq_len, dtype=np.int32)
    N = np.ascontiguousarray(shard_degree, dtype=np.int32)
    R = np.ascontiguousarray(shard_index, dtype=np.int32)
    Z = None if shard_cut is None else np.ascontiguousarray(shard_cut, dtype=np.int32)
    if not (S.shape == N.shape == R.shape and S.ndim == 1 and (Z is None or Z.shape == S.shape)):
        raise SkrullError(SKRULL_EINVAL, "seq_len / shard_degree / shard_index / shard_cut must be 1-D and equally long")
    i32p = ctypes.POINTER(ctypes.c_int32)
    prob = Problem(int(S.shape[0]), S.ctypes.data_as(i32p), N.ctypes.data_as(i32p),
                   R.ctypes.data_as(i32p), num_q_heads, num_kv_heads, head_dim,
                   float(softmax_scale), block_m, block_n,
                   None if Z is None else Z.ctypes.data_as(i32p), int(head_split), int(wg_query_rows))
    handle = ctypes.c_void_p()
    st = raw_stream if raw_stream is not None else _stream_ptr(stream)
    _check(lib().skrull_attn_plan(ctypes.byref(prob), st, ctypes.byref(handle)))
    info = PlanInfo()
    _check(lib().skrull_attn_plan_info(handle, ctypes.byref(info)))
    return Plan(handle, info)


def skrull_attn_plan_info(plan: Plan) -> PlanInfo:
    info = PlanInfo()
    _check(lib().skrull_attn_plan_info(plan.handle, ctypes.byref(info)))
    return info


def skrull_attn_plan_export(plan: Plan, which: int) -> np.ndarray:
    K = plan.info.num_segments
    shape = {ARRAY_CU_Q: (K + 1,), ARRAY_CU_K: (K + 1,), ARRAY_Q_BEGIN: (K,), ARRAY_Q_LEN: (K,),
             ARRAY_KV_LEN: (K,), ARRAY_SHARES_KV: (K,), ARRAY_FWD_ITEMS: (plan.info.n_fwd_items, 4),
             ARRAY_DKV_ITEMS: (plan.info.n_dkv_items, 4)}[which]
    out = np.zeros(shape, np.int32)
    _check(lib().skrull_attn_plan_export(plan.handle, which, out.ctypes.data_as(ctypes.c_void_p),
                                         out.nbytes))
    return out


def _ptr(t):
    return t.data_ptr()   # (the argument types say that it is a pointer)


def skrull_attn_fwd(plan: Plan, q, k, v, o, lse, stream=None):
    _check(lib().skrull_attn_fwd(plan.handle, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse),
                                 _stream_ptr(stream)))


def skrull_attn_bwd(plan: Plan, q, k, v, o, lse, d_o, dq, dk, dv, workspace, stream=None):
    _check(lib().skrull_attn_bwd(plan.handle, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse),
                                 _ptr(d_o), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), _stream_ptr(stream)))


STATIC_SCRATCH_BYTES = 32 * 1024 * 1024


def skrull_attn_bwd_static(plan: Plan, q, k, v, o, lse, d_o, dq, dk, dv, stream=None):
    """skrull_attn_bwd on the library's static workspace (no allocation anywhere)."""
    _check(lib().skrull_attn_bwd_static(plan.handle, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse),
                                        _ptr(d_o), _ptr(dq), _ptr(dk), _ptr(dv), _stream_ptr(stream)))


def skrull_attn_profile(enable: bool):
    _check(lib().skrull_attn_profile(int(bool(enable))))


def skrull_attn_profile_read():
    """Kernel durations (ms) of the last forward / backward: [fwd, 0, dkv, dq] (the second
    slot was a separate rowsum(dO*O) kernel; the dQ kernel forms it now)."""
    ms = (ctypes.c_float * 4)()
    _check(lib().skrull_attn_profile_read(ms))
    return [float(x) for x in ms]


def skrull_attn_trace(records=None):
    """Switch the per-workgroup trace on (records: a zeroed torch uint8 CUDA tensor) or off (None)."""
    if records is None:
        _check(lib().skrull_attn_trace(None, 0))
    else:
        _check(lib().skrull_attn_trace(_ptr(records), records.numel() * records.element_size()))


def skrull_attn_trace_layout(plan: Plan):
    """(first_record[3], num_records[3]) of the forward, dQ and dK/dV kernels of `plan`."""
    first, num = (ctypes.c_int32 * 3)(), (ctypes.c_int32 * 3)()
    _check(lib().skrull_attn_trace_layout(plan.handle, first, num))
    return [int(x) for x in first], [int(x) for x in num]


def skrull_attn_mfma_ceiling(stream=None) -> float:
    """TFLOP/s this GPU sustains on bf16 MFMAs alone (measurement aid)."""
    out = ctypes.c_float(0.0)
    _check(lib().skrull_attn_mfma_ceiling(_stream_ptr(stream), ctypes.byref(out)))
    return float(out.value)


def skrull_dacp_schedule(seq_len, bucket_size, cp_degree, hidden, hidden_kv, batch=1) -> np.ndarray:
    """ret[K]: the rank that keeps sequence k whole, or -1 if it is distributed.
    Raises SkrullError(SKRULL_ESCHED) when the micro-batch does not fit."""
    S = np.ascontiguousarray(seq_len, dtype=np.int32)
    if S.ndim != 1:
        raise SkrullError(SKRULL_EINVAL, "seq_len must be 1-D")
    ret = np.zeros(S.shape[0], np.int32)
    i32p = ctypes.POINTER(ctypes.c_int32)
    model = FlopsModel(int(hidden), int(hidden_kv), int(batch))
    _check(lib().skrull_dacp_schedule(int(S.shape[0]), S.ctypes.data_as(i32p), int(bucket_size),
                                      int(cp_degree), ctypes.byref(model), ret.ctypes.data_as(i32p)))
    return ret


def skrull_dacp_rank_batch(seq_len, ret, cp_degree, rank):
    """(seq_len, shard_degree, shard_index, source) of rank `rank`'s micro-batch."""
    S = np.ascontiguousarray(seq_len, dtype=np.int32)
    R = np.ascontiguousarray(ret, dtype=np.int32)
    if S.ndim != 1 or S.shape != R.shape:
        raise SkrullError(SKRULL_EINVAL, "seq_len / ret must be 1-D and equally long")
    K = int(S.shape[0])
    out = [np.zeros(max(K, 1), np.int32) for _ in range(4)]
    n = ctypes.c_int32(0)
    i32p = ctypes.POINTER(ctypes.c_int32)
    _check(lib().skrull_dacp_rank_batch(K, S.ctypes.data_as(i32p), R.ctypes.data_as(i32p),
                                        int(cp_degree), int(rank), *[o.ctypes.data_as(i32p) for o in out],
                                        ctypes.byref(n)))
    return tuple(o[:n.value].copy() for o in out)


def _lengths(seq_len) -> np.ndarray:
    S = np.ascontiguousarray(seq_len, dtype=np.int32)
    if S.ndim != 1:
        raise SkrullError(SKRULL_EINVAL, "seq_len must be 1-D")
    return S


def skrull_gds_binpack(seq_len, dp_world_size, hidden, hidden_kv, batch=1) -> np.ndarray:
    """dp_bin[K]: the DP rank of every sequence of the global batch."""
    S = _lengths(seq_len)
    out = np.zeros(S.shape[0], np.int32)
    i32p = ctypes.POINTER(ctypes.c_int32)
    model = FlopsModel(int(hidden), int(hidden_kv), int(batch))
    _check(lib().skrull_gds_binpack(int(S.shape[0]), S.ctypes.data_as(i32p), int(dp_world_size),
                                    ctypes.byref(model), out.ctypes.data_as(i32p)))
    return out


def skrull_gds_schedule(seq_len, bucket_size, cp_degree, dp_world_size, dp_rank, hidden, hidden_kv, batch=1):
    """(dp_bin[K], micro_batch[K], ret[K], num_micro_batches) for DP rank `dp_rank`."""
    S = _lengths(seq_len)
    K = int(S.shape[0])
    bins, mb, ret = (np.zeros(K, np.int32) for _ in range(3))
    n = ctypes.c_int32(0)
    i32p = ctypes.POINTER(ctypes.c_int32)
    model = FlopsModel(int(hidden), int(hidden_kv), int(batch))
    _check(lib().skrull_gds_schedule(K, S.ctypes.data_as(i32p), int(bucket_size), int(cp_degree),
                                     int(dp_world_size), int(dp_rank), ctypes.byref(model),
                                     bins.ctypes.data_as(i32p), mb.ctypes.data_as(i32p),
                                     ret.ctypes.data_as(i32p), ctypes.byref(n)))
    return bins, mb, ret, int(n.value)


def skrull_gds_micro_batch(seq_len, micro_batch, index) -> np.ndarray:
    """Positions (caller's list) of the members of micro-batch `index`, ascending length."""
    S = _lengths(seq_len)
    M = np.ascontiguousarray(micro_batch, dtype=np.int32)
    if M.shape != S.shape:
        raise SkrullError(SKRULL_EINVAL, "seq_len / micro_batch must be equally long")
    out = np.zeros(max(int(S.shape[0]), 1), np.int32)
    n = ctypes.c_int32(0)
    i32p = ctypes.POINTER(ctypes.c_int32)
    _check(lib().skrull_gds_micro_batch(int(S.shape[0]), S.ctypes.data_as(i32p), M.ctypes.data_as(i32p),
                                        int(index), out.ctypes.data_as(i32p), ctypes.byref(n)))
    return out[:n.value].copy()


# ---- rotary positions, norm, loss ---------------------------------------------------------------------------------
# These take strided tensors, so shapes, types and devices are checked here; a tensor on another device than the
# current one is refused, as the library refuses a plan of another device.

def _refuse(why):
    raise SkrullError(SKRULL_EINVAL, f"invalid argument ({why})")


def _int32(value, name):
    """`value` for a field of 32 bits, of which ctypes would keep the low ones."""
    value = int(value)
    if not -(1 << 31) <= value < 1 << 31:
        _refuse(f"{name} {value}")
    return value


def _on_current_device(*tensors):
    import torch
    device = torch.cuda.current_device() if torch.cuda.is_initialized() else -2   # (-1: of a tensor that is on no GPU)
    for t in tensors:
        if t is not None and t.get_device() != device:
            _refuse(f"a tensor is on {t.device}, not on the current GPU")


def skrull_rotary_init(head_dim, rotary_dim=None, layout=ROTARY_HALF, base=10000.0, scaling=ROTARY_PLAIN, factor=1.0,
                       original_length=0.0, low_turns=0.0, high_turns=0.0, amplitude=1.0) -> Rotary:
    """What skrull_rotary needs to know of the model, checked."""
    r = Rotary(_int32(head_dim, "head_dim"), _int32(head_dim if rotary_dim is None else rotary_dim, "rotary_dim"), _int32(layout, "layout"),
               _int32(scaling, "scaling"), float(base), float(factor), float(original_length), float(low_turns), float(high_turns), float(amplitude))
    _check(lib().skrull_rotary_check(ctypes.byref(r)))
    return r


def _rotary_tensor(info, x, out, rows):
    import torch
    if out is None:
        _refuse("a tensor to turn has no output")
    want, d = info.total_q if rows == ROWS_Q else info.total_k, info.head_dim
    shape, strides = x.shape, []
    for t in (x, out):
        if t.dtype is not torch.bfloat16 or len(shape) != 3 or shape[0] != want or shape[2] != d or t.shape != shape:
            _refuse(f"a tensor of bf16 [{want}, heads, {d}] is needed, got {t.dtype} {list(t.shape)}")
        row, head, one = t.stride()
        if one != 1 or (head != d and shape[1] > 1):
            _refuse("the heads of a row must be contiguous")
        strides.append(row if want > 1 else shape[1] * d)   # (a single row's stride says nothing)
    return RotaryTensor(x.data_ptr(), out.data_ptr(), strides[0], strides[1], _int32(shape[1], "heads"), _int32(rows, "rows"))


_turn = None


def _native_turn():
    """The native marshalling of skrull_rotary, False where it cannot be loaded."""
    global _turn
    if _turn is None:
        from . import autograd
        module = autograd._module()
        _turn = module.turn if module is not None else False
    return _turn


def skrull_rotary(plan: Plan, rotary: Rotary, q, k, q_out, k_out, inverse=False, k_rows=ROWS_K, stream=None):
    """q_out, k_out = q, k turned by the positions of the plan's rows (`inverse`: turned back).  q or k may be None.  k_rows: whether
    k holds the gathered prefixes (ROWS_K) or this rank's own tokens (ROWS_Q)."""
    # (932 rows, 4/4 heads of 64, which the GPU turns in 2.9 us: 3.6 us a call in native code, 9.1 by what follows)
    turn = _native_turn()
    if turn and type(rotary) is Rotary and turn(plan, ctypes.addressof(rotary), q, k, q_out, k_out, inverse, k_rows,
                                                None if stream is None else _stream_ptr(stream)):
        return
    _on_current_device(q, k, q_out, k_out)
    info = plan.info
    t = [_rotary_tensor(info, x, out, rows) for x, out, rows in ((q, q_out, ROWS_Q), (k, k_out, k_rows)) if x is not None]
    if not t:
        _refuse("neither q nor k")
    _check(lib().skrull_rotary(plan.handle, ctypes.byref(rotary), ctypes.byref(t[0]),
                               ctypes.byref(t[1]) if len(t) > 1 else None, int(bool(inverse)), _stream_ptr(stream)))


def _type_of(t):
    import torch
    if t.dtype == torch.bfloat16:
        return TYPE_BF16
    if t.dtype == torch.float32:
        return TYPE_FP32
    _refuse(f"bf16 and fp32 are taken, got {t.dtype}")


def _norm_of(x, weight, eps, kind, **rows) -> Norm:
    p = Norm(x.shape[0] if x.dim() == 2 else -1, _int32(x.shape[-1], "cols"), _int32(kind, "kind"), _type_of(x), _type_of(weight), float(eps))
    for name, t in dict(rows, x=x).items():
        if t.dim() != 2 or t.shape != x.shape or t.dtype != x.dtype or (t.shape[1] > 1 and t.stride(1) != 1):
            _refuse(f"{name} must be {x.dtype} [rows, cols] with contiguous rows, as x is")
        setattr(p, name + "_stride", t.stride(0) if t.shape[0] > 1 else t.shape[1])
    return p


def _vector(t, n, dtype, name):
    if t is not None and (t.shape != (n,) or t.dtype != dtype or not t.is_contiguous()):
        _refuse(f"{name} must be contiguous {dtype} [{n}]")
    return None if t is None else _ptr(t)


def _scratch(t):
    """The address and size of a workspace."""
    if t is None:
        return None, 0
    if not t.is_contiguous():
        _refuse("workspace must be contiguous")
    return _ptr(t), t.numel() * t.element_size()


def skrull_norm_fwd(x, weight, bias, y, mean, rstd, eps=1e-5, kind=NORM_LAYER, stream=None):
    """y = the norm of the rows of x; mean and rstd (fp32 [rows], may be None) for the backward."""
    import torch
    _on_current_device(x, weight, bias, y, mean, rstd)
    p = _norm_of(x, weight, eps, kind, y=y)
    cols, wt, rows = p.cols, weight.dtype, p.rows
    _check(lib().skrull_norm_fwd(ctypes.byref(p), _ptr(x), _vector(weight, cols, wt, "weight"), _vector(bias, cols, wt, "bias"), _ptr(y),
                                 _vector(mean, rows, torch.float32, "mean"), _vector(rstd, rows, torch.float32, "rstd"), _stream_ptr(stream)))


def skrull_norm_workspace(x, weight, kind=NORM_LAYER) -> int:
    """Bytes that skrull_norm_bwd asks for."""
    return int(lib().skrull_norm_workspace(ctypes.byref(_norm_of(x, weight, 0.0, kind))))


def skrull_norm_bwd(x, weight, mean, rstd, dy, dx, dweight, dbias, workspace, kind=NORM_LAYER, stream=None):
    """dx, and dweight and dbias where they are wanted (else None)."""
    import torch
    _on_current_device(x, weight, mean, rstd, dy, dx, dweight, dbias, workspace)
    p = _norm_of(x, weight, 0.0, kind, dy=dy, dx=dx)
    cols, wt, rows = p.cols, weight.dtype, p.rows
    _check(lib().skrull_norm_bwd(ctypes.byref(p), _ptr(x), _vector(weight, cols, wt, "weight"), _vector(mean, rows, torch.float32, "mean"),
                                 _vector(rstd, rows, torch.float32, "rstd"), _ptr(dy), _ptr(dx), _vector(dweight, cols, wt, "dweight"),
                                 _vector(dbias, cols, wt, "dbias"), *_scratch(workspace), _stream_ptr(stream)))


def _loss_of(x, weight, target) -> Loss:
    import torch
    if x.dim() != 2 or x.dtype != torch.bfloat16 or x.stride(1) != 1:
        _refuse(f"x must be bf16 [rows, hidden] with contiguous rows, got {x.dtype} {list(x.shape)}")
    if weight.dtype != torch.bfloat16 or weight.dim() != 2 or weight.shape[1] != x.shape[1] or not weight.is_contiguous():
        _refuse(f"weight must be contiguous bf16 [vocab, {x.shape[1]}], got {weight.dtype} {list(weight.shape)}")
    if target is not None and (target.dtype != torch.int64 or target.shape != (x.shape[0],) or not target.is_contiguous()):
        _refuse(f"target must be contiguous int64 [{x.shape[0]}], got {target.dtype} {list(target.shape)}")
    return Loss(x.shape[0], _int32(x.shape[1], "hidden"), _int32(weight.shape[0], "vocab"), x.stride(0) if x.shape[0] > 1 else x.shape[1])


def skrull_loss_workspace(x, weight, backward: bool) -> int:
    """Bytes that skrull_loss_fwd or skrull_loss_bwd asks for; SkrullError where the sizes are outside the limits."""
    n = int(lib().skrull_loss_workspace(ctypes.byref(_loss_of(x, weight, None)), int(backward)))
    if n == 0:
        _check(SKRULL_EINVAL)
    return n


def skrull_loss_fwd(x, weight, target, loss, lse, workspace, stream=None):
    """loss, lse (fp32 [rows]) of the rows x against the vocabulary's weight; rows with a negative target have none."""
    import torch
    _on_current_device(x, weight, target, loss, lse, workspace)
    p = _loss_of(x, weight, target)
    _check(lib().skrull_loss_fwd(ctypes.byref(p), _ptr(x), _ptr(weight), _ptr(target), _vector(loss, p.rows, torch.float32, "loss"),
                                 _vector(lse, p.rows, torch.float32, "lse"), *_scratch(workspace), _stream_ptr(stream)))


def skrull_loss_bwd(x, weight, target, lse, d_loss, dx, dweight, workspace, stream=None):
    """dx and dweight (either may be None) for the gradient d_loss (fp32 [rows])."""
    import torch
    _on_current_device(x, weight, target, lse, d_loss, dx, dweight, workspace)
    p = _loss_of(x, weight, target)
    for name, t, like in (("dx", dx, x), ("dweight", dweight, weight)):
        if t is not None and (t.dtype != torch.bfloat16 or t.shape != like.shape or not t.is_contiguous()):
            _refuse(f"{name} must be contiguous bf16 {list(like.shape)}")
    _check(lib().skrull_loss_bwd(ctypes.byref(p), _ptr(x), _ptr(weight), _ptr(target), _vector(lse, p.rows, torch.float32, "lse"),
                                 _vector(d_loss, p.rows, torch.float32, "d_loss"), None if dx is None else _ptr(dx),
                                 None if dweight is None else _ptr(dweight), *_scratch(workspace), _stream_ptr(stream)))
