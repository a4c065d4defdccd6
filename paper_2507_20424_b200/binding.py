"""ctypes binding of ``libdppf.so``: argument marshalling only.

Every function takes torch CUDA tensors (used purely as device memory) and
passes raw pointers, sizes and the current CUDA stream to the C entry point of
the same name (``include/dppf.h``).  There is no CPU fallback: if the library
is missing or a call returns an error status, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
from typing import NamedTuple

import torch

from . import build as _build

PATH_AUTO, PATH_TWO_KERNEL, PATH_COOPERATIVE, PATH_STAGED = 0, 1, 2, 3
OK, ERR_INVALID_ARG, ERR_ALIGNMENT, ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT = range(6)

EXPORTS = ("dppf_workspace_bytes", "dppf_consensus", "dppf_consensus_ex", "dppf_local_step",
           "dppf_local_step_and_consensus", "dppf_local_step_and_consensus_ex",
           "dppf_consensus_host", "dppf_device_status", "dppf_device_schedule", "dppf_status_string", "dppf_launch_count",
           "dppf_consensus_static", "dppf_static_device_status", "dppf_consensus_general", "dppf_consensus_general_ex",
           "dppf_distance_partials", "dppf_update_from_sums", "dppf_worker_update", "dppf_adamw_step_and_consensus_ex",
           "dppf_consensus_rounds", "dppf_consensus_rounds_ex", "dppf_debug_set_poll_limits",
           "dppf_adamw_step", "dppf_adamw_step_and_consensus",
           "dppf_embedding", "dppf_embedding_grad", "dppf_embedding_workspace_bytes",
           "dppf_policy_loss", "dppf_policy_workspace_bytes", "dppf_adamw_tensors",
           "dppf_lambda_schedule", "dppf_lr_cosine", "dppf_qsr_period", "dppf_round_metrics")

FLOAT32, BFLOAT16 = 0, 1
STATE_BLOCK = 256            # elements that share a scale in the 8-bit optimiser states

_lib = None


class _Tensor(ctypes.Structure):      # dppf_tensor
    _fields_ = [(n, ctypes.c_void_p) for n in ("param", "grad", "exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale")] + \
               [("numel", ctypes.c_int64), ("decay", ctypes.c_float)]


class DppfError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


def library_path() -> str:
    return _build.LIB_PATH


def load(rebuild_if_stale: bool = False) -> ctypes.CDLL:
    """Load the shared library (building it first only when asked to)."""
    global _lib
    if _lib is not None:
        return _lib
    if rebuild_if_stale:
        _build.build()
    if not os.path.exists(_build.LIB_PATH):
        raise RuntimeError(f"{_build.LIB_PATH} not found: build it with "
                           "`python -m paper_2507_20424_b200.build` (no CPU fallback exists)")
    lib = ctypes.CDLL(_build.LIB_PATH)
    vp, f32, i32, i64, sz = ctypes.c_void_p, ctypes.c_float, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
    lib.dppf_workspace_bytes.argtypes = [i32, i64]
    lib.dppf_workspace_bytes.restype = sz
    lib.dppf_consensus.argtypes = [vp, i32, i64, i64, f32, f32, vp, vp, sz, vp]
    lib.dppf_consensus_ex.argtypes = [vp, i32, i64, i64, f32, f32, vp, vp, sz, i32, vp]
    lib.dppf_local_step.argtypes = [vp, vp, vp, i32, i64, i64, f32, f32, f32, vp]
    lib.dppf_local_step_and_consensus.argtypes = [vp, vp, vp, i32, i64, i64, f32, f32, f32, f32, f32, vp, vp, sz, vp]
    lib.dppf_local_step_and_consensus_ex.argtypes = [vp, vp, vp, i32, i64, i64, f32, f32, f32, f32, f32, vp, vp, sz, i32, vp]
    lib.dppf_consensus_host.argtypes = [vp, i32, i64, i64, f32, f32, vp, vp, vp, sz, vp]
    lib.dppf_device_status.argtypes = [vp, vp]
    lib.dppf_device_schedule.argtypes = [vp, vp]
    lib.dppf_device_schedule.restype = i32
    lib.dppf_lambda_schedule.argtypes = [i32, f32, i64, i64]
    lib.dppf_lambda_schedule.restype = f32
    lib.dppf_lr_cosine.argtypes = [f32, i64, i64]
    lib.dppf_lr_cosine.restype = f32
    lib.dppf_qsr_period.argtypes = [i64, f32, f32]
    lib.dppf_qsr_period.restype = i64
    lib.dppf_round_metrics.argtypes = [ctypes.POINTER(f32), i32, f32, f32, ctypes.POINTER(f32),
                                       ctypes.POINTER(f32), ctypes.POINTER(f32)]
    lib.dppf_round_metrics.restype = i32
    lib.dppf_adamw_step.argtypes = [vp, vp, vp, vp, i32, i64, i64, f32, f32, f32, f32, f32, i32, vp]
    lib.dppf_adamw_step.restype = i32
    lib.dppf_adamw_step_and_consensus.argtypes = [vp, vp, vp, vp, i32, i64, i64, f32, f32, f32, f32, f32, i32,
                                                  f32, f32, vp, vp, sz, vp]
    lib.dppf_adamw_step_and_consensus.restype = i32
    lib.dppf_consensus_general.argtypes = [vp, i32, i64, i64, f32, f32, ctypes.POINTER(f32), i32, i32, vp, vp,
                                           vp, sz, vp]
    lib.dppf_consensus_general.restype = i32
    lib.dppf_consensus_rounds.argtypes = [vp, i32, i64, i64, f32, f32, ctypes.POINTER(f32), i32, vp, vp, sz, vp]
    lib.dppf_consensus_rounds.restype = i32
    lib.dppf_consensus_rounds_ex.argtypes = [vp, i32, i64, i64, f32, f32, ctypes.POINTER(f32), i32, vp, vp, sz,
                                             i32, vp]
    lib.dppf_consensus_rounds_ex.restype = i32
    lib.dppf_distance_partials.argtypes = [vp, i32, i64, i64, vp, vp, sz, vp]
    lib.dppf_distance_partials.restype = i32
    lib.dppf_update_from_sums.argtypes = [vp, i32, i64, i64, f32, f32, vp, vp, vp]
    lib.dppf_update_from_sums.restype = i32
    lib.dppf_worker_update.argtypes = [vp, vp, f32, i64, f32, f32, vp, vp, sz, vp]
    lib.dppf_worker_update.restype = i32
    lib.dppf_static_device_status.argtypes = [vp]
    lib.dppf_static_device_status.restype = i32
    lib.dppf_consensus_general_ex.argtypes = [vp, i32, i64, i64, f32, f32, ctypes.POINTER(f32), i32, i32, vp, vp,
                                              vp, sz, i32, vp]
    lib.dppf_consensus_general_ex.restype = i32
    lib.dppf_adamw_step_and_consensus_ex.argtypes = [vp, vp, vp, vp, i32, i64, i64, f32, f32, f32, f32, f32, i32,
                                                     f32, f32, vp, vp, sz, i32, vp]
    lib.dppf_adamw_step_and_consensus_ex.restype = i32
    lib.dppf_debug_set_poll_limits.argtypes = [i32, i32]
    lib.dppf_debug_set_poll_limits.restype = i32
    lib.dppf_consensus_static.argtypes = [vp, i32, i64, i64, f32, f32, vp, vp]
    lib.dppf_consensus_static.restype = i32
    lib.dppf_embedding.argtypes = [vp, i32, i64, i32, i64, vp, i32, i64, f32, vp, i32, i64, vp]
    lib.dppf_embedding.restype = i32
    lib.dppf_embedding_workspace_bytes.argtypes = [i64, i32]
    lib.dppf_embedding_workspace_bytes.restype = sz
    lib.dppf_embedding_grad.argtypes = [vp, i32, i64, vp, i32, i64, f32, vp, i32, i64, i32, i64, i32, vp, sz, vp]
    lib.dppf_embedding_grad.restype = i32
    lib.dppf_policy_workspace_bytes.argtypes = [i64]
    lib.dppf_policy_workspace_bytes.restype = sz
    lib.dppf_policy_loss.argtypes = [vp, i32, i64, i32, i64, vp, i32, vp, vp, vp, vp, f32, f32, f32, f32, vp, vp, vp, i64, vp, sz, vp]
    lib.dppf_policy_loss.restype = i32
    lib.dppf_adamw_tensors.argtypes = [ctypes.POINTER(_Tensor), i32, i32, i32, i32, f32, f32, f32, f32, f32, i32, vp, ctypes.c_uint32, vp]
    lib.dppf_adamw_tensors.restype = i32
    lib.dppf_status_string.argtypes = [i32]
    lib.dppf_status_string.restype = ctypes.c_char_p
    lib.dppf_launch_count.argtypes = [i32, i64, i32, i32]
    for name in ("dppf_consensus", "dppf_consensus_ex", "dppf_local_step", "dppf_local_step_and_consensus",
                 "dppf_local_step_and_consensus_ex", "dppf_consensus_host", "dppf_device_status", "dppf_device_schedule",
                 "dppf_launch_count"):
        getattr(lib, name).restype = i32
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().dppf_status_string(int(status)).decode()


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _check(rc: int, where: str) -> None:
    if rc != OK:
        raise DppfError(rc, where)


def _dims(x: torch.Tensor, d):
    if x.dim() != 2 or x.dtype != torch.float32 or not x.is_cuda or x.stride(1) != 1:
        raise ValueError("expected a 2-D fp32 CUDA tensor with unit column stride")
    M, ld = x.shape[0], x.stride(0)
    return M, (x.shape[1] if d is None else int(d)), ld


def workspace_bytes(M: int, d: int) -> int:
    return int(load().dppf_workspace_bytes(int(M), int(d)))


def alloc_workspace(M: int, d: int, device="cuda") -> torch.Tensor:
    n = workspace_bytes(M, d)
    if n == 0:
        raise ValueError("invalid M or d")
    return torch.empty(n, dtype=torch.uint8, device=device)


def alloc_rows(M: int, d: int, device="cuda", fill=None) -> torch.Tensor:
    """[M, ld] fp32 device buffer with 128-byte rows (ld = d rounded up to 32)."""
    ld = (int(d) + 31) // 32 * 32
    t = torch.empty((M, ld), dtype=torch.float32, device=device)
    if fill is not None:
        t.fill_(fill)
    return t


def _ptr(t):
    return None if t is None else t.data_ptr()


def dppf_consensus(x, alpha, lam, norms_out=None, ws=None, d=None, path=PATH_AUTO):
    """One pull-push round in place on ``x[M, ld]``; returns the workspace used."""
    M, d, ld = _dims(x, d)
    ws = alloc_workspace(M, d, x.device) if ws is None else ws
    rc = load().dppf_consensus_ex(x.data_ptr(), M, d, ld, alpha, lam, _ptr(norms_out),
                                  ws.data_ptr(), ws.numel(), int(path), _stream())
    _check(rc, "dppf_consensus")
    return ws


def dppf_consensus_rounds(x, alpha, lam, n_rounds, lambdas=None, norms_out=None, ws=None, d=None, path=PATH_AUTO):
    """``n_rounds`` rounds in place on ``x[M, ld]`` in one pass sequence; ``lambdas`` (host
    sequence of n_rounds floats) overrides ``lam`` per round; ``norms_out`` is [n_rounds, M]."""
    M, d, ld = _dims(x, d)
    ws = alloc_workspace(M, d, x.device) if ws is None else ws
    lp = None
    if lambdas is not None:
        if len(lambdas) != n_rounds:
            raise ValueError("lambdas must have one entry per round")
        lp = (ctypes.c_float * n_rounds)(*[float(v) for v in lambdas])
    if norms_out is not None and norms_out.numel() < n_rounds * M:
        raise ValueError("norms_out must hold n_rounds x M floats")
    rc = load().dppf_consensus_rounds_ex(x.data_ptr(), M, d, ld, alpha, lam, lp, int(n_rounds), _ptr(norms_out),
                                         ws.data_ptr(), ws.numel(), int(path), _stream())
    _check(rc, "dppf_consensus_rounds")
    return ws


def dppf_distance_partials(x, sums_out, ws=None, d=None):
    """Sums of squared distances to the column average over this column shard -> ``sums_out``
    (fp64 CUDA tensor of M entries).  Returns the workspace used."""
    M, d, ld = _dims(x, d)
    if sums_out.dtype != torch.float64 or not sums_out.is_cuda or sums_out.numel() < M:
        raise ValueError("sums_out must be an fp64 CUDA tensor with M entries")
    ws = alloc_workspace(M, d, x.device) if ws is None else ws
    _check(load().dppf_distance_partials(x.data_ptr(), M, d, ld, sums_out.data_ptr(), ws.data_ptr(), ws.numel(),
                                         _stream()), "dppf_distance_partials")
    return ws


def dppf_update_from_sums(x, alpha, lam, sums, norms_out=None, d=None):
    """Update pass on this column shard from the sums of squares totalled over all shards."""
    M, d, ld = _dims(x, d)
    if sums.dtype != torch.float64 or not sums.is_cuda or sums.numel() < M:
        raise ValueError("sums must be an fp64 CUDA tensor with M entries")
    _check(load().dppf_update_from_sums(x.data_ptr(), M, d, ld, alpha, lam, sums.data_ptr(), _ptr(norms_out),
                                        _stream()), "dppf_update_from_sums")


def dppf_worker_update(x, x_reduced, scale, alpha, lam, norm_out=None, ws=None):
    """This worker's pull-push update from the all-reduced parameters (one replica per GPU):
    ``x`` and ``x_reduced`` are 1-D fp32 CUDA tensors of the same length; x_A = scale * x_reduced."""
    for t in (x, x_reduced):
        if t.dim() != 1 or t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous():
            raise ValueError("expected contiguous 1-D fp32 CUDA tensors")
    if x.numel() != x_reduced.numel():
        raise ValueError("x and x_reduced must have the same length")
    d = x.numel()
    ws = alloc_workspace(1, d, x.device) if ws is None else ws
    _check(load().dppf_worker_update(x.data_ptr(), x_reduced.data_ptr(), scale, d, alpha, lam, _ptr(norm_out),
                                     ws.data_ptr(), ws.numel(), _stream()), "dppf_worker_update")
    return ws


def debug_set_poll_limits(first_pass_polls=-1, later_pass_polls=-1) -> None:
    """Testing hook: poll budget of the bounded waits of later calls (negative = default)."""
    load().dppf_debug_set_poll_limits(int(first_pass_polls), int(later_pass_polls))


PUSH_FROM_AVERAGE, PUSH_FROM_CONSENSUS = 0, 1


def dppf_consensus_general(x, alpha, lam, weights=None, push_from=PUSH_FROM_AVERAGE, two_term=False,
                           norms_out=None, push_norms_out=None, ws=None, d=None, path=PATH_AUTO):
    """General round in place on ``x[M, ld]``: consensus variable from ``weights`` (host
    sequence of M floats, None = plain average), push from x_A or x_C, optional second term."""
    M, d, ld = _dims(x, d)
    ws = alloc_workspace(M, d, x.device) if ws is None else ws
    wp = None
    if weights is not None:
        if len(weights) != M:
            raise ValueError("weights must have one entry per worker")
        wp = (ctypes.c_float * M)(*[float(v) for v in weights])
    rc = load().dppf_consensus_general_ex(x.data_ptr(), M, d, ld, alpha, lam, wp, int(push_from),
                                          int(bool(two_term)), _ptr(norms_out), _ptr(push_norms_out),
                                          ws.data_ptr(), ws.numel(), int(path), _stream())
    _check(rc, "dppf_consensus_general")
    return ws


def dppf_consensus_static(x, alpha, lam, norms_out=None, d=None):
    """One round in place on ``x[M, ld]`` using the library's built-in scratch: no
    workspace argument and no allocation anywhere in the call (M <= 16).  Calls that
    may overlap on the GPU must be ordered by the caller; they share the scratch."""
    M, d, ld = _dims(x, d)
    rc = load().dppf_consensus_static(x.data_ptr(), M, d, ld, alpha, lam, _ptr(norms_out), _stream())
    _check(rc, "dppf_consensus_static")


def dppf_local_step(x, v, g, lr, momentum, weight_decay, d=None):
    M, d, ld = _dims(x, d)
    for t in (v, g):
        if _dims(t, d) != (M, d, ld):
            raise ValueError("x, v and g must share shape and row stride")
    _check(load().dppf_local_step(x.data_ptr(), v.data_ptr(), g.data_ptr(), M, d, ld,
                                  lr, momentum, weight_decay, _stream()), "dppf_local_step")


def dppf_local_step_and_consensus(x, v, g, lr, momentum, weight_decay, alpha, lam,
                                  norms_out=None, ws=None, d=None, path=PATH_AUTO):
    M, d, ld = _dims(x, d)
    for t in (v, g):
        if _dims(t, d) != (M, d, ld):
            raise ValueError("x, v and g must share shape and row stride")
    ws = alloc_workspace(M, d, x.device) if ws is None else ws
    rc = load().dppf_local_step_and_consensus_ex(
        x.data_ptr(), v.data_ptr(), g.data_ptr(), M, d, ld, lr, momentum, weight_decay,
        alpha, lam, _ptr(norms_out), ws.data_ptr(), ws.numel(), int(path), _stream())
    _check(rc, "dppf_local_step_and_consensus")
    return ws


def _same_shape(x, others, d):
    M, d, ld = _dims(x, d)
    for t in others:
        if _dims(t, d) != (M, d, ld):
            raise ValueError("all buffers must share shape and row stride")
    return M, d, ld


def dppf_adamw_step(x, exp_avg, exp_avg_sq, g, lr, beta1, beta2, eps, weight_decay, step, d=None):
    M, d, ld = _same_shape(x, (exp_avg, exp_avg_sq, g), d)
    _check(load().dppf_adamw_step(x.data_ptr(), exp_avg.data_ptr(), exp_avg_sq.data_ptr(), g.data_ptr(), M, d, ld,
                                  lr, beta1, beta2, eps, weight_decay, int(step), _stream()), "dppf_adamw_step")


def dppf_adamw_step_and_consensus(x, exp_avg, exp_avg_sq, g, lr, beta1, beta2, eps, weight_decay, step,
                                  alpha, lam, norms_out=None, ws=None, d=None, path=PATH_AUTO):
    M, d, ld = _same_shape(x, (exp_avg, exp_avg_sq, g), d)
    ws = alloc_workspace(M, d, x.device) if ws is None else ws
    rc = load().dppf_adamw_step_and_consensus_ex(
        x.data_ptr(), exp_avg.data_ptr(), exp_avg_sq.data_ptr(), g.data_ptr(), M, d, ld, lr, beta1, beta2, eps,
        weight_decay, int(step), alpha, lam, _ptr(norms_out), ws.data_ptr(), ws.numel(), int(path), _stream())
    _check(rc, "dppf_adamw_step_and_consensus")
    return ws


def dppf_consensus_host(x_host, alpha, lam, norms_host, x_dev, ws, d=None):
    """Round on host-resident replicas (pinned CPU tensors), staged through ``x_dev``."""
    M, d, ld = _dims(x_dev, d)
    if x_host.dtype != torch.float32 or x_host.is_cuda or x_host.shape[0] != M or x_host.stride(0) != ld:
        raise ValueError("x_host must be a CPU fp32 tensor with the row stride of x_dev")
    rc = load().dppf_consensus_host(x_host.data_ptr(), M, d, ld, alpha, lam, _ptr(norms_host),
                                    x_dev.data_ptr(), ws.data_ptr(), ws.numel(), _stream())
    _check(rc, "dppf_consensus_host")


SCHEDULE_FIXED, SCHEDULE_DECREASING, SCHEDULE_INCREASING = 0, 1, 2


def dppf_lambda_schedule(kind, lam, t, T) -> float:
    return float(load().dppf_lambda_schedule(int(kind), lam, int(t), int(T)))


def dppf_lr_cosine(lr_max, t, T) -> float:
    return float(load().dppf_lr_cosine(lr_max, int(t), int(T)))


def dppf_qsr_period(tau_base, beta, lr_t) -> int:
    return int(load().dppf_qsr_period(int(tau_base), beta, lr_t))


def dppf_round_metrics(norms, alpha, lam):
    """(mean distance, [pull strength per worker], push strength) from host distances."""
    M = len(norms)
    arr = (ctypes.c_float * M)(*[float(v) for v in norms])
    pull = (ctypes.c_float * M)()
    mean, push = ctypes.c_float(), ctypes.c_float()
    _check(load().dppf_round_metrics(arr, M, alpha, lam, ctypes.byref(mean), pull, ctypes.byref(push)),
           "dppf_round_metrics")
    return mean.value, list(pull), push.value


def dppf_device_status(ws) -> int:
    return int(load().dppf_device_status(ws.data_ptr(), _stream()))


def dppf_device_schedule(ws) -> int:
    """PATH_* of the kernels that ran the last call on this workspace (synchronises the stream)."""
    return int(load().dppf_device_schedule(ws.data_ptr(), _stream()))


def launch_count(M: int, d: int, path=PATH_AUTO, fused=False) -> int:
    return int(load().dppf_launch_count(int(M), int(d), int(path), int(bool(fused))))


def adamw_launch_count(M: int, path=PATH_AUTO) -> int:
    """Kernel launches of one dppf_adamw_step_and_consensus call."""
    return int(load().dppf_launch_count(int(M), 1, int(path), 2))


def dppf_static_device_status() -> int:
    """Status word of the built-in scratch that dppf_consensus_static uses on the current device."""
    return int(load().dppf_static_device_status(_stream()))


# ---------------------------------------------------------------- a worker's local step on a language model
# The functions below launch on the current stream of the device that holds their tensors.

_TYPES = {torch.float32: FLOAT32, torch.bfloat16: BFLOAT16}
_ID_BITS = {torch.int32: 32, torch.int64: 64}


def _type(t: torch.Tensor, what: str) -> int:
    if t.dtype not in _TYPES:
        raise ValueError(f"{what} must be fp32 or bf16, not {t.dtype}")
    return _TYPES[t.dtype]


def _matrix(t: torch.Tensor, what: str):
    """(rows, columns, row stride) of a 2-D CUDA tensor with unit column stride."""
    if t.dim() != 2 or not t.is_cuda or (t.stride(1) != 1 and t.shape[1] > 1):
        raise ValueError(f"{what} must be a 2-D CUDA tensor with unit column stride")
    rows, cols = t.shape
    return rows, cols, (t.stride(0) if rows > 1 else cols)     # the stride of a single row says nothing


def _vector(t: torch.Tensor, n: int, what: str, device, dtypes=(torch.float32,)) -> torch.Tensor:
    if t.dtype not in dtypes or t.device != device or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous tensor of {n} entries of type {' or '.join(str(d) for d in dtypes)} on {device}")
    return t


def _workspace(ws: torch.Tensor, device) -> torch.Tensor:
    """ws, whose bytes the kernels will use: they must be memory of this device, and all of them there."""
    if ws.device != device or not ws.is_contiguous():
        raise ValueError(f"ws must be a contiguous tensor on {device}")
    return ws


def _call(device, fn, where, *args):
    """fn(*args, stream) with `device` current; raises on a status other than OK."""
    if device.index == torch._C._cuda_getDevice():            # the calls behind torch.cuda.current_device() and
        rc = fn(*args, torch._C._cuda_getCurrentRawStream(device.index))   # current_stream(): a microsecond less a call
    else:
        with torch.cuda.device(device):
            rc = fn(*args, torch._C._cuda_getCurrentRawStream(device.index))
    if rc != OK:
        raise DppfError(rc, where)


def dppf_embedding(table, ids, scale=1.0, out=None, out_dtype=None):
    """Rows ``ids`` of ``table[V, H]`` times ``scale`` -> ``out[*ids.shape, H]`` (zeros where an id is
    outside [0, V)).  ``out_dtype`` (default: the table's) is used when ``out`` is not given."""
    V, H, ld = _matrix(table, "table")
    dev = table.device
    if ids.dtype not in _ID_BITS or ids.device != dev or not ids.is_contiguous():
        _vector(ids, ids.numel(), "ids", dev, tuple(_ID_BITS))
    T = ids.numel()
    if out is None:
        out = flat = table.new_empty((*ids.shape, H), dtype=out_dtype)
        ld_out = H
    else:
        if out.device != dev or out.numel() != T * H or out.shape[-1:] != (H,):
            raise ValueError("out must hold one row of H columns per id, on the table's device")
        flat = out if out.dim() == 2 else out.view(-1, H)
        _, _, ld_out = _matrix(flat, "out")
    _call(dev, load().dppf_embedding, "dppf_embedding", table.data_ptr(), _type(table, "table"), V, H, ld, ids.data_ptr(), _ID_BITS[ids.dtype], T, scale,
          flat.data_ptr(), _type(flat, "out"), ld_out)
    return out


def embedding_workspace_bytes(T: int, H: int) -> int:
    return int(load().dppf_embedding_workspace_bytes(int(T), int(H)))


def alloc_embedding_workspace(T: int, H: int, device="cuda") -> torch.Tensor:
    n = embedding_workspace_bytes(T, H)
    if n == 0:
        raise ValueError("invalid T or H")
    return torch.empty(n, dtype=torch.uint8, device=device)


def dppf_embedding_grad(grad_out, ids, grad_table, scale=1.0, accumulate=False, ws=None):
    """Gradient of :func:`dppf_embedding` with respect to the table, written to (or, with ``accumulate``,
    added to) ``grad_table[V, H]``; ``grad_out[*ids.shape, H]``.  Returns the workspace used (None for no tokens)."""
    V, H, ld = _matrix(grad_table, "grad_table")
    dev = grad_table.device
    ids = _vector(ids, ids.numel(), "ids", dev, tuple(_ID_BITS))
    T = ids.numel()
    if grad_out.device != dev or grad_out.numel() != T * H or grad_out.shape[-1:] != (H,):
        raise ValueError("grad_out must hold one row of H columns per id, on the table's device")
    flat = grad_out if grad_out.dim() == 2 else grad_out.view(-1, H)
    _, _, ld_out = _matrix(flat, "grad_out")
    if ws is not None:
        _workspace(ws, dev)
    elif T:
        ws = alloc_embedding_workspace(T, H, dev)
    _call(dev, load().dppf_embedding_grad, "dppf_embedding_grad", flat.data_ptr(), _type(flat, "grad_out"), ld_out, ids.data_ptr(), _ID_BITS[ids.dtype], T, scale,
          grad_table.data_ptr(), _type(grad_table, "grad_table"), V, H, ld, int(bool(accumulate)), _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size())
    return ws


class PolicyLoss(NamedTuple):
    loss: torch.Tensor          # 0-d: sum of weight * loss
    kl: torch.Tensor            # 0-d: sum of weight * KL estimate
    clipped: torch.Tensor       # 0-d: sum of weight over clipped tokens
    logp: torch.Tensor          # [T]
    ws: torch.Tensor            # the workspace used; what was given (or None) where there was no token


def alloc_policy_workspace(T: int, device="cuda") -> torch.Tensor:
    """Workspace of :func:`dppf_policy_loss` for up to T tokens, zeroed as its first call needs it."""
    n = int(load().dppf_policy_workspace_bytes(int(T)))
    if n == 0:
        raise ValueError("invalid T")
    return torch.zeros(n, dtype=torch.uint8, device=device)


def dppf_policy_loss(logits, targets, old_logp, advantage, weight, ref_logp=None, clip_low=0.2, clip_high=0.2, kl_coef=0.0,
                     temperature=1.0, grad_logits=None, ws=None) -> PolicyLoss:
    """Clipped policy loss with a KL term from ``logits[T, V]``; with ``grad_logits`` (may be ``logits``) also its
    gradient.  ``weight`` carries mask and normalisation; rows with weight 0 are not read.  No tokens: zero sums, no launch."""
    T, V, ld = _matrix(logits, "logits")
    dev, code = logits.device, _type(logits, "logits")
    if targets.device != dev or targets.numel() != T or targets.dtype not in _ID_BITS or not targets.is_contiguous():
        _vector(targets, T, "targets", dev, tuple(_ID_BITS))
    for t in (old_logp, advantage, weight, ref_logp):             # quickly; _vector says what is wrong
        if t is not None and (t.dtype is not torch.float32 or t.numel() != T or t.device != dev or not t.is_contiguous()):
            _vector(t, T, "old_logp, advantage, weight and ref_logp", dev)
    ld_grad, grad_ptr = 0, None
    if grad_logits is not None:
        rows, cols, ld_grad = _matrix(grad_logits, "grad_logits")
        if grad_logits.dtype != logits.dtype or grad_logits.device != dev or rows != T or cols != V:
            raise ValueError("grad_logits must have the type, shape and device of logits")
        grad_ptr = grad_logits.data_ptr()
    if T == 0:
        none = torch.zeros(3, dtype=torch.float32, device=dev)
        return PolicyLoss(*none.unbind(), none[:0], ws)
    ws = alloc_policy_workspace(T, dev) if ws is None else _workspace(ws, dev)
    out = logits.new_empty(3 + T, dtype=torch.float32)
    sums_ptr = out.data_ptr()
    _call(dev, load().dppf_policy_loss, "dppf_policy_loss", logits.data_ptr(), code, T, V, ld, targets.data_ptr(), _ID_BITS[targets.dtype], old_logp.data_ptr(),
          None if ref_logp is None else ref_logp.data_ptr(), advantage.data_ptr(), weight.data_ptr(), clip_low, clip_high, kl_coef, temperature, sums_ptr,
          sums_ptr + 12, grad_ptr, ld_grad, ws.data_ptr(), ws.nbytes)
    sums, logp = out.split_with_sizes((3, T))
    loss, kl, clipped = sums.unbind()
    return PolicyLoss(loss, kl, clipped, logp, ws)


class AdamWTensors:
    """The tensors of :func:`dppf_adamw_tensors`: parameters, gradients and optimiser state, held for as long as
    the object lives.  ``state_bits`` 32: fp32 moments; 8: e4m3 codes with one fp32 scale per 256 elements (of the
    first moment, and of the root of the second; for beta1 up to 0.95, above which the first moment follows falling
    gradients too slowly).  State that is not given starts at zero.  ``decay``: factor on the weight decay per tensor (default 1).

    The step writes to the memory that the tensors have when the object is made (and reads the gradients' when they are
    bound).  That memory is kept alive: a tensor that is given other memory later, as by ``p.data = q``, is not followed."""

    def __init__(self, params, grads, state_bits=32, exp_avgs=None, exp_avg_sqs=None, exp_avg_scales=None, exp_avg_sq_scales=None, decay=None):
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32")
        self.params, self.state_bits = list(params), state_bits
        if not self.params:
            raise ValueError("no tensors")
        self.device, n = self.params[0].device, len(self.params)
        self.param_type = _type(self.params[0], "params")
        dtype = torch.float32 if state_bits == 32 else torch.float8_e4m3fn
        sizes = [p.numel() for p in self.params]
        blocks = [-(-k // STATE_BLOCK) for k in sizes]

        def state(given, counts, kind, what):
            if given is None:
                return [torch.zeros(c, dtype=kind, device=self.device) for c in counts]
            given = list(given)
            if len(given) != n:
                raise ValueError(f"{what} must have one entry per tensor")
            return [_vector(t, c, what, self.device, (kind,)) for t, c in zip(given, counts)]

        for p in self.params:
            _vector(p, p.numel(), "params", self.device, (self.params[0].dtype,))
        if not self.params[0].is_cuda:
            raise ValueError("params must be CUDA tensors")
        self.exp_avgs = state(exp_avgs, sizes, dtype, "exp_avgs")
        self.exp_avg_sqs = state(exp_avg_sqs, sizes, dtype, "exp_avg_sqs")
        self.exp_avg_scales = self.exp_avg_sq_scales = None
        if state_bits == 8:
            self.exp_avg_scales = state(exp_avg_scales, blocks, torch.float32, "exp_avg_scales")
            self.exp_avg_sq_scales = state(exp_avg_sq_scales, blocks, torch.float32, "exp_avg_sq_scales")
        self.decay = [1.0] * n if decay is None else [float(d) for d in decay]
        if len(self.decay) != n:
            raise ValueError("decay must have one entry per tensor")
        width, code = self.params[0].element_size(), state_bits // 8
        arrays = [("param", self.params, sizes, width), ("exp_avg", self.exp_avgs, sizes, code), ("exp_avg_sq", self.exp_avg_sqs, sizes, code)]
        if state_bits == 8:
            arrays += [("exp_avg_scale", self.exp_avg_scales, blocks, 4), ("exp_avg_sq_scale", self.exp_avg_sq_scales, blocks, 4)]
        self._table, self._sizes, self._memory = (_Tensor * n)(), sizes, []
        for e, count, d in zip(self._table, sizes, self.decay):
            e.numel, e.decay = count, d
        starts, ends = [], []                                     # of what the step writes
        for field, ts, counts, each in arrays:
            at = [t.data_ptr() for t in ts]
            for e, pointer in zip(self._table, at):
                setattr(e, field, pointer)
            self._memory += [t.untyped_storage() for t in ts]     # stays, even if a tensor is given other memory
            starts += [a for a, c in zip(at, counts) if c]
            ends += [a + c * each for a, c in zip(at, counts) if c]
        # All tensors are updated side by side, so none may share memory (as tied weights listed twice would): in order, each start is
        # past the end before it.
        starts.sort()
        ends.sort()
        if any(after < end for after, end in zip(starts[1:], ends)):
            raise ValueError("parameters and optimiser states must not overlap")
        self.bind_grads(grads)

    def bind_grads(self, grads) -> None:
        """Use these gradient tensors from now on (all fp32 or all bf16)."""
        grads = list(grads)
        if len(grads) != len(self.params):
            raise ValueError("grads must have one entry per tensor")
        self.grad_type = _type(grads[0], "grads")
        kind, dev = grads[0].dtype, self.device
        for n, g in zip(self._sizes, grads):                      # quickly; _vector says what is wrong
            if g.dtype is not kind or g.numel() != n or g.device != dev or not g.is_contiguous():
                _vector(g, n, "grads", dev, (kind,))
        self.grads, self._grad_memory = grads, [g.untyped_storage() for g in grads]
        for e, g in zip(self._table, grads):
            e.grad = g.data_ptr()


def dppf_adamw_tensors(tensors: AdamWTensors, lr, beta1, beta2, eps, weight_decay, step, grad_scale=None, seed=0) -> None:
    """One AdamW step on all tensors.  ``grad_scale``: fp32 CUDA tensor of one entry that multiplies the gradients
    (the step is skipped if it is not finite); ``seed``: for the rounding of 8-bit states, another one each step."""
    if grad_scale is not None:
        _vector(grad_scale, 1, "grad_scale", tensors.device)
    _call(tensors.device, load().dppf_adamw_tensors, "dppf_adamw_tensors", tensors._table, len(tensors.params), tensors.param_type, tensors.grad_type, tensors.state_bits,
          lr, beta1, beta2, eps, weight_decay, int(step), _ptr(grad_scale), int(seed) & 0xffffffff)
