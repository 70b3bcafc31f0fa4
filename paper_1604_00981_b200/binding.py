"""ctypes binding of libsgdb.so: the same names and arguments as include/sgdb.h.

This layer only marshals arguments (tensor -> device pointer, current torch stream
-> cudaStream_t).  Every step of the path runs in the library's CUDA kernels; if
the library is missing the import fails: there is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass, field

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsgdb.so")

SGDB_OK, SGDB_ERR_INVALID_ARG, SGDB_ERR_INSUFFICIENT, SGDB_ERR_CUDA, SGDB_ERR_UNSUPPORTED, SGDB_ERR_TIMEOUT = range(6)
SGDB_F32, SGDB_BF16 = 0, 1
SGDB_E4M3, SGDB_E5M2 = 0, 1
SGDB_SGD, SGDB_MOMENTUM, SGDB_RMSPROP, SGDB_ADAM, SGDB_ADAGRAD = range(5)
SGDB_MAX_WORKERS = 1024
SGDB_MAX_SEGMENTS = 4096
_KINDS = {"sgd": SGDB_SGD, "momentum": SGDB_MOMENTUM, "rmsprop": SGDB_RMSPROP, "adam": SGDB_ADAM,
          "adagrad": SGDB_ADAGRAD}

EXPORTS = (
    "sgdb_select", "sgdb_aggregate", "sgdb_update", "sgdb_step", "sgdb_step_segmented",
    "sgdb_select_deadline", "sgdb_step_deadline", "sgdb_step_ema", "sgdb_ema", "sgdb_learning_rate", "sgdb_accumulate_arrival", "sgdb_accumulate_arrival_ema", "sgdb_step_host", "sgdb_step_host_workspace_bytes", "sgdb_step_host_static",
    "sgdb_select_grouped", "sgdb_step_grouped", "sgdb_step_segmented_ema", "sgdb_step_segmented_deadline",
    "sgdb_accumulate_arrival_deadline", "sgdb_accumulate_close", "sgdb_set_tuning", "sgdb_set_arrival_tuning", "sgdb_strerror", "sgdb_version",
    "sgdb_step_rows", "sgdb_step_rows_ordered", "sgdb_shard_range", "sgdb_enable_peer_access", "sgdb_selftest_bounded_wait", "sgdb_set_wait_limit_ns",
    "sgdb_layer_norm", "sgdb_layer_norm_backward", "sgdb_layer_norm_backward_workspace_bytes",
    "sgdb_route", "sgdb_dispatch", "sgdb_combine", "sgdb_combine_backward",
    "sgdb_quantize", "sgdb_quantize_matrices", "sgdb_gate", "sgdb_gate_backward", "sgdb_experts_product",
    "sgdb_experts_gradient", "sgdb_experts_gradient_workspace_bytes",
    "sgdb_balance_loss", "sgdb_balance_loss_workspace_bytes", "sgdb_balance_loss_backward",
    "sgdb_orthogonalize", "sgdb_orthogonalize_workspace_bytes", "sgdb_step_orthogonal", "sgdb_step_orthogonal_workspace_bytes",
)
SGDB_STATIC_SCRATCH_BYTES = 8 << 20
SGDB_MAX_REPLICAS = 64
SGDB_SHARD_ALIGN = 64


class SgdbError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s: %s (status %d)" % (where, sgdb_strerror(status), status))


class _COpt(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("lr", ctypes.c_float), ("momentum", ctypes.c_float),
                ("decay", ctypes.c_float), ("beta1", ctypes.c_float), ("beta2", ctypes.c_float),
                ("eps", ctypes.c_float), ("step", ctypes.c_int64)]


class CSegment(ctypes.Structure):
    """sgdb_segment_t: one tensor of a multi-tensor model (all device pointers)."""

    _fields_ = [("theta", ctypes.c_void_p), ("state0", ctypes.c_void_p), ("state1", ctypes.c_void_p),
                ("grad", ctypes.c_void_p), ("ld", ctypes.c_int64), ("len", ctypes.c_int64)]


@dataclass
class Opt:
    """sgdb_opt_t.  `kind` is "sgd" | "momentum" | "rmsprop" | "adam" | "adagrad" (or the enum value)."""

    kind: object = "sgd"
    lr: float = 0.1
    momentum: float = 0.0
    decay: float = 0.0
    beta1: float = 0.0
    beta2: float = 0.0
    eps: float = 0.0
    step: int = 1

    def _c(self) -> _COpt:
        kind = _KINDS[self.kind] if isinstance(self.kind, str) else int(self.kind)
        return _COpt(kind, self.lr, self.momentum, self.decay, self.beta1, self.beta2, self.eps, self.step)


class _CNewtonSchulz(ctypes.Structure):
    _fields_ = [("steps", ctypes.c_int32), ("a", ctypes.c_float), ("b", ctypes.c_float), ("c", ctypes.c_float), ("eps", ctypes.c_float)]


class _COrthogonalOpt(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_float), ("momentum", ctypes.c_float), ("weight_decay", ctypes.c_float), ("scale", ctypes.c_float),
                ("nesterov", ctypes.c_int32), ("newton_schulz", _CNewtonSchulz)]


@dataclass
class NewtonSchulz:
    """The products of sgdb_orthogonalize: X <- (a I + b A + c A^2) X, `steps` times."""
    steps: int = 5
    a: float = 3.4445
    b: float = -4.7750
    c: float = 2.0315
    eps: float = 1e-7

    def _c(self) -> _CNewtonSchulz:
        return _CNewtonSchulz(self.steps, self.a, self.b, self.c, self.eps)


@dataclass
class OrthogonalOpt:
    """Hyper-parameters of sgdb_step_orthogonal."""
    lr: float = 0.02
    momentum: float = 0.95
    nesterov: bool = True
    weight_decay: float = 0.0
    scale: float = 1.0
    newton_schulz: NewtonSchulz = field(default_factory=NewtonSchulz)

    def _c(self) -> _COrthogonalOpt:
        return _COrthogonalOpt(self.lr, self.momentum, self.weight_decay, self.scale, int(self.nesterov), self.newton_schulz._c())


def _load():
    if not os.path.exists(LIB_PATH):
        # not built yet: compile it now if the CUDA toolkit is here; there is nothing else to fall back to
        try:
            from . import build as _build

            _build.build()
        except Exception as e:
            raise ImportError(
                "libsgdb.so is not built (%s) and building it failed: %s. Run `python -m paper_1604_00981_b200.build`; "
                "this package has no CPU fallback." % (LIB_PATH, e))
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    sigs = {
        "sgdb_select": (i32, [vp, vp, i32, i32, i32, vp, vp, vp, vp]),
        "sgdb_aggregate": (i32, [vp, i32, i64, i64, i32, vp, vp, vp, vp]),
        "sgdb_update": (i32, [vp, vp, vp, vp, i64, ctypes.POINTER(_COpt), vp, vp]),
        "sgdb_step": (i32, [vp, i32, i64, i64, vp, vp, i32, i32, i32, vp, vp, vp, ctypes.POINTER(_COpt), vp, vp, vp, vp]),
        "sgdb_select_deadline": (i32, [vp, vp, i32, i32, ctypes.c_float, i32, vp, vp, vp, vp]),
        "sgdb_step_deadline": (i32, [vp, i32, i64, i64, vp, vp, i32, i32, ctypes.c_float, i32, vp, vp, vp,
                                     ctypes.POINTER(_COpt), vp, vp, vp, vp]),
        "sgdb_step_ema": (i32, [vp, i32, i64, i64, vp, vp, i32, i32, i32, vp, vp, vp, ctypes.POINTER(_COpt), vp,
                                ctypes.c_float, vp, vp, vp, vp]),
        "sgdb_ema": (i32, [vp, vp, i64, ctypes.c_float, vp, vp]),
        "sgdb_learning_rate": (ctypes.c_double, [ctypes.c_double, ctypes.c_double, i64, i64, ctypes.c_double]),
        "sgdb_step_segmented": (i32, [vp, i32, i32, vp, vp, i32, i32, i32, ctypes.POINTER(_COpt), vp, vp, vp, vp]),
        "sgdb_step_segmented_ema": (i32, [vp, vp, ctypes.c_float, i32, i32, vp, vp, i32, i32, i32, ctypes.POINTER(_COpt),
                                          vp, vp, vp, vp]),
        "sgdb_step_segmented_deadline": (i32, [vp, i32, i32, vp, vp, i32, i32, ctypes.c_float, i32, ctypes.POINTER(_COpt),
                                               vp, vp, vp, vp]),
        "sgdb_accumulate_arrival_deadline": (i32, [vp, i32, i32, ctypes.c_float, i32, ctypes.c_float, i64, vp, vp, vp, vp]),
        "sgdb_accumulate_close": (i32, [i32, i32, i64, vp, vp, vp, vp, vp, ctypes.POINTER(_COpt), vp, ctypes.c_float, vp, vp]),
        "sgdb_select_grouped": (i32, [vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, vp, vp]),
        "sgdb_step_grouped": (i32, [vp, i32, i64, i64, vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, ctypes.POINTER(_COpt),
                                    vp, vp, vp, vp, vp]),
        "sgdb_step_rows": (i32, [vp, i32, i64, vp, vp, i32, i32, i32, vp, vp, vp, ctypes.POINTER(_COpt), vp, i32,
                                 vp, vp, vp, vp]),
        "sgdb_step_rows_ordered": (i32, [vp, i32, i32, i64, i32, vp, vp, vp, vp, vp, ctypes.POINTER(_COpt), vp, i32, vp]),
        "sgdb_shard_range": (i32, [i64, i32, i32, ctypes.POINTER(i64), ctypes.POINTER(i64)]),
        "sgdb_accumulate_arrival": (i32, [vp, i32, i32, i32, i32, i64, vp, vp, vp, vp, vp, ctypes.POINTER(_COpt), vp, vp]),
        "sgdb_accumulate_arrival_ema": (i32, [vp, i32, i32, i32, i32, i64, vp, vp, vp, vp, vp, ctypes.POINTER(_COpt), vp,
                                              ctypes.c_float, vp, vp]),
        "sgdb_step_host": (i32, [vp, i32, i64, i64, vp, vp, i32, i32, i32, vp, vp, vp, ctypes.POINTER(_COpt),
                                 vp, vp, vp, vp, vp, sz, vp]),
        "sgdb_step_host_workspace_bytes": (sz, [i32, i64, i64, i32, i32]),
        "sgdb_step_host_static": (i32, [vp, i32, i64, i64, vp, vp, i32, i32, i32, vp, vp, vp, ctypes.POINTER(_COpt),
                                        vp, vp, vp, vp, vp]),
        "sgdb_selftest_bounded_wait": (i32, [i64, vp, vp]),
        "sgdb_enable_peer_access": (i32, [i32]),
        "sgdb_set_tuning": (i32, [i32, i32]),
        "sgdb_set_wait_limit_ns": (i32, [i64]),
        "sgdb_set_arrival_tuning": (i32, [i64, i32]),
        "sgdb_layer_norm": (i32, [vp, i32, i64, i64, i64, vp, vp, i32, ctypes.c_float, vp, i64, vp, vp, vp]),
        "sgdb_layer_norm_backward": (i32, [vp, i64, vp, i64, i32, i64, i64, vp, i32, vp, vp, vp, i64, vp, vp, i32, vp, sz, vp]),
        "sgdb_layer_norm_backward_workspace_bytes": (sz, [i64, i64]),
        "sgdb_route": (i32, [vp, i64, i32, i32, vp, vp, vp, vp]),
        "sgdb_dispatch": (i32, [vp, i32, i64, i64, i64, vp, i32, vp, i32, vp, i64, vp]),
        "sgdb_combine": (i32, [vp, i32, i64, i64, i64, vp, i32, vp, vp, i64, vp]),
        "sgdb_combine_backward": (i32, [vp, i64, vp, i64, i32, i64, i64, vp, i32, vp, vp, i32, vp, i64, vp, vp]),
        "sgdb_orthogonalize": (i32, [vp, i32, i32, i64, i64, i64, i64, ctypes.POINTER(_CNewtonSchulz), vp, i32, i64, i64, vp, sz,
                                     vp, vp]),
        "sgdb_quantize": (i32, [vp, i32, i64, i64, i64, vp, i32, i64, vp, i64, vp]),
        "sgdb_quantize_matrices": (i32, [vp, i32, i32, i64, i64, i64, i64, i32, vp, i64, i64, vp, i64, i64, vp, vp]),
        "sgdb_gate": (i32, [vp, i32, i64, i64, i64, i32, vp, i64, vp, i64, vp, i64, vp, i64, vp]),
        "sgdb_gate_backward": (i32, [vp, i64, i32, i64, i64, i32, vp, i64, vp, i64, vp, i64, vp]),
        "sgdb_experts_product": (i32, [vp, i32, i64, i64, i64, vp, i64, vp, i32, i32, i64, i64, i64, vp, i64, i64, i64, vp, vp, i32, i64, vp, vp]),
        "sgdb_experts_gradient": (i32, [vp, i32, i64, i64, i64, vp, i32, i64, i64, vp, i64, vp, i32, vp, i32, i64, i64, vp, sz, vp, vp]),
        "sgdb_experts_gradient_workspace_bytes": (sz, [i64, i64, i64, i32]),
        "sgdb_balance_loss": (i32, [vp, i32, i64, i32, i64, vp, i32, vp, vp, vp, vp, vp, sz, vp]),
        "sgdb_balance_loss_workspace_bytes": (sz, [i64, i32]),
        "sgdb_balance_loss_backward": (i32, [vp, vp, i32, i64, i32, i64, vp, vp, vp, i64, vp]),
        "sgdb_orthogonalize_workspace_bytes": (sz, [i32, i64, i64]),
        "sgdb_step_orthogonal": (i32, [vp, i32, i32, i64, i64, i64, vp, vp, i32, i32, i32, vp, vp,
                                       ctypes.POINTER(_COrthogonalOpt), vp, vp, vp, vp, sz, vp]),
        "sgdb_step_orthogonal_workspace_bytes": (sz, [i32, i64, i64]),
        "sgdb_strerror": (ctypes.c_char_p, [i32]),
        "sgdb_version": (ctypes.c_int, []),
    }
    for name, (res, args) in sigs.items():
        fn = getattr(lib, name)  # AttributeError here means the library lacks a declared symbol
        fn.restype, fn.argtypes = res, args
    return lib


_lib = _load()


# The current stream's handle without a torch.cuda.Stream object around it, where torch offers that: the calls of small
# operators are bound by the host.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream(stream=None) -> int:
    if stream is not None:
        return int(stream.cuda_stream)
    if _raw_stream is None:
        return int(torch.cuda.current_stream().cuda_stream)
    return _raw_stream(_current_device())


def _dev(x, dtype=None, name="tensor") -> int:
    """Device pointer of a CUDA tensor (None -> NULL)."""
    if x is None:
        return 0
    if not x.is_cuda or not x.is_contiguous():
        raise ValueError("%s must be a contiguous CUDA tensor" % name)
    if dtype is not None and x.dtype != dtype:
        raise ValueError("%s must have dtype %s, got %s" % (name, dtype, x.dtype))
    return x.data_ptr()


def _host(x, dtype=None, name="tensor") -> int:
    if x is None:
        return 0
    if x.is_cuda or not x.is_contiguous():
        raise ValueError("%s must be a contiguous host tensor" % name)
    if dtype is not None and x.dtype != dtype:
        raise ValueError("%s must have dtype %s, got %s" % (name, dtype, x.dtype))
    return x.data_ptr()


def _grad_dtype(g) -> int:
    if g.dtype == torch.float32:
        return SGDB_F32
    if g.dtype == torch.bfloat16:
        return SGDB_BF16
    raise ValueError("gradient rows must be float32 or bfloat16, got %s" % g.dtype)


def _check(status: int, where: str):
    if status != SGDB_OK:
        raise SgdbError(status, where)


def sgdb_strerror(status: int) -> str:
    return _lib.sgdb_strerror(int(status)).decode()


def sgdb_version() -> int:
    return int(_lib.sgdb_version())


def sgdb_selftest_bounded_wait(limit_ns: int, out, stream=None) -> None:
    """A wait for a barrier that nothing completes, with the kernels' own wait routine: out i32[3] receives
    {SGDB_ERR_TIMEOUT, nanoseconds waited, 1 if a second waiter was released by the give-up}."""
    _check(_lib.sgdb_selftest_bounded_wait(limit_ns, _dev(out, torch.int32, "out"), _stream(stream)),
           "sgdb_selftest_bounded_wait")


def sgdb_set_tuning(stages: int = 0, ctas_per_sm: int = 0) -> None:
    _check(_lib.sgdb_set_tuning(stages, ctas_per_sm), "sgdb_set_tuning")


def sgdb_set_wait_limit_ns(limit_ns: int = -1) -> None:
    """Patience of the waits inside the row-streaming kernels and the products of matrices in nanoseconds (negative: the 2 s default)."""
    _check(_lib.sgdb_set_wait_limit_ns(limit_ns), "sgdb_set_wait_limit_ns")


def sgdb_set_arrival_tuning(resident_bytes: int = -1, blocks_per_sm: int = 0) -> None:
    _check(_lib.sgdb_set_arrival_tuning(resident_bytes, blocks_per_sm), "sgdb_set_arrival_tuning")


def sgdb_select(arrival, tags, t: int, N: int, b: int, mask, order, info, stream=None) -> None:
    """arrival f32[W], tags i32[W] -> mask u8[W], order i32[N], info i32[2] (all CUDA tensors)."""
    _check(_lib.sgdb_select(_dev(arrival, torch.float32, "arrival"), _dev(tags, torch.int32, "tags"), t, N, b,
                            _dev(mask, torch.uint8, "mask"), _dev(order, torch.int32, "order"),
                            _dev(info, torch.int32, "info"), _stream(stream)), "sgdb_select")


def sgdb_aggregate(grad, P: int, N: int, order, info, mean, ld: int | None = None, stream=None) -> None:
    """grad [W, ld] (f32 or bf16) -> mean f32[P] of the rows named in order[N]."""
    ld = grad.stride(0) if ld is None else ld
    _check(_lib.sgdb_aggregate(_dev(grad, None, "grad"), _grad_dtype(grad), P, ld, N,
                               _dev(order, torch.int32, "order"), _dev(info, torch.int32, "info"),
                               _dev(mean, torch.float32, "mean"), _stream(stream)), "sgdb_aggregate")


def sgdb_update(theta, state0, state1, mean, opt: Opt, info=None, P: int | None = None, stream=None) -> None:
    P = theta.numel() if P is None else P
    c = opt._c()
    _check(_lib.sgdb_update(_dev(theta, torch.float32, "theta"), _dev(state0, torch.float32, "state0"),
                            _dev(state1, torch.float32, "state1"), _dev(mean, torch.float32, "mean"), P,
                            ctypes.byref(c), _dev(info, torch.int32, "info"), _stream(stream)), "sgdb_update")


def sgdb_step(grad, P: int, arrival, tags, t: int, N: int, b: int, theta, state0, state1, opt: Opt,
              mask, order, info, ld: int | None = None, stream=None) -> None:
    """One fused iteration: select + mean of the kept rows + optimizer rule."""
    ld = grad.stride(0) if ld is None else ld
    c = opt._c()
    _check(_lib.sgdb_step(_dev(grad, None, "grad"), _grad_dtype(grad), P, ld,
                          _dev(arrival, torch.float32, "arrival"), _dev(tags, torch.int32, "tags"), t, N, b,
                          _dev(theta, torch.float32, "theta"), _dev(state0, torch.float32, "state0"),
                          _dev(state1, torch.float32, "state1"), ctypes.byref(c),
                          _dev(mask, torch.uint8, "mask"), _dev(order, torch.int32, "order"),
                          _dev(info, torch.int32, "info"), _stream(stream)), "sgdb_step")


def sgdb_select_deadline(arrival, tags, t: int, deadline: float, n_min: int, mask, order, info, stream=None) -> None:
    """Time-out rule: keep every gradient tagged t with arrival <= deadline.  order has W entries; info = {n, status}."""
    W = arrival.numel()
    _check(_lib.sgdb_select_deadline(_dev(arrival, torch.float32, "arrival"), _dev(tags, torch.int32, "tags"), t, W,
                                     deadline, n_min, _dev(mask, torch.uint8, "mask"),
                                     _dev(order, torch.int32, "order"), _dev(info, torch.int32, "info"),
                                     _stream(stream)), "sgdb_select_deadline")


def sgdb_step_deadline(grad, P: int, arrival, tags, t: int, deadline: float, n_min: int, theta, state0, state1,
                       opt: Opt, mask, order, info, ld: int | None = None, stream=None) -> None:
    """One fused iteration with the time-out rule: mean over the n gradients kept, then the optimizer rule."""
    ld = grad.stride(0) if ld is None else ld
    W = arrival.numel()
    c = opt._c()
    _check(_lib.sgdb_step_deadline(_dev(grad, None, "grad"), _grad_dtype(grad), P, ld,
                                   _dev(arrival, torch.float32, "arrival"), _dev(tags, torch.int32, "tags"), t, W,
                                   deadline, n_min, _dev(theta, torch.float32, "theta"),
                                   _dev(state0, torch.float32, "state0"), _dev(state1, torch.float32, "state1"),
                                   ctypes.byref(c), _dev(mask, torch.uint8, "mask"), _dev(order, torch.int32, "order"),
                                   _dev(info, torch.int32, "info"), _stream(stream)), "sgdb_step_deadline")


def sgdb_step_ema(grad, P: int, arrival, tags, t: int, N: int, b: int, theta, state0, state1, opt: Opt, ema,
                  alpha: float, mask, order, info, ld: int | None = None, stream=None) -> None:
    """sgdb_step plus avg <- alpha * avg + (1 - alpha) * theta(before the update), in the same launch."""
    ld = grad.stride(0) if ld is None else ld
    c = opt._c()
    _check(_lib.sgdb_step_ema(_dev(grad, None, "grad"), _grad_dtype(grad), P, ld,
                              _dev(arrival, torch.float32, "arrival"), _dev(tags, torch.int32, "tags"), t, N, b,
                              _dev(theta, torch.float32, "theta"), _dev(state0, torch.float32, "state0"),
                              _dev(state1, torch.float32, "state1"), ctypes.byref(c),
                              _dev(ema, torch.float32, "ema"), alpha, _dev(mask, torch.uint8, "mask"),
                              _dev(order, torch.int32, "order"), _dev(info, torch.int32, "info"), _stream(stream)),
           "sgdb_step_ema")


def sgdb_ema(ema, theta, alpha: float, info=None, P: int | None = None, stream=None) -> None:
    """avg <- alpha * avg + (1 - alpha) * theta on its own."""
    P = theta.numel() if P is None else P
    _check(_lib.sgdb_ema(_dev(ema, torch.float32, "ema"), _dev(theta, torch.float32, "theta"), P, alpha,
                         _dev(info, torch.int32, "info"), _stream(stream)), "sgdb_ema")


def sgdb_learning_rate(gamma0: float, beta: float, t: int, N: int, T: float) -> float:
    """gamma0 * beta^(t N / (2 T)): the paper's schedule (host computation)."""
    return float(_lib.sgdb_learning_rate(gamma0, beta, t, N, T))


def make_segment_table(segments, device) -> torch.Tensor:
    """Device table for sgdb_step_segmented from (theta, state0, state1, grad) tensor tuples.

    grad is [W, ld] with ld = grad.stride(0); len = theta.numel().  Returns a uint8 CUDA tensor
    holding the packed sgdb_segment_t array; the caller keeps the listed tensors alive.
    """
    arr = (CSegment * len(segments))()
    for i, (theta, s0, s1, grad) in enumerate(segments):
        arr[i] = CSegment(_dev(theta, torch.float32, "theta"), _dev(s0, torch.float32, "state0"),
                          _dev(s1, torch.float32, "state1"), grad.data_ptr(), grad.stride(0), theta.numel())
    raw = bytes(arr)
    host = torch.frombuffer(bytearray(raw), dtype=torch.uint8) if raw else torch.empty(0, dtype=torch.uint8)
    return host.to(device)


def sgdb_step_segmented(table, S: int, grad_dtype, arrival, tags, t: int, N: int, b: int, opt: Opt,
                        mask, order, info, stream=None) -> None:
    dt = SGDB_BF16 if grad_dtype == torch.bfloat16 else SGDB_F32
    c = opt._c()
    _check(_lib.sgdb_step_segmented(_dev(table, torch.uint8, "segment table"), S, dt,
                                    _dev(arrival, torch.float32, "arrival"), _dev(tags, torch.int32, "tags"),
                                    t, N, b, ctypes.byref(c), _dev(mask, torch.uint8, "mask"),
                                    _dev(order, torch.int32, "order"), _dev(info, torch.int32, "info"),
                                    _stream(stream)), "sgdb_step_segmented")


def make_pointer_table(tensors, device) -> torch.Tensor:
    """Device array of device pointers (int64 CUDA tensor) from a list of CUDA tensors; None -> NULL.
    The caller keeps the listed tensors alive."""
    return torch.tensor([0 if x is None else _dev(x, torch.float32, "tensor") for x in tensors], dtype=torch.int64).to(device)


def sgdb_step_segmented_ema(table, ema_table, alpha: float, S: int, grad_dtype, arrival, tags, t: int, N: int, b: int,
                            opt: Opt, mask, order, info, stream=None) -> None:
    """sgdb_step_segmented plus the per-tensor parameter averages (ema_table from make_pointer_table)."""
    dt = SGDB_BF16 if grad_dtype == torch.bfloat16 else SGDB_F32
    c = opt._c()
    _check(_lib.sgdb_step_segmented_ema(_dev(table, torch.uint8, "segment table"), _dev(ema_table, torch.int64, "ema table"),
                                        alpha, S, dt, _dev(arrival, torch.float32, "arrival"),
                                        _dev(tags, torch.int32, "tags"), t, N, b, ctypes.byref(c),
                                        _dev(mask, torch.uint8, "mask"), _dev(order, torch.int32, "order"),
                                        _dev(info, torch.int32, "info"), _stream(stream)), "sgdb_step_segmented_ema")


def sgdb_step_segmented_deadline(table, S: int, grad_dtype, arrival, tags, t: int, deadline: float, n_min: int, opt: Opt,
                                 mask, order, info, stream=None) -> None:
    """sgdb_step_segmented with the time-out rule; order has W entries, info = {n, status}."""
    dt = SGDB_BF16 if grad_dtype == torch.bfloat16 else SGDB_F32
    W = arrival.numel()
    c = opt._c()
    _check(_lib.sgdb_step_segmented_deadline(_dev(table, torch.uint8, "segment table"), S, dt,
                                             _dev(arrival, torch.float32, "arrival"), _dev(tags, torch.int32, "tags"),
                                             t, W, deadline, n_min, ctypes.byref(c), _dev(mask, torch.uint8, "mask"),
                                             _dev(order, torch.int32, "order"), _dev(info, torch.int32, "info"),
                                             _stream(stream)), "sgdb_step_segmented_deadline")


def sgdb_accumulate_arrival_deadline(row, row_tag: int, row_arrival: float, t: int, deadline: float, acc, counter, info,
                                     P: int | None = None, stream=None) -> None:
    """Time-out rule, one arriving gradient: joins the running sum iff tagged t, t open and arrived by the deadline."""
    P = acc.numel() if P is None else P
    _check(_lib.sgdb_accumulate_arrival_deadline(_dev(row, None, "row"), _grad_dtype(row), row_tag, row_arrival, t,
                                                 deadline, P, _dev(acc, torch.float32, "acc"),
                                                 _dev(counter, torch.int32, "counter"), _dev(info, torch.int32, "info"),
                                                 _stream(stream)), "sgdb_accumulate_arrival_deadline")


def sgdb_accumulate_close(t: int, n_min: int, acc, counter, theta, state0, state1, opt: Opt, info, ema=None,
                          alpha: float = 0.0, P: int | None = None, stream=None) -> None:
    """The deadline of iteration t has passed: update from the mean of the set if it holds at least n_min gradients."""
    P = theta.numel() if P is None else P
    c = opt._c()
    _check(_lib.sgdb_accumulate_close(t, n_min, P, _dev(acc, torch.float32, "acc"), _dev(counter, torch.int32, "counter"),
                                      _dev(theta, torch.float32, "theta"), _dev(state0, torch.float32, "state0"),
                                      _dev(state1, torch.float32, "state1"), ctypes.byref(c),
                                      _dev(ema, torch.float32, "ema"), alpha, _dev(info, torch.int32, "info"),
                                      _stream(stream)), "sgdb_accumulate_close")


def sgdb_select_grouped(arrival, tags, group, t: int, M: int, N: int, mask, group_order, order, info, stream=None) -> None:
    """Two-level selection: the first N machine messages.  mask u8[W], group_order i32[N], order i32[W], info i32[3]."""
    W = arrival.numel()
    _check(_lib.sgdb_select_grouped(_dev(arrival, torch.float32, "arrival"), _dev(tags, torch.int32, "tags"),
                                    _dev(group, torch.int32, "group"), t, W, M, N, _dev(mask, torch.uint8, "mask"),
                                    _dev(group_order, torch.int32, "group_order"), _dev(order, torch.int32, "order"),
                                    _dev(info, torch.int32, "info"), _stream(stream)), "sgdb_select_grouped")


def sgdb_step_grouped(grad, P: int, arrival, tags, group, t: int, M: int, N: int, theta, state0, state1, opt: Opt,
                      mask, group_order, order, info, ld: int | None = None, stream=None) -> None:
    """One fused iteration over machine messages: machines send the mean of their workers' rows, the first N
    messages are averaged, then the optimizer rule."""
    ld = grad.stride(0) if ld is None else ld
    W = arrival.numel()
    c = opt._c()
    _check(_lib.sgdb_step_grouped(_dev(grad, None, "grad"), _grad_dtype(grad), P, ld,
                                  _dev(arrival, torch.float32, "arrival"), _dev(tags, torch.int32, "tags"),
                                  _dev(group, torch.int32, "group"), t, W, M, N, _dev(theta, torch.float32, "theta"),
                                  _dev(state0, torch.float32, "state0"), _dev(state1, torch.float32, "state1"),
                                  ctypes.byref(c), _dev(mask, torch.uint8, "mask"),
                                  _dev(group_order, torch.int32, "group_order"), _dev(order, torch.int32, "order"),
                                  _dev(info, torch.int32, "info"), _stream(stream)), "sgdb_step_grouped")


def make_address_table(addresses, device) -> torch.Tensor:
    """Device array of device addresses (int64 CUDA tensor) from integers, e.g. tensor.data_ptr() plus a byte
    offset, or the address of a peer GPU's buffer mapped into this process.  The caller keeps the memory alive."""
    return torch.tensor([int(a) for a in addresses], dtype=torch.int64).to(device)


def sgdb_step_rows(rows, grad_dtype, length: int, arrival, tags, t: int, N: int, b: int, theta, state0, state1, opt: Opt,
                   replicas, mask, order, info, stream=None) -> None:
    """The fused step of one parameter server over its range of `length` columns: rows i64[W] holds the address of
    each worker's gradient at the range's first column (make_address_table), replicas i64[R] or None the addresses
    the new parameters are also stored to."""
    dt = SGDB_BF16 if grad_dtype == torch.bfloat16 else SGDB_F32
    R = 0 if replicas is None else replicas.numel()
    c = opt._c()
    _check(_lib.sgdb_step_rows(_dev(rows, torch.int64, "rows"), dt, length, _dev(arrival, torch.float32, "arrival"),
                               _dev(tags, torch.int32, "tags"), t, N, b, _dev(theta, torch.float32, "theta"),
                               _dev(state0, torch.float32, "state0"), _dev(state1, torch.float32, "state1"),
                               ctypes.byref(c), _dev(replicas, torch.int64, "replicas"), R,
                               _dev(mask, torch.uint8, "mask"), _dev(order, torch.int32, "order"),
                               _dev(info, torch.int32, "info"), _stream(stream)), "sgdb_step_rows")


def sgdb_step_rows_ordered(rows, grad_dtype, length: int, N: int, order, info, theta, state0, state1, opt: Opt,
                           replicas, stream=None) -> None:
    """sgdb_step_rows with the selection given: order i32[N] row ids in summation sequence, info i32[2] in/out."""
    dt = SGDB_BF16 if grad_dtype == torch.bfloat16 else SGDB_F32
    R = 0 if replicas is None else replicas.numel()
    c = opt._c()
    _check(_lib.sgdb_step_rows_ordered(_dev(rows, torch.int64, "rows"), rows.numel(), dt, length, N,
                                       _dev(order, torch.int32, "order"), _dev(info, torch.int32, "info"),
                                       _dev(theta, torch.float32, "theta"), _dev(state0, torch.float32, "state0"),
                                       _dev(state1, torch.float32, "state1"), ctypes.byref(c),
                                       _dev(replicas, torch.int64, "replicas"), R, _stream(stream)),
           "sgdb_step_rows_ordered")


def sgdb_shard_range(P: int, n_servers: int, j: int):
    """(first column, number of columns) of parameter server j out of n_servers over P columns (host computation)."""
    first, length = ctypes.c_int64(0), ctypes.c_int64(0)
    _check(_lib.sgdb_shard_range(P, n_servers, j, ctypes.byref(first), ctypes.byref(length)), "sgdb_shard_range")
    return int(first.value), int(length.value)


def sgdb_enable_peer_access(peer_device: int) -> None:
    """Kernels launched on the current device may then use the memory of peer_device (one-time set-up)."""
    _check(_lib.sgdb_enable_peer_access(int(peer_device)), "sgdb_enable_peer_access")


def sgdb_accumulate_arrival(row, row_tag: int, t: int, N: int, acc, counter, theta, state0, state1,
                            opt: Opt, info, P: int | None = None, stream=None) -> None:
    """One arriving gradient row (f32 or bf16 [P]); counter i32[4] is the server state, info i32[2] the outcome."""
    P = theta.numel() if P is None else P
    c = opt._c()
    _check(_lib.sgdb_accumulate_arrival(_dev(row, None, "row"), _grad_dtype(row), row_tag, t, N, P,
                                        _dev(acc, torch.float32, "acc"), _dev(counter, torch.int32, "counter"),
                                        _dev(theta, torch.float32, "theta"), _dev(state0, torch.float32, "state0"),
                                        _dev(state1, torch.float32, "state1"), ctypes.byref(c),
                                        _dev(info, torch.int32, "info"), _stream(stream)),
           "sgdb_accumulate_arrival")


def sgdb_accumulate_arrival_ema(row, row_tag: int, t: int, N: int, acc, counter, theta, state0, state1, opt: Opt, ema,
                                alpha: float, info, P: int | None = None, stream=None) -> None:
    """sgdb_accumulate_arrival that also moves the parameter average when the N-th gradient fires the update."""
    P = theta.numel() if P is None else P
    c = opt._c()
    _check(_lib.sgdb_accumulate_arrival_ema(_dev(row, None, "row"), _grad_dtype(row), row_tag, t, N, P,
                                            _dev(acc, torch.float32, "acc"), _dev(counter, torch.int32, "counter"),
                                            _dev(theta, torch.float32, "theta"), _dev(state0, torch.float32, "state0"),
                                            _dev(state1, torch.float32, "state1"), ctypes.byref(c),
                                            _dev(ema, torch.float32, "ema"), alpha, _dev(info, torch.int32, "info"),
                                            _stream(stream)), "sgdb_accumulate_arrival_ema")


def sgdb_step_host_workspace_bytes(grad_dtype, P: int, ld: int, N: int, b: int) -> int:
    dt = SGDB_BF16 if grad_dtype == torch.bfloat16 else SGDB_F32
    return int(_lib.sgdb_step_host_workspace_bytes(dt, P, ld, N, b))


def sgdb_step_host(h_grad, P: int, h_arrival, h_tags, t: int, N: int, b: int, theta, state0, state1, opt: Opt,
                   h_theta_out, h_mask, h_order, h_info, workspace, ld: int | None = None, stream=None) -> int:
    """sgdb_step with gradients, arrival times and tags in host memory; returns the status (0 or INSUFFICIENT)."""
    ld = h_grad.stride(0) if ld is None else ld
    c = opt._c()
    st = _lib.sgdb_step_host(_host(h_grad, None, "h_grad"), _grad_dtype(h_grad), P, ld,
                             _host(h_arrival, torch.float32, "h_arrival"), _host(h_tags, torch.int32, "h_tags"),
                             t, N, b, _dev(theta, torch.float32, "theta"), _dev(state0, torch.float32, "state0"),
                             _dev(state1, torch.float32, "state1"), ctypes.byref(c),
                             _host(h_theta_out, torch.float32, "h_theta_out"), _host(h_mask, torch.uint8, "h_mask"),
                             _host(h_order, torch.int32, "h_order"), _host(h_info, torch.int32, "h_info"),
                             _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream))
    if st not in (SGDB_OK, SGDB_ERR_INSUFFICIENT):
        raise SgdbError(st, "sgdb_step_host")
    return st


def sgdb_step_host_static(h_grad, P: int, h_arrival, h_tags, t: int, N: int, b: int, theta, state0, state1, opt: Opt,
                          h_theta_out, h_mask, h_order, h_info, ld: int | None = None, stream=None) -> int:
    """sgdb_step_host without a workspace argument, for callers that can neither supply device memory nor
    allocate any: the staging area is a fixed SGDB_STATIC_SCRATCH_BYTES array inside the library.  Sizes that
    do not fit raise SgdbError (SGDB_ERR_UNSUPPORTED).  Calls on one device share that array: do not overlap
    them.  Returns the status (0 or SGDB_ERR_INSUFFICIENT)."""
    ld = h_grad.stride(0) if ld is None else ld
    c = opt._c()
    st = _lib.sgdb_step_host_static(_host(h_grad, None, "h_grad"), _grad_dtype(h_grad), P, ld,
                                    _host(h_arrival, torch.float32, "h_arrival"), _host(h_tags, torch.int32, "h_tags"),
                                    t, N, b, _dev(theta, torch.float32, "theta"), _dev(state0, torch.float32, "state0"),
                                    _dev(state1, torch.float32, "state1"), ctypes.byref(c),
                                    _host(h_theta_out, torch.float32, "h_theta_out"),
                                    _host(h_mask, torch.uint8, "h_mask"), _host(h_order, torch.int32, "h_order"),
                                    _host(h_info, torch.int32, "h_info"), _stream(stream))
    if st not in (SGDB_OK, SGDB_ERR_INSUFFICIENT):
        raise SgdbError(st, "sgdb_step_host_static")
    return st


# ------------------------------------------------------------------ operators for language models


_DTYPES = {torch.float32: SGDB_F32, torch.bfloat16: SGDB_BF16}


def _code(dtype, name) -> int:
    code = _DTYPES.get(dtype)
    if code is None:
        raise ValueError("%s must be float32 or bfloat16, got %s" % (name, dtype))
    return code


def _here(x) -> int:
    """The current device, on which all tensors of a call have to be; no device's number when x is not on a GPU."""
    return _current_device() if x.is_cuda else -2


def _mat(x, name, rows: int, cols: int, dtype, here: int) -> tuple:
    """(device pointer, elements between rows) of a 2-D tensor on the current GPU whose rows are contiguous."""
    if x.shape != (rows, cols):
        raise ValueError("%s must have shape %s, got %s" % (name, (rows, cols), tuple(x.shape)))
    if x.dtype is not dtype:
        raise ValueError("%s must have dtype %s, got %s" % (name, dtype, x.dtype))
    ld, inner = x.stride()
    if rows <= 1:
        ld = cols if cols > 1 else 1
    if x.get_device() != here or (inner != 1 and cols > 1) or ld < cols:
        raise ValueError("%s must be a 2-D CUDA tensor on the current device with contiguous rows" % name)
    return x.data_ptr(), ld


def _vec(x, n: int, name, dtype, here: int | None = None) -> int:
    """Device pointer of a contiguous tensor of n elements on the current GPU (None -> NULL)."""
    if x is None:
        return 0
    if x.dtype is not dtype or x.get_device() != (_here(x) if here is None else here) or x.numel() != n or not x.is_contiguous():
        raise ValueError("%s must be a contiguous CUDA tensor on the current device of %d elements of dtype %s, got %s of dtype %s on %s"
                         % (name, n, dtype, tuple(x.shape), x.dtype, x.device))
    return x.data_ptr()


def _whole(x, name, here: int, dtype=None) -> int:
    """Device pointer of a contiguous tensor of any size on the current GPU (None -> NULL)."""
    return 0 if x is None else _vec(x, x.numel(), name, x.dtype if dtype is None else dtype, here)


def _shared_dtype(a, b):
    """The dtype that two optional tensors have to share (float32 when neither is given)."""
    return a.dtype if a is not None else b.dtype if b is not None else torch.float32


def sgdb_layer_norm(x, gamma, beta, eps: float, y, mean=None, rstd=None, stream=None) -> None:
    """x [tokens, width] -> y, with gamma, beta [width] (None: ones, zeros); mean, rstd f32[tokens] for the backward pass."""
    T, D = x.shape
    dtype, here = x.dtype, _here(x)
    px, ldx = _mat(x, "x", T, D, dtype, here)
    py, ldy = _mat(y, "y", T, D, dtype, here)
    dt_w = _shared_dtype(gamma, beta)
    status = _lib.sgdb_layer_norm(px, _code(dtype, "x"), T, D, ldx, _vec(gamma, D, "gamma", dt_w, here), _vec(beta, D, "beta", dt_w, here),
                                  _code(dt_w, "gamma and beta"), eps, py, ldy, _vec(mean, T, "mean", torch.float32, here),
                                  _vec(rstd, T, "rstd", torch.float32, here), _stream(stream))
    if status:
        _check(status, "sgdb_layer_norm")


def sgdb_layer_norm_backward_workspace_bytes(tokens: int, width: int) -> int:
    return int(_lib.sgdb_layer_norm_backward_workspace_bytes(tokens, width))


def sgdb_layer_norm_backward(dy, x, gamma, mean, rstd, dx, dgamma=None, dbeta=None, workspace=None, stream=None) -> None:
    """dy, x [tokens, width], mean, rstd of the forward pass -> dx, and dgamma, dbeta [width] (f32 or bf16; None: not wanted)."""
    T, D = x.shape
    dtype, here = x.dtype, _here(x)
    px, ldx = _mat(x, "x", T, D, dtype, here)
    pdy, lddy = _mat(dy, "dy", T, D, dtype, here)
    pdx, lddx = _mat(dx, "dx", T, D, dtype, here)
    dt_w, dt_g = _shared_dtype(gamma, None), _shared_dtype(dgamma, dbeta)
    _check(_lib.sgdb_layer_norm_backward(
        pdy, lddy, px, ldx, _code(dtype, "x"), T, D, _vec(gamma, D, "gamma", dt_w, here), _code(dt_w, "gamma"),
        _vec(mean, T, "mean", torch.float32, here), _vec(rstd, T, "rstd", torch.float32, here), pdx, lddx, _vec(dgamma, D, "dgamma", dt_g, here),
        _vec(dbeta, D, "dbeta", dt_g, here), _code(dt_g, "dgamma and dbeta"), _whole(workspace, "workspace", here),
        0 if workspace is None else workspace.numel() * workspace.element_size(), _stream(stream)), "sgdb_layer_norm_backward")


def sgdb_route(expert, E: int, offsets, slot, source, stream=None) -> None:
    """expert i32[tokens, k] -> offsets i32[E + 1], slot i32[tokens, k] (-1: dropped), source i32[tokens * k] (-1: not in use)."""
    (T, k), here = expert.shape, _here(expert)
    _check(_lib.sgdb_route(_vec(expert, T * k, "expert", torch.int32, here), T, k, E, _vec(offsets, E + 1, "offsets", torch.int32, here),
                           _vec(slot, T * k, "slot", torch.int32, here), _vec(source, T * k, "source", torch.int32, here),
                           _stream(stream)), "sgdb_route")


def sgdb_dispatch(x, slot, offsets, xs, stream=None) -> None:
    """x [tokens, width], slot i32[tokens, k], offsets i32[E + 1] -> xs [tokens * k, width], tokens in their experts' rows."""
    (T, k), D, here = slot.shape, x.size(1), _here(x)
    px, ldx = _mat(x, "x", T, D, x.dtype, here)
    pxs, ldxs = _mat(xs, "xs", T * k, D, x.dtype, here)
    _check(_lib.sgdb_dispatch(px, _code(x.dtype, "x"), T, D, ldx, _vec(slot, T * k, "slot", torch.int32, here), k,
                              _whole(offsets, "offsets", here, torch.int32), offsets.numel() - 1, pxs, ldxs, _stream(stream)), "sgdb_dispatch")


def sgdb_combine(ys, slot, weights, out, stream=None) -> None:
    """ys [tokens * k, width], slot i32[tokens, k], weights f32[tokens, k] or None -> out [tokens, width]."""
    (T, k), D, here = slot.shape, ys.size(1), _here(ys)
    pys, ldys = _mat(ys, "ys", T * k, D, ys.dtype, here)
    po, ldo = _mat(out, "out", T, D, ys.dtype, here)
    _check(_lib.sgdb_combine(pys, _code(ys.dtype, "ys"), T, D, ldys, _vec(slot, T * k, "slot", torch.int32, here), k,
                             _vec(weights, T * k, "weights", torch.float32, here), po, ldo, _stream(stream)), "sgdb_combine")


def sgdb_combine_backward(dout, ys, slot, weights, offsets, dys, dweights=None, stream=None) -> None:
    """dout [tokens, width], ys [tokens * k, width] -> dys like ys, dweights f32[tokens, k] (None: not wanted)."""
    (T, k), D, here = slot.shape, ys.size(1), _here(ys)
    pys, ldys = _mat(ys, "ys", T * k, D, ys.dtype, here)
    pdo, lddo = _mat(dout, "dout", T, D, ys.dtype, here)
    pdys, lddys = _mat(dys, "dys", T * k, D, ys.dtype, here)
    _check(_lib.sgdb_combine_backward(pdo, lddo, pys, ldys, _code(ys.dtype, "ys"), T, D, _vec(slot, T * k, "slot", torch.int32, here), k,
                                      _vec(weights, T * k, "weights", torch.float32, here), _whole(offsets, "offsets", here, torch.int32),
                                      offsets.numel() - 1, pdys, lddys, _vec(dweights, T * k, "dweights", torch.float32, here),
                                      _stream(stream)), "sgdb_combine_backward")


_FORMATS = {torch.float8_e4m3fn: SGDB_E4M3, torch.float8_e5m2: SGDB_E5M2}
_SCALE = torch.float8_e8m0fnu


def _format(x, name) -> int:
    code = _FORMATS.get(x.dtype)
    if code is None:
        raise ValueError("%s must be float8_e4m3fn or float8_e5m2, got %s" % (name, x.dtype))
    return code


def _blocks(n: int) -> int:
    return (n + 127) // 128


def empty_f8(*shape, dtype=torch.float8_e4m3fn, device=None):
    """A new array of 8-bit elements whose rows begin on 16-byte boundaries, as the experts' products take them."""
    if not shape or dtype not in _FORMATS:
        raise ValueError("empty_f8 takes a shape and float8_e4m3fn or float8_e5m2, got %s and %s" % (shape, dtype))
    return torch.empty(*shape[:-1], (shape[-1] + 15) // 16 * 16, dtype=dtype, device=device)[..., :shape[-1]]


def empty_scale(*shape, device=None):
    """A new array of the scales of 8-bit values of this shape, whose rows begin on 16-byte boundaries: the experts' products read those fastest."""
    n = _blocks(shape[-1])
    return torch.empty(*shape[:-1], (n + 15) // 16 * 16, dtype=_SCALE, device=device)[..., :n]


def sgdb_quantize(x, q, scale, stream=None) -> None:
    """x [rows, width] -> q of the same shape in 8 bits (float8_e4m3fn or float8_e5m2), scale float8_e8m0fnu [rows, ceil(width / 128)]."""
    (R, D), here = x.shape, _here(x)
    px, ldx = _mat(x, "x", R, D, x.dtype, here)
    fmt = _format(q, "q")
    pq, ldq = _mat(q, "q", R, D, q.dtype, here)
    ps, lds = _mat(scale, "scale", R, _blocks(D), _SCALE, here)
    _check(_lib.sgdb_quantize(px, _code(x.dtype, "x"), R, D, ldx, pq, fmt, ldq, ps, lds, _stream(stream)), "sgdb_quantize")


def sgdb_quantize_matrices(w, q, qt, scale, stream=None) -> None:
    """w [batch, rows, cols] -> q of the same shape, qt [batch, cols, rows] in 8 bits (either may be None), scale float8_e8m0fnu
    [batch, ceil(rows / 128), ceil(cols / 128)] of both."""
    here = _here(w)
    if w.dim() != 3:
        raise ValueError("w must be a 3-D CUDA tensor, got %s" % (tuple(w.shape),))
    pw, B, R, C, ldw, sw = _matrices(w, "w", here)
    out = []
    for x, name, shape in ((q, "q", (B, R, C)), (qt, "qt", (B, C, R))):
        if x is None:
            out.append((0, max(R, C), 0))
            continue
        if tuple(x.shape) != shape:
            raise ValueError("%s must have shape %s, got %s" % (name, shape, tuple(x.shape)))
        p, _, _, _, ld, between = _matrices(x, name, here)
        out.append((p, ld, between))
    given = q if q is not None else qt
    if given is None or (q is not None and qt is not None and q.dtype is not qt.dtype):
        raise ValueError("q or qt is needed, and both in the same format")
    (pq, ldq, sq), (pqt, ldqt, sqt) = out
    _check(_lib.sgdb_quantize_matrices(pw, _code(w.dtype, "w"), B, R, C, ldw, sw, _format(given, "q and qt"), pq, ldq, sq, pqt, ldqt, sqt,
                                       _vec(scale, B * _blocks(R) * _blocks(C), "scale", _SCALE, here), _stream(stream)), "sgdb_quantize_matrices")


def _halves(x, name, R: int, n: int, dtype, here: int) -> tuple:
    """(pointer, elements between rows) of a gate's checkpoint [rows, 2, width] or of its scales, as 2 rows rows."""
    if x.shape != (R, 2, n) or x.dtype is not dtype:
        raise ValueError("%s must have shape %s and dtype %s, got %s of %s" % (name, (R, 2, n), dtype, tuple(x.shape), x.dtype))
    between, ld, inner = x.stride()
    if x.get_device() != here or (inner != 1 and n > 1) or ld < n or (between != 2 * ld and R > 1):
        raise ValueError("%s must be a CUDA tensor on the current device with contiguous, evenly spaced rows" % name)
    return x.data_ptr(), ld


def sgdb_gate(h, a, a_scale, h8, h_scale, stream=None) -> None:
    """h [rows, 2 width] = [g | u] -> silu(g) u in 8 bits: a [rows, width], a_scale [rows, blocks of width]; and h in 8 bits for the
    backward pass: h8 [rows, 2, width], h_scale [rows, 2, blocks of width]."""
    (R, F), here = a.shape, _here(h)
    ph, ldh = _mat(h, "h", R, 2 * F, h.dtype, here)
    fmt = _format(a, "a")
    pa, lda = _mat(a, "a", R, F, a.dtype, here)
    pas, ldas = _mat(a_scale, "a_scale", R, _blocks(F), _SCALE, here)
    p8, ld8 = _halves(h8, "h8", R, F, a.dtype, here)
    ps, lds = _halves(h_scale, "h_scale", R, _blocks(F), _SCALE, here)
    _check(_lib.sgdb_gate(ph, _code(h.dtype, "h"), R, F, ldh, fmt, pa, lda, pas, ldas, p8, ld8, ps, lds, _stream(stream)), "sgdb_gate")


def sgdb_gate_backward(da, h8, h_scale, dh, stream=None) -> None:
    """da [rows, width] and the checkpoint of sgdb_gate -> dh [rows, 2 width] = [dg | du]."""
    (R, F), here = da.shape, _here(da)
    pda, ldda = _mat(da, "da", R, F, da.dtype, here)
    pdh, lddh = _mat(dh, "dh", R, 2 * F, da.dtype, here)
    fmt = _format(h8, "h8")
    p8, ld8 = _halves(h8, "h8", R, F, h8.dtype, here)
    ps, lds = _halves(h_scale, "h_scale", R, _blocks(F), _SCALE, here)
    _check(_lib.sgdb_gate_backward(pda, ldda, _code(da.dtype, "da"), R, F, fmt, p8, ld8, ps, lds, pdh, lddh, _stream(stream)), "sgdb_gate_backward")


def sgdb_experts_product(x, x_scale, w, w_scale, offsets, y, info=None, stream=None) -> None:
    """x [rows, depth] in 8 bits with x_scale [rows, blocks of depth], w [E, width, depth] in 8 bits with w_scale [E, blocks of width, blocks
    of depth] (any strides: for the qt of sgdb_quantize_matrices, its scale transposed), offsets i32[E + 1] or None (E = 1: all rows)
    -> y [rows, width] (f32 or bf16)."""
    (S, K), here, kinds = x.shape, _here(x), (x.dtype, w.dtype, y.dtype)
    px, ldx = _mat(x, "x", S, K, kinds[0], here)
    KB = (K + 127) // 128
    pxs, ldxs = _mat(x_scale, "x_scale", S, KB, _SCALE, here)
    if w.dim() != 3 or w.size(2) != K:
        raise ValueError("w must have shape (experts, width, %d), got %s" % (K, tuple(w.shape)))
    pw, E, N, _, ldw, sw = _matrices(w, "w", here)
    if S <= 1:
        ldx = (ldx + 15) // 16 * 16  # of no row
    if N <= 1:
        ldw = (ldw + 15) // 16 * 16
    if w_scale.shape != (E, (N + 127) // 128, KB) or w_scale.dtype is not _SCALE or w_scale.get_device() != here:
        raise ValueError("w_scale must be a CUDA tensor on the current device of shape %s and dtype %s, got %s of %s"
                         % ((E, _blocks(N), KB), _SCALE, tuple(w_scale.shape), w_scale.dtype))
    py, ldy = _mat(y, "y", S, N, kinds[2], here)
    fx, fw = _FORMATS.get(kinds[0]), _FORMATS.get(kinds[1])
    if fx is None or fw is None:
        _format(x, "x"), _format(w, "w")
    status = _lib.sgdb_experts_product(px, fx, S, K, ldx, pxs, ldxs, pw, fw, E, N, ldw, sw, w_scale.data_ptr(), *w_scale.stride(),
                                       0 if offsets is None else _vec(offsets, E + 1, "offsets", torch.int32, here), py, _code(kinds[2], "y"), ldy,
                                       0 if info is None else _vec(info, 2, "info", torch.int32, here), _stream(stream))
    if status:
        _check(status, "sgdb_experts_product")


def sgdb_experts_gradient_workspace_bytes(rows: int, width: int, depth: int, E: int) -> int:
    return int(_lib.sgdb_experts_gradient_workspace_bytes(rows, width, depth, E))


def sgdb_experts_gradient(dy, x, x_scale, offsets, dw, workspace=None, info=None, stream=None) -> None:
    """dy [rows, width], x [rows, depth] in 8 bits with x_scale [rows, blocks of depth] -> dw [E, width, depth] (f32 or bf16): the sums of
    dy x over each expert's rows."""
    (S, N), K, here = dy.shape, x.size(1), _here(dy)
    pdy, lddy = _mat(dy, "dy", S, N, dy.dtype, here)
    fmt = _format(x, "x")
    px, ldx = _mat(x, "x", S, K, x.dtype, here)
    pxs, ldxs = _mat(x_scale, "x_scale", S, _blocks(K), _SCALE, here)
    if dw.dim() != 3 or tuple(dw.shape[1:]) != (N, K):
        raise ValueError("dw must have shape (experts, %d, %d), got %s" % (N, K, tuple(dw.shape)))
    pdw, E, _, _, lddw, sdw = _matrices(dw, "dw", here)
    _check(_lib.sgdb_experts_gradient(pdy, _code(dy.dtype, "dy"), S, N, lddy, px, fmt, K, ldx, pxs, ldxs,
                                      _vec(offsets, E + 1, "offsets", torch.int32, here), E, pdw, _code(dw.dtype, "dw"), lddw, sdw,
                                      _whole(workspace, "workspace", here), 0 if workspace is None else workspace.numel() * workspace.element_size(),
                                      _vec(info, 2, "info", torch.int32, here), _stream(stream)), "sgdb_experts_gradient")


def sgdb_balance_loss_workspace_bytes(tokens: int, E: int) -> int:
    return int(_lib.sgdb_balance_loss_workspace_bytes(tokens, E))


def sgdb_balance_loss(logits, expert, mask, loss, counts, slope, workspace, stream=None) -> None:
    """logits [tokens, E], expert i32[tokens, k], mask u8[tokens] or None -> loss f32[1], counts i32[E], slope f32[E] for the backward pass."""
    (T, E), here = logits.shape, _here(logits)
    pl, ld = _mat(logits, "logits", T, E, logits.dtype, here)
    if expert.dim() != 2:
        raise ValueError("expert must have shape (tokens, choices), got %s" % (tuple(expert.shape),))
    k = expert.size(1)
    status = _lib.sgdb_balance_loss(pl, _code(logits.dtype, "logits"), T, E, ld, _vec(expert, T * k, "expert", torch.int32, here), k,
                                    _vec(mask, T, "mask", torch.uint8, here), _vec(loss, 1, "loss", torch.float32, here),
                                    _vec(counts, E, "counts", torch.int32, here), _vec(slope, E, "slope", torch.float32, here),
                                    _whole(workspace, "workspace", here), workspace.numel() * workspace.element_size(), _stream(stream))
    if status:
        _check(status, "sgdb_balance_loss")


def sgdb_balance_loss_backward(grad, logits, mask, slope, dlogits, stream=None) -> None:
    """grad f32[1], the loss's gradient, and the forward pass's logits, mask and slope -> dlogits like logits."""
    (T, E), here = logits.shape, _here(logits)
    pl, ld = _mat(logits, "logits", T, E, logits.dtype, here)
    pd, ldd = _mat(dlogits, "dlogits", T, E, logits.dtype, here)
    status = _lib.sgdb_balance_loss_backward(_vec(grad, 1, "grad", torch.float32, here), pl, _code(logits.dtype, "logits"), T, E, ld,
                                             _vec(mask, T, "mask", torch.uint8, here), _vec(slope, E, "slope", torch.float32, here), pd, ldd,
                                             _stream(stream))
    if status:
        _check(status, "sgdb_balance_loss_backward")


def _matrices(x, name, here: int) -> tuple:
    """(device pointer, matrices, rows, columns, elements between rows, between matrices) of a 2-D or 3-D tensor on the current GPU."""
    if x.get_device() != here or x.dim() not in (2, 3):
        raise ValueError("%s must be a 2-D or 3-D CUDA tensor on the current device" % name)
    (B, R, C), (between, ld, inner) = (x.shape, x.stride()) if x.dim() == 3 else ((1, *x.shape), (0, *x.stride()))
    if R <= 1:
        ld = max(1, C)
    if B <= 1:
        between = R * ld
    if (C > 1 and inner != 1) or ld < C or (B > 1 and between < (R - 1) * ld + C):
        raise ValueError("%s must hold contiguous rows that do not overlap" % name)
    return x.data_ptr(), B, R, C, ld, between


def sgdb_orthogonalize_workspace_bytes(batch: int, rows: int, cols: int) -> int:
    return int(_lib.sgdb_orthogonalize_workspace_bytes(batch, rows, cols))


def sgdb_orthogonalize(u, out, newton_schulz: NewtonSchulz, workspace, info=None, stream=None) -> None:
    """u [rows, cols] or [batch, rows, cols] (f32 or bf16) -> out of the same shape (f32 or bf16): Newton-Schulz products."""
    here = _here(u)
    pu, B, R, C, ldu, su = _matrices(u, "u", here)
    po, *shape, ldo, so = _matrices(out, "out", here)
    if shape != [B, R, C]:
        raise ValueError("out must have the shape of u, got %s and %s" % (tuple(out.shape), tuple(u.shape)))
    c = newton_schulz._c()
    _check(_lib.sgdb_orthogonalize(pu, _code(u.dtype, "u"), B, R, C, ldu, su, ctypes.byref(c), po, _code(out.dtype, "out"), ldo, so,
                                   _whole(workspace, "workspace", here), workspace.numel() * workspace.element_size(),
                                   _vec(info, 2, "info", torch.int32, here), _stream(stream)), "sgdb_orthogonalize")


def sgdb_step_orthogonal_workspace_bytes(batch: int, rows: int, cols: int) -> int:
    return int(_lib.sgdb_step_orthogonal_workspace_bytes(batch, rows, cols))


def sgdb_step_orthogonal(grad, batch: int, rows: int, cols: int, arrival, tags, t: int, N: int, b: int, theta, momentum,
                         opt: OrthogonalOpt, mask, order, info, workspace, ld: int | None = None, stream=None) -> None:
    """One iteration for matrix parameters: select + mean of the kept rows + momentum + Newton-Schulz + update of theta."""
    ld = grad.stride(0) if ld is None else ld
    P, here = batch * rows * cols, _here(grad)
    for x, least, name in ((grad, (N + b - 1) * ld + P, "grad"), (arrival, N + b, "arrival"), (tags, N + b, "tags"), (mask, N + b, "mask"),
                           (order, N, "order"), (info, 2, "info")):
        if x.numel() < least:
            raise ValueError("%s must have at least %d elements, got %d" % (name, least, x.numel()))
    c = opt._c()
    _check(_lib.sgdb_step_orthogonal(
        _whole(grad, "grad", here), _grad_dtype(grad), batch, rows, cols, ld, _whole(arrival, "arrival", here, torch.float32),
        _whole(tags, "tags", here, torch.int32), t, N, b, _vec(theta, P, "theta", torch.float32, here),
        _vec(momentum, P, "momentum", torch.float32, here), ctypes.byref(c), _whole(mask, "mask", here, torch.uint8),
        _whole(order, "order", here, torch.int32), _whole(info, "info", here, torch.int32),
        _whole(workspace, "workspace", here), workspace.numel() * workspace.element_size(), _stream(stream)), "sgdb_step_orthogonal")
