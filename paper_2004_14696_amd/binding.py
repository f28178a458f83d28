"""ctypes binding of libdbw.so (the C ABI declared in include/dbw.h).

Argument marshalling only: every step of the DBW iteration runs in the HIP
library.  PyTorch supplies device memory and the stream; tensors are checked
for dtype, device, contiguity and shape before their pointers are passed.
The binding fails loudly when the library is not built -- there is no
fallback implementation.
"""
from __future__ import annotations

import ctypes
import functools
import os
from ctypes import POINTER, c_double, c_int32, c_int64, c_size_t, c_uint8, c_uint32, c_void_p

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libdbw.so")

DBW_OK, DBW_EINVAL, DBW_ERANGE, DBW_EHIP, DBW_ESTATE, DBW_EUNSUPPORTED = 0, -1, -2, -3, -4, -5
DBW_SOFTMAX, DBW_MLP, DBW_CNN = 0, 1, 2
DBW_CLOCK_FRESH, DBW_CLOCK_PSW, DBW_CLOCK_PSI = 0, 1, 2
DBW_POLICY_DBW, DBW_POLICY_STATIC, DBW_POLICY_BLIND = 0, 1, 2
DBW_ESTIMATOR_ISOTONIC, DBW_ESTIMATOR_NAIVE = 0, 1
DBW_G_ROWS_ALL, DBW_G_ROWS_SELECTED, DBW_G_ROWS_NONE = 0, 1, 2
DBW_MAX_N, DBW_MAX_D = 1024, 64
DBW_KT_GRADS, DBW_KT_AGGREGATE, DBW_KT_CHOOSE, DBW_KT_HOST_ESTIMATE, DBW_KT_HOST_STEP = 0, 1, 2, 3, 4
DBW_KT_HOST_WAIT, DBW_KT_HOST_QUEUE = 5, 6
DBW_F32, DBW_BF16, DBW_F16 = 0, 1, 2
DBW_GROUP_FORWARD, DBW_GROUP_INPUT_GRAD, DBW_GROUP_WEIGHT_GRAD = 0, 1, 2
ADAMW_BLOCK = 256   # values of one scale of the 8-bit states

STATUS_NAMES = {0: "DBW_OK", -1: "DBW_EINVAL", -2: "DBW_ERANGE", -3: "DBW_EHIP",
                -4: "DBW_ESTATE", -5: "DBW_EUNSUPPORTED"}

EXPORTED = (
    "dbw_param_count", "dbw_create", "dbw_destroy", "dbw_last_error", "dbw_sync",
    "dbw_worker_grads", "dbw_aggregate_fastest", "dbw_grad_stats", "dbw_choose_b", "dbw_step",
    "dbw_step_outputs", "dbw_time_estimate", "dbw_state_export", "dbw_state_import",
    "dbw_samples_export", "dbw_samples_import", "dbw_profile_enable", "dbw_kernel_time",
    "dbw_profile_reset", "dbw_time_estimator_create", "dbw_time_estimator_destroy",
    "dbw_time_estimator_solve", "dbw_time_estimator_stats", "dbw_busy_export", "dbw_busy_import",
    "dbw_grad_stats_static", "dbw_grads_route",
    "dbw_group_workspace", "dbw_group_product", "dbw_token_workspace", "dbw_token_loss",
    "dbw_adamw_create", "dbw_adamw_destroy", "dbw_adamw_step", "dbw_adamw_export", "dbw_adamw_import",
    "dbw_adamw_bits", "dbw_set_adamw",
)
DBW_STATIC_SCRATCH_BYTES = 8 * 1024 * 1024


class DBWError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


class Config(ctypes.Structure):
    _fields_ = [("model", c_int32), ("n", c_int32), ("B", c_int32), ("d", c_int32),
                ("C", c_int32), ("H", c_int32), ("D", c_int32), ("clock", c_int32),
                ("policy", c_int32), ("k_static", c_int32), ("estimator", c_int32),
                ("g_rows", c_int32), ("eta", c_double), ("beta", c_double), ("S", c_int64)]


class IterStats(ctypes.Structure):
    _fields_ = [("gnorm2", c_double), ("V_plus", c_double), ("N_plus", c_double), ("F_hat", c_double)]


class EstimatorState(ctypes.Structure):
    _fields_ = [("t", c_int64), ("k_prev", c_int32), ("nV", c_int32), ("nL", c_int32),
                ("nF", c_int32), ("F_prev", c_double), ("F_prev2", c_double),
                ("hV", c_double * DBW_MAX_D), ("hN", c_double * DBW_MAX_D),
                ("hL", c_double * DBW_MAX_D)]


class StepBuffers(ctypes.Structure):
    _fields_ = [(name, c_void_p) for name in
                ("G", "loss", "g", "mask", "sqnorm", "stats", "T_hat", "objective", "k", "b")]


class GroupShape(ctypes.Structure):
    _fields_ = [("form", c_int32), ("dtype", c_int32), ("out_dtype", c_int32), ("n", c_int32), ("d", c_int32),
                ("C", c_int32), ("T", c_int64), ("ld_d", c_int64), ("ld_C", c_int64), ("ld_W", c_int64),
                ("st_W", c_int64)]


class AdamWTensor(ctypes.Structure):
    _fields_ = [("w", c_void_p), ("g", c_void_p), ("m", c_void_p), ("v", c_void_p), ("m_scale", c_void_p),
                ("v_scale", c_void_p), ("w_low", c_void_p), ("count", c_int64), ("lr_scale", c_double),
                ("weight_decay", c_double)]


class AdamWConfig(ctypes.Structure):
    _fields_ = [("state_bits", c_int32), ("g_dtype", c_int32), ("low_dtype", c_int32), ("tensors", c_int32),
                ("t", c_int64)]


class AdamWHyper(ctypes.Structure):
    _fields_ = [("lr", c_double), ("beta1", c_double), ("beta2", c_double), ("eps", c_double),
                ("grad_scale", c_double), ("max_norm", c_double), ("seed", c_uint32)]


_lib = None


def load_library(path: str = LIB_PATH):
    """Load libdbw.so and declare its prototypes (raises if it is missing)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise ImportError(f"{path} is not built; run `python -m paper_2004_14696_amd.build`")
    # torch carries its own HIP runtime; loaded first, it is the one the
    # library binds to (loaded after the library, it would be a second
    # runtime in the process, and device memory and streams would not be
    # shared between the two)
    try:
        import torch  # noqa: F401
    except ImportError:
        pass
    lib = ctypes.CDLL(path)
    st = c_int32
    P = c_void_p
    lib.dbw_param_count.argtypes = [POINTER(Config)]
    lib.dbw_param_count.restype = c_int64
    lib.dbw_grads_route.argtypes = [POINTER(Config), POINTER(c_int32), POINTER(c_int32), POINTER(c_int32)]
    lib.dbw_grads_route.restype = st
    lib.dbw_create.argtypes = [POINTER(Config), P, POINTER(P)]
    lib.dbw_create.restype = st
    lib.dbw_destroy.argtypes = [P]
    lib.dbw_destroy.restype = None
    lib.dbw_last_error.argtypes = [P]
    lib.dbw_last_error.restype = ctypes.c_char_p
    lib.dbw_sync.argtypes = [P]
    lib.dbw_sync.restype = st
    lib.dbw_worker_grads.argtypes = [P, P, P, P, P, P, P]
    lib.dbw_worker_grads.restype = st
    lib.dbw_aggregate_fastest.argtypes = [P, P, P, c_int32, P, P]
    lib.dbw_aggregate_fastest.restype = st
    lib.dbw_grad_stats.argtypes = [P, P, P, c_int32, P, P, P, P]
    lib.dbw_grad_stats.restype = st
    lib.dbw_choose_b.argtypes = [P, P, P, P, P]
    lib.dbw_choose_b.restype = st
    lib.dbw_step.argtypes = [P, P, P, P, P, POINTER(c_int64), POINTER(c_int32)]
    lib.dbw_step.restype = st
    lib.dbw_step_outputs.argtypes = [P, POINTER(StepBuffers)]
    lib.dbw_step_outputs.restype = st
    lib.dbw_time_estimate.argtypes = [c_int32, POINTER(c_int64), POINTER(c_int64), POINTER(c_double)]
    lib.dbw_time_estimate.restype = st
    lib.dbw_time_estimator_create.argtypes = [POINTER(P)]
    lib.dbw_time_estimator_create.restype = st
    lib.dbw_time_estimator_destroy.argtypes = [P]
    lib.dbw_time_estimator_destroy.restype = None
    lib.dbw_time_estimator_solve.argtypes = [P, c_int32, POINTER(c_int64), POINTER(c_int64), POINTER(c_double)]
    lib.dbw_time_estimator_solve.restype = st
    lib.dbw_time_estimator_stats.argtypes = [P, POINTER(c_int64), POINTER(c_int64), POINTER(c_int64)]
    lib.dbw_time_estimator_stats.restype = st
    lib.dbw_busy_export.argtypes = [P, POINTER(c_int64)]
    lib.dbw_busy_export.restype = st
    lib.dbw_busy_import.argtypes = [P, POINTER(c_int64)]
    lib.dbw_busy_import.restype = st
    lib.dbw_state_export.argtypes = [P, POINTER(EstimatorState)]
    lib.dbw_state_export.restype = st
    lib.dbw_state_import.argtypes = [P, POINTER(EstimatorState)]
    lib.dbw_state_import.restype = st
    lib.dbw_samples_export.argtypes = [P, POINTER(c_int64), POINTER(c_int64), POINTER(c_int64)]
    lib.dbw_samples_export.restype = st
    lib.dbw_samples_import.argtypes = [P, POINTER(c_int64), POINTER(c_int64), c_int64]
    lib.dbw_samples_import.restype = st
    lib.dbw_profile_enable.argtypes = [P, c_int32]
    lib.dbw_profile_enable.restype = st
    lib.dbw_kernel_time.argtypes = [P, c_int32, POINTER(c_double), POINTER(c_int64)]
    lib.dbw_kernel_time.restype = st
    lib.dbw_profile_reset.argtypes = [P]
    lib.dbw_profile_reset.restype = st
    lib.dbw_grad_stats_static.argtypes = [c_int32, c_int64, P, P, c_int32, P, P, c_double, P, P, P]
    lib.dbw_grad_stats_static.restype = st
    lib.dbw_group_workspace.argtypes = [POINTER(GroupShape), POINTER(c_int64)]
    lib.dbw_group_workspace.restype = st
    lib.dbw_group_product.argtypes = [POINTER(GroupShape), P, P, P, P, P, c_int64, P]
    lib.dbw_group_product.restype = st
    lib.dbw_token_workspace.argtypes = [c_int32, c_int64]
    lib.dbw_token_workspace.restype = c_int64
    lib.dbw_token_loss.argtypes = [c_int32, c_int64, c_int32, c_int32, P, P, c_int64, P, c_double, P, c_int64, P, P,
                                   c_int64, P]
    lib.dbw_token_loss.restype = st
    lib.dbw_adamw_create.argtypes = [POINTER(AdamWConfig), POINTER(AdamWTensor), POINTER(P)]
    lib.dbw_adamw_create.restype = st
    lib.dbw_adamw_destroy.argtypes = [P]
    lib.dbw_adamw_destroy.restype = None
    lib.dbw_adamw_step.argtypes = [P, POINTER(AdamWHyper), P, P]
    lib.dbw_adamw_step.restype = st
    lib.dbw_adamw_export.argtypes = [P, POINTER(c_int64)]
    lib.dbw_adamw_export.restype = st
    lib.dbw_adamw_import.argtypes = [P, c_int64]
    lib.dbw_adamw_import.restype = st
    lib.dbw_set_adamw.argtypes = [P, P, POINTER(AdamWHyper)]
    lib.dbw_set_adamw.restype = st
    lib.dbw_adamw_bits.argtypes = [c_uint32, c_int64, c_int32, c_int64]
    lib.dbw_adamw_bits.restype = c_uint32
    _lib = lib
    return lib


CLOCKS = {"fresh": DBW_CLOCK_FRESH, "psw": DBW_CLOCK_PSW, "psi": DBW_CLOCK_PSI}
POLICIES = {"dbw": DBW_POLICY_DBW, "static": DBW_POLICY_STATIC, "blind": DBW_POLICY_BLIND}
ESTIMATORS = {"isotonic": DBW_ESTIMATOR_ISOTONIC, "naive": DBW_ESTIMATOR_NAIVE}
G_ROWS = {"all": DBW_G_ROWS_ALL, "selected": DBW_G_ROWS_SELECTED, "none": DBW_G_ROWS_NONE}


def make_config(model: str | int, n: int, B: int, d: int, C: int, H: int = 0, eta: float = 0.1,
                beta: float = 1.01, D: int = 5, S: int = 0, clock: str | int = DBW_CLOCK_FRESH,
                policy: str | int = DBW_POLICY_DBW, k_static: int = 0,
                estimator: str | int = DBW_ESTIMATOR_ISOTONIC, g_rows: str | int = DBW_G_ROWS_ALL) -> Config:
    if isinstance(model, str):
        model = {"softmax": DBW_SOFTMAX, "mlp": DBW_MLP, "cnn": DBW_CNN}[model]
    if isinstance(clock, str):
        clock = CLOCKS[clock]
    if isinstance(policy, str):
        policy = POLICIES[policy]
    if isinstance(estimator, str):
        estimator = ESTIMATORS[estimator]
    if isinstance(g_rows, str):
        g_rows = G_ROWS[g_rows]
    return Config(model=model, n=n, B=B, d=d, C=C, H=H, D=D, clock=clock, policy=policy,
                  k_static=k_static, estimator=estimator, g_rows=g_rows, eta=eta, beta=beta, S=S)


def param_count(cfg: Config) -> int:
    return int(load_library().dbw_param_count(ctypes.byref(cfg)))


def grads_route(cfg: Config) -> tuple[bool, int, bool]:
    """Kernels of the softmax gradients of a configuration (dbw_grads_route):
    (single pass over X, row slabs per worker, logits per dataset row)."""
    out = [c_int32() for _ in range(3)]
    st = load_library().dbw_grads_route(ctypes.byref(cfg), *map(ctypes.byref, out))
    if st != DBW_OK:
        raise DBWError(st, "invalid configuration")
    return bool(out[0].value), out[1].value, bool(out[2].value)


def time_estimate(cnt, tsum) -> np.ndarray:
    """Host time estimate (dbw_time_estimate): T_hat[k-1] for k = 1..n (NaN
    where no estimate exists)."""
    lib = load_library()
    cnt = np.ascontiguousarray(cnt, dtype=np.int64)
    tsum = np.ascontiguousarray(tsum, dtype=np.int64)
    n = cnt.shape[0]
    if cnt.shape != (n, n) or tsum.shape != (n, n):
        raise ValueError("cnt and tsum must be n x n")
    out = np.empty(n, dtype=np.float64)
    s = lib.dbw_time_estimate(n, cnt.ctypes.data_as(POINTER(c_int64)),
                              tsum.ctypes.data_as(POINTER(c_int64)),
                              out.ctypes.data_as(POINTER(c_double)))
    if s != DBW_OK:
        raise DBWError(s, "dbw_time_estimate rejected its input")
    return out


class TimeEstimator:
    """Incremental exact time estimate (dbw_time_estimator_*)."""

    def __init__(self):
        self.lib = load_library()
        h = c_void_p()
        s = self.lib.dbw_time_estimator_create(ctypes.byref(h))
        if s != DBW_OK:
            raise DBWError(s, "dbw_time_estimator_create failed")
        self.h = h

    def solve(self, cnt, tsum) -> np.ndarray:
        cnt = np.ascontiguousarray(cnt, dtype=np.int64)
        tsum = np.ascontiguousarray(tsum, dtype=np.int64)
        n = cnt.shape[0]
        if cnt.shape != (n, n) or tsum.shape != (n, n):
            raise ValueError("cnt and tsum must be n x n")
        out = np.empty(n, dtype=np.float64)
        s = self.lib.dbw_time_estimator_solve(self.h, n, cnt.ctypes.data_as(POINTER(c_int64)),
                                              tsum.ctypes.data_as(POINTER(c_int64)),
                                              out.ctypes.data_as(POINTER(c_double)))
        if s != DBW_OK:
            raise DBWError(s, "dbw_time_estimator_solve rejected its input")
        return out

    def stats(self) -> dict:
        """Solves so far by path: fast (per-column fit feasible), warm, full."""
        f, w, u = c_int64(), c_int64(), c_int64()
        s = self.lib.dbw_time_estimator_stats(self.h, ctypes.byref(f), ctypes.byref(w), ctypes.byref(u))
        if s != DBW_OK:
            raise DBWError(s, "dbw_time_estimator_stats failed")
        return {"fast": f.value, "warm": w.value, "full": u.value}

    def __del__(self):
        if getattr(self, "h", None):
            self.lib.dbw_time_estimator_destroy(self.h)
            self.h = None


def grad_stats_static(G, mask, k, g, loss, V_window=0.0, sqnorm=None, stats=None, stream=None):
    """dbw_grad_stats_static: the statistics of dbw_grad_stats with no context
    and no allocation inside the call (scratch in the library's static device
    array).  G [n][P] float32, mask [n] uint8, g [P] float32, loss [n]
    float32, all on the current device; V_window is V_plus for k = 1.
    Returns (sqnorm [n] float32, stats float64 [4] = gnorm2, V_plus, N_plus,
    F_hat); pass sqnorm and stats to write into existing tensors."""
    torch = _torch()
    lib = load_library()
    if G.dim() != 2:
        raise ValueError("G must be [n][P]")
    n, P = G.shape
    dev = G.device
    for name, t, dtype, shape in (("G", G, torch.float32, (n, P)), ("mask", mask, torch.uint8, (n,)),
                                  ("g", g, torch.float32, (P,)), ("loss", loss, torch.float32, (n,))):
        if t.device != dev or t.dtype != dtype or not t.is_contiguous() or tuple(t.shape) != shape:
            raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {shape} on {dev}")
    sqnorm = torch.empty(n, dtype=torch.float32, device=dev) if sqnorm is None else sqnorm
    stats = torch.empty(4, dtype=torch.float64, device=dev) if stats is None else stats
    if tuple(sqnorm.shape) != (n,) or sqnorm.dtype != torch.float32 or sqnorm.device != dev:
        raise ValueError("sqnorm must be float32 [n] on the device of G")
    if tuple(stats.shape) != (4,) or stats.dtype != torch.float64 or stats.device != dev:
        raise ValueError("stats must be float64 [4] on the device of G")
    if stream is None:
        stream = torch.cuda.current_stream(dev)
    s = lib.dbw_grad_stats_static(int(n), int(P), c_void_p(G.data_ptr()), c_void_p(mask.data_ptr()), int(k),
                                  c_void_p(g.data_ptr()), c_void_p(loss.data_ptr()), float(V_window),
                                  c_void_p(sqnorm.data_ptr()), c_void_p(stats.data_ptr()),
                                  c_void_p(stream.cuda_stream))
    if s != DBW_OK:
        raise DBWError(s, lib.dbw_last_error(None).decode())
    return sqnorm, stats


# -- operators for language models ---------------------------------------------
_codes = None


def _dtype_code(torch, dtype, name, allowed):
    global _codes
    if _codes is None:
        _codes = {torch.float32: DBW_F32, torch.bfloat16: DBW_BF16, torch.float16: DBW_F16}
    code = _codes.get(dtype)
    if code is None or code not in allowed:
        raise ValueError(f"{name} has an unsupported type: {dtype}")
    return code


def _rows_of(t, shape, dtype, dev, name):
    """Pointer and row stride of a tensor [..][rows][columns] with contiguous
    columns."""
    if t.device != dev or t.dtype != dtype or t.shape != shape:
        raise ValueError(f"{name} must be {dtype} {shape} on {dev}, not {t.dtype} {tuple(t.shape)} on {t.device}")
    strides = t.stride()
    if strides[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"the last dimension of {name} must be contiguous")
    # a single row has no stride of its own
    return t.data_ptr(), strides[-2] if shape[-2] > 1 else shape[-1]


def _flat(t, shape, dtype, dev, name):
    if t.device != dev or t.dtype != dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {dev}")
    return t.data_ptr()


def _stream_of(torch, dev):
    """The raw handle of the current stream of `dev`."""
    if dev.type != "cuda":
        raise ValueError(f"tensors must live on a GPU, not {dev}")
    return torch._C._cuda_getCurrentRawStream(dev.index)


def _on(stream, dev, function, *args, **kw):
    """function with `stream` as the current one, so that what it allocates
    belongs to that stream."""
    if stream.device != dev:
        raise ValueError(f"the stream is of {stream.device}, the tensors are on {dev}")
    with _torch().cuda.stream(stream):
        return function(*args, **kw)


def _call(torch, lib, dev, function, *args):
    """function(*args) with `dev` as the current device; raises its error."""
    if torch.cuda.current_device() == dev.index:
        st = function(*args)
    else:
        with torch.cuda.device(dev):
            st = function(*args)
    if st != DBW_OK:
        raise DBWError(st, lib.dbw_last_error(None).decode())


def _workspace(torch, nbytes, dev, workspace):
    """Pointer, size and tensor of a workspace of at least nbytes."""
    if workspace is None:
        if nbytes <= 0:
            return None, 0, None
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    elif workspace.device != dev or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on {dev}")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


_HALVES = (DBW_BF16, DBW_F16)
_FLOATS = (DBW_F32, DBW_BF16, DBW_F16)


@functools.lru_cache(maxsize=512)
def _group_shape(*sizes):
    """A dbw_group_shape, by reference, and its bytes of workspace."""
    lib = load_library()
    ref = ctypes.byref(GroupShape(*sizes))
    need = c_int64()
    st = lib.dbw_group_workspace(ref, ctypes.byref(need))
    if st != DBW_OK:
        raise DBWError(st, lib.dbw_last_error(None).decode())
    return ref, need.value


def _group(form, a, b, offsets, out, out_dtype, d, C, workspace, stream=None):
    if stream is not None:
        return _on(stream, a.device, _group, form, a, b, offsets, out, out_dtype, d, C, workspace)
    torch = _torch()
    lib = load_library()
    dev, dtype = a.device, a.dtype
    if offsets.dim() != 1 or offsets.numel() < 2:
        raise ValueError("offsets must be [n + 1]")
    if a.dim() != 2:
        raise ValueError("token rows must be [T][columns]")
    n, T = offsets.numel() - 1, a.shape[0]
    po = _flat(offsets, (n + 1,), torch.int32, dev, "offsets")
    if out_dtype is None:
        out_dtype = dtype if out is None else out.dtype
    codes = _dtype_code(torch, dtype, "the inputs", _HALVES), _dtype_code(torch, out_dtype, "the output", _FLOATS)
    raw = _stream_of(torch, dev)
    if form == DBW_GROUP_WEIGHT_GRAD:
        if out is None:
            out = torch.empty((n, d, C), dtype=out_dtype, device=dev)
        pa, ld_d = _rows_of(a, (T, d), dtype, dev, "X")
        pb, ld_C = _rows_of(b, (T, C), dtype, dev, "dY")
        pc, ld_W = _rows_of(out, (n, d, C), out_dtype, dev, "G")
        st_W = out.stride(0)
    else:
        forward = form == DBW_GROUP_FORWARD
        K, N = (d, C) if forward else (C, d)
        if out is None:
            out = torch.empty((T, N), dtype=out_dtype, device=dev)
        pa, lda = _rows_of(a, (T, K), dtype, dev, "X" if forward else "dY")
        pb, ld_W = _rows_of(b, (n, d, C) if b.dim() == 3 else (d, C), dtype, dev, "W")
        pc, ldo = _rows_of(out, (T, N), out_dtype, dev, "Y" if forward else "dX")
        ld_d, ld_C = (lda, ldo) if forward else (ldo, lda)
        # one matrix for all groups has no distance to the next one
        st_W = b.stride(0) if b.dim() == 3 and n > 1 else 0
    ref, need = _group_shape(form, codes[0], codes[1], n, d, C, T, ld_d, ld_C, ld_W, st_W)
    pw, nbytes, keep = _workspace(torch, need, dev, workspace)
    _call(torch, lib, dev, lib.dbw_group_product, ref, po, pa, pb, pc, pw, nbytes, raw)
    return out


def group_matmul(X, W, offsets, out=None, out_dtype=None, workspace=None, stream=None):
    """Y[t] = X[t] W_i for the rows t = offsets[i] .. offsets[i+1]-1 of each
    group i (dbw_group_product, FORWARD).  X [T][d] bf16 or fp16, W [n][d][C], or
    [d][C] for all groups, offsets [n+1] int32; rows may be strided.  Returns
    Y [T][C] in ``out_dtype`` (that of X, or float32); rows of no group keep
    what ``out`` held."""
    if W.dim() not in (2, 3):
        raise ValueError("W must be [n][d][C] or [d][C]")
    d, C = W.shape[-2:]
    return _group(DBW_GROUP_FORWARD, X, W, offsets, out, out_dtype, d, C, workspace, stream)


def group_input_grad(dY, W, offsets, out=None, out_dtype=None, workspace=None, stream=None):
    """dX[t] = dY[t] W_i^T: the gradient of group_matmul to its rows
    (dbw_group_product, INPUT_GRAD).  Returns dX [T][d]."""
    if W.dim() not in (2, 3):
        raise ValueError("W must be [n][d][C] or [d][C]")
    d, C = W.shape[-2:]
    return _group(DBW_GROUP_INPUT_GRAD, dY, W, offsets, out, out_dtype, d, C, workspace, stream)


def group_weight_grad(X, dY, offsets, out=None, out_dtype=None, workspace=None, stream=None):
    """G_i = sum over the rows t of group i of X[t]^T dY[t]: the gradient of
    group_matmul to its weights, or the worker gradients of workers with
    ragged minibatches (dbw_group_product, WEIGHT_GRAD).  Returns G [n][d][C]
    in ``out_dtype`` (float32 unless given)."""
    if dY.dim() != 2 or X.dim() != 2:
        raise ValueError("X must be [T][d] and dY [T][C]")
    if out_dtype is None:
        out_dtype = _torch().float32 if out is None else out.dtype
    return _group(DBW_GROUP_WEIGHT_GRAD, X, dY, offsets, out, out_dtype, X.shape[1], dY.shape[1], workspace, stream)


def token_loss(Z, y, offsets, scale=1.0, dZ=None, loss=None, grad=True, workspace=None, stream=None):
    """Mean cross entropy of each worker's tokens and its gradient
    (dbw_token_loss).  Z [T][C] float32, bfloat16 or float16 logits, y [T] int32
    labels (negative: the row is masked), offsets [n+1] int32.  Returns
    (loss [n] float32, dZ [T][C] of the type of Z, times ``scale``); dZ may be
    Z, to write the gradient in its place; ``grad`` False: no gradient (None),
    and nothing is written to a dZ that is given."""
    if stream is not None:
        return _on(stream, Z.device, token_loss, Z, y, offsets, scale, dZ, loss, grad, workspace)
    torch = _torch()
    lib = load_library()
    dev, dtype = Z.device, Z.dtype
    if Z.dim() != 2 or offsets.dim() != 1 or offsets.numel() < 2:
        raise ValueError("Z must be [T][C] and offsets [n + 1]")
    T, C = Z.shape
    n = offsets.numel() - 1
    code = _dtype_code(torch, dtype, "Z", _FLOATS)
    raw = _stream_of(torch, dev)
    po = _flat(offsets, (n + 1,), torch.int32, dev, "offsets")
    py = _flat(y, (T,), torch.int32, dev, "y")
    pz, ld_Z = _rows_of(Z, (T, C), dtype, dev, "Z")
    if not grad:
        dZ = None
    elif dZ is None:
        dZ = torch.empty((T, C), dtype=dtype, device=dev)
    pd, ld_dZ = _rows_of(dZ, (T, C), dtype, dev, "dZ") if dZ is not None else (None, 0)
    if loss is None:
        loss = torch.empty(n, dtype=torch.float32, device=dev)
    pl = _flat(loss, (n,), torch.float32, dev, "loss")
    pw, nbytes, keep = _workspace(torch, lib.dbw_token_workspace(n, T), dev, workspace)
    _call(torch, lib, dev, lib.dbw_token_loss, n, T, C, code, po, pz, ld_Z, py, scale, pd, ld_dZ, pl, pw, nbytes, raw)
    return loss, dZ


def adamw_states(w, bits=32):
    """Zero states of AdamW for the tensors ``w``: keyword arguments m, v (and
    m_scale, v_scale with 8 bits)."""
    torch = _torch()
    if bits == 32:
        return {"m": [torch.zeros_like(t) for t in w], "v": [torch.zeros_like(t) for t in w]}
    if bits != 8:
        raise ValueError("states have 8 or 32 bits")
    codes = lambda: [torch.zeros(t.shape, dtype=torch.uint8, device=t.device).view(torch.float8_e4m3fn) for t in w]  # noqa: E731
    scales = lambda: [torch.ones(-(-t.numel() // ADAMW_BLOCK), dtype=torch.uint8, device=t.device)                   # noqa: E731
                      .view(torch.float8_e8m0fnu) for t in w]
    return {"m": codes(), "v": codes(), "m_scale": scales(), "v_scale": scales()}


class AdamW:
    """AdamW over a list of tensors (dbw_adamw_*), updated in place.

    w float32 tensors, g their gradients (all of one type: float32, bfloat16 or
    float16), m and v their states: float32, or float8_e4m3fn codes with
    m_scale and v_scale, one float8_e8m0fnu for each 256 values (adamw_states
    makes either).  low: bfloat16 or float16 copies of w, written by every step.
    weight_decay and lr_scale: a number, or one for each tensor.  step: steps
    made before.  The tensors' memory is kept, so gradients are written into
    the same g before every step."""

    def __init__(self, w, g, m, v, m_scale=None, v_scale=None, low=None, weight_decay=0.0, lr_scale=1.0, step=0):
        torch = _torch()
        self.lib = load_library()
        self.h = None
        w, g, m, v = list(w), list(g), list(m), list(v)
        n = len(w)
        if n == 0:
            raise ValueError("no tensors")
        bits = 32 if m_scale is None and v_scale is None else 8
        lists = {"g": g, "m": m, "v": v}
        if bits == 8:
            if m_scale is None or v_scale is None:
                raise ValueError("8-bit states need m_scale and v_scale")
            m_scale, v_scale = list(m_scale), list(v_scale)
            lists |= {"m_scale": m_scale, "v_scale": v_scale}
        if low is not None:
            low = list(low)
            lists["low"] = low
        per = lambda x: list(x) if isinstance(x, (list, tuple)) else [x] * n   # noqa: E731
        decay, scale = per(weight_decay), per(lr_scale)
        for name, x in {**lists, "weight_decay": decay, "lr_scale": scale}.items():
            if len(x) != n:
                raise ValueError(f"{name} must have one entry for each of the {n} tensors")
        dev = w[0].device
        state = torch.float32 if bits == 32 else torch.float8_e4m3fn
        table = (AdamWTensor * n)()
        low_type = low[0].dtype if low is not None else torch.bfloat16
        cfg = AdamWConfig(state_bits=bits, tensors=n, t=int(step),
                          g_dtype=_dtype_code(torch, g[0].dtype, "g", (DBW_F32, DBW_BF16, DBW_F16)),
                          low_dtype=_dtype_code(torch, low_type, "low", (DBW_BF16, DBW_F16)))
        for i, t in enumerate(table):
            shape = w[i].shape
            t.count = w[i].numel()
            blocks = (-(-t.count // ADAMW_BLOCK),)
            t.w = _flat(w[i], shape, torch.float32, dev, f"w[{i}]")
            t.g = _flat(g[i], shape, g[0].dtype, dev, f"g[{i}]")
            t.m = _flat(m[i], shape, state, dev, f"m[{i}]")
            t.v = _flat(v[i], shape, state, dev, f"v[{i}]")
            if bits == 8:
                t.m_scale = _flat(m_scale[i], blocks, torch.float8_e8m0fnu, dev, f"m_scale[{i}]")
                t.v_scale = _flat(v_scale[i], blocks, torch.float8_e8m0fnu, dev, f"v_scale[{i}]")
            if low is not None:
                t.w_low = _flat(low[i], shape, low_type, dev, f"low[{i}]")
            t.lr_scale, t.weight_decay = float(scale[i]), float(decay[i])
        self.device = dev
        self._keep = (w, lists)      # the plan holds their addresses
        _stream_of(torch, dev)
        handle = c_void_p()
        _call(torch, self.lib, dev, self.lib.dbw_adamw_create, ctypes.byref(cfg), table, ctypes.byref(handle))
        self.h = handle

    def step(self, lr, beta1=0.9, beta2=0.999, eps=1e-8, max_norm=0.0, grad_scale=1.0, seed=0, norm=None, stream=None):
        """One step.  grad_scale multiplies the gradients; max_norm > 0 clips
        their norm (over all tensors).  Returns the norm before clipping, a
        float32 scalar tensor, where max_norm or ``norm`` (a tensor to write
        it to) is given, else None."""
        if stream is not None:
            return _on(stream, self.device, self.step, lr, beta1, beta2, eps, max_norm, grad_scale, seed, norm)
        self._open()
        torch = _torch()
        if norm is None and max_norm:
            norm = torch.empty((), dtype=torch.float32, device=self.device)
        pn = _flat(norm, norm.shape, torch.float32, self.device, "norm") if norm is not None else None
        if norm is not None and norm.numel() != 1:
            raise ValueError("norm must have one element")
        hyper = AdamWHyper(lr, beta1, beta2, eps, grad_scale, max_norm, int(seed) & 0xFFFFFFFF)
        st = self.lib.dbw_adamw_step(self.h, ctypes.byref(hyper), pn, _stream_of(torch, self.device))
        if st != DBW_OK:
            raise DBWError(st, self.lib.dbw_last_error(None).decode())
        return norm

    @property
    def t(self) -> int:
        """Steps made (waits for the device)."""
        out, plan = c_int64(), self._open()
        st = self.lib.dbw_adamw_export(plan, ctypes.byref(out))
        if st != DBW_OK:
            raise DBWError(st, self.lib.dbw_last_error(None).decode())
        return out.value

    @t.setter
    def t(self, value: int):
        plan = self._open()
        st = self.lib.dbw_adamw_import(plan, int(value))
        if st != DBW_OK:
            raise DBWError(st, self.lib.dbw_last_error(None).decode())

    def _open(self):
        """The plan's handle."""
        if self.h is None:
            raise ValueError("the AdamW plan is closed")
        return self.h

    def close(self):
        if self.h is not None:
            self.lib.dbw_adamw_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---------------------------------------------------------------------------
_hip = None


def _hip_runtime():
    """libamdhip64 for device-to-device copies out of the library's buffers."""
    global _hip
    if _hip is None:
        _hip = ctypes.CDLL("libamdhip64.so")
        _hip.hipMemcpyAsync.argtypes = [c_void_p, c_void_p, c_size_t, c_int32, c_void_p]
        _hip.hipMemcpyAsync.restype = c_int32
    return _hip


HIP_MEMCPY_D2D = 3


def _torch():
    import torch
    return torch


class _Simulation:
    """A dbw_ctx, destroyed with the last reference to it: its Context's, and
    those of views of its memory.  It refers to neither, as no collector would
    find a cycle through a tensor's memory."""

    def __init__(self, lib, handle):
        self.lib, self.handle = lib, handle

    def __del__(self):
        try:
            self.lib.dbw_destroy(self.handle)
        except Exception:
            pass


class _DeviceArray:
    """float32 [n] device memory of a _Simulation, for torch.as_tensor."""

    def __init__(self, owner, ptr, n):
        self.owner = owner
        self.__cuda_array_interface__ = {"shape": (n,), "typestr": "<f4", "data": (ptr, False), "version": 2}


class Context:
    """One DBW parameter-server simulation bound to a torch CUDA (HIP) stream."""

    _adamw = None   # the plan of use_adamw
    _simulation = None

    def __init__(self, cfg: Config, stream=None, device=None):
        torch = _torch()
        self.lib = load_library()
        self.cfg = cfg
        self.device = torch.device("cuda", torch.cuda.current_device() if device is None else device)
        with torch.cuda.device(self.device):
            self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
            handle = c_void_p()
            s = self.lib.dbw_create(ctypes.byref(cfg), c_void_p(self.stream.cuda_stream), ctypes.byref(handle))
        if s != DBW_OK:
            raise DBWError(s, "dbw_create failed (invalid configuration or HIP error)")
        self.h = handle
        self._simulation = _Simulation(self.lib, handle)
        self.P = param_count(cfg)

    def close(self):
        """Ends the simulation.  Its memory is freed here, or with the last
        view of gradient() (a plan keeps those that it was given)."""
        self.h = self._adamw = self._simulation = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- helpers -------------------------------------------------------------
    def _check(self, s: int, what: str):
        if s != DBW_OK:
            raise DBWError(s, f"{what}: {self.lib.dbw_last_error(self.h).decode()}")

    def _dev(self, t, dtype, shape, name):
        torch = _torch()
        if not isinstance(t, torch.Tensor):
            raise TypeError(f"{name} must be a torch tensor")
        if t.device != self.device:
            raise ValueError(f"{name} must live on {self.device}, not {t.device}")
        if t.dtype != dtype:
            raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        if shape is not None and tuple(t.shape) != tuple(shape):
            raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
        return c_void_p(t.data_ptr())

    def _empty(self, shape, dtype):
        return _torch().empty(shape, dtype=dtype, device=self.device)

    def _batch(self, X, y, rows):
        torch = _torch()
        c = self.cfg
        if rows is None:
            return (self._dev(X, torch.float32, (c.n, c.B, c.d), "X"),
                    self._dev(y, torch.int32, (c.n, c.B), "y"), None)
        return (self._dev(X, torch.float32, (c.S, c.d), "X (dataset)"),
                self._dev(y, torch.int32, (c.S,), "y (labels)"),
                self._dev(rows, torch.int32, (c.n, c.B), "rows"))

    # -- the five calls --------------------------------------------------------
    def worker_grads(self, w, X, y, rows=None, G=None, loss=None):
        torch = _torch()
        c = self.cfg
        G = self._empty((c.n, self.P), torch.float32) if G is None else G
        loss = self._empty((c.n,), torch.float32) if loss is None else loss
        px, py, pr = self._batch(X, y, rows)
        self._check(self.lib.dbw_worker_grads(self.h, self._dev(w, torch.float32, (self.P,), "w"), px, py, pr,
                                              self._dev(G, torch.float32, (c.n, self.P), "G"),
                                              self._dev(loss, torch.float32, (c.n,), "loss")),
                    "dbw_worker_grads")
        return G, loss

    def aggregate_fastest(self, G, ticks, k, g=None, mask=None):
        torch = _torch()
        c = self.cfg
        g = self._empty((self.P,), torch.float32) if g is None else g
        mask = self._empty((c.n,), torch.uint8) if mask is None else mask
        self._check(self.lib.dbw_aggregate_fastest(
            self.h, self._dev(G, torch.float32, (c.n, self.P), "G"),
            self._dev(ticks, torch.int64, (c.n,), "ticks"), int(k),
            self._dev(g, torch.float32, (self.P,), "g"), self._dev(mask, torch.uint8, (c.n,), "mask")),
            "dbw_aggregate_fastest")
        return g, mask

    def grad_stats(self, G, mask, k, g, loss, sqnorm=None, stats=None):
        """Returns (sqnorm [n] float32, stats float64 [4] = gnorm2, V_plus, N_plus, F_hat)."""
        torch = _torch()
        c = self.cfg
        sqnorm = self._empty((c.n,), torch.float32) if sqnorm is None else sqnorm
        stats = self._empty((4,), torch.float64) if stats is None else stats
        self._check(self.lib.dbw_grad_stats(
            self.h, self._dev(G, torch.float32, (c.n, self.P), "G"),
            self._dev(mask, torch.uint8, (c.n,), "mask"), int(k),
            self._dev(g, torch.float32, (self.P,), "g"), self._dev(loss, torch.float32, (c.n,), "loss"),
            self._dev(sqnorm, torch.float32, (c.n,), "sqnorm"), self._dev(stats, torch.float64, (4,), "stats")),
            "dbw_grad_stats")
        return sqnorm, stats

    def choose_b(self, T_hat, k=None, b=None, objective=None):
        torch = _torch()
        c = self.cfg
        k = self._empty((1,), torch.int32) if k is None else k
        b = self._empty((1,), torch.int32) if b is None else b
        objective = self._empty((c.n,), torch.float64) if objective is None else objective
        self._check(self.lib.dbw_choose_b(self.h, self._dev(T_hat, torch.float64, (c.n,), "T_hat"),
                                          self._dev(k, torch.int32, (1,), "k"),
                                          self._dev(b, torch.int32, (1,), "b"),
                                          self._dev(objective, torch.float64, (c.n,), "objective")),
                    "dbw_choose_b")
        return k, b, objective

    def step(self, w, X, y, ticks, rows=None, wait: bool = False):
        """One DBW iteration; updates w in place.  Returns k_t if ``wait``."""
        if self._adamw is not None:
            self._adamw._open()      # not closed since use_adamw
        torch = _torch()
        c = self.cfg
        ticks = np.ascontiguousarray(ticks, dtype=np.int64)
        if ticks.shape != (c.n,):
            raise ValueError(f"ticks must have shape ({c.n},)")
        px, py, pr = self._batch(X, y, rows)
        kout = c_int32(0)
        self._check(self.lib.dbw_step(self.h, self._dev(w, torch.float32, (self.P,), "w"), px, py, pr,
                                      ticks.ctypes.data_as(POINTER(c_int64)),
                                      ctypes.byref(kout) if wait else None), "dbw_step")
        return int(kout.value) if wait else None

    def gradient(self):
        """The context's g_t [P], which every step writes (a view, which keeps
        the simulation's memory): the gradients of a plan for use_adamw."""
        bufs = StepBuffers()
        self._check(self.lib.dbw_step_outputs(self.h, ctypes.byref(bufs)), "dbw_step_outputs")
        return _torch().as_tensor(_DeviceArray(self._simulation, bufs.g, self.P), device=self.device)

    def use_adamw(self, opt, lr=0.0, beta1=0.9, beta2=0.999, eps=1e-8, max_norm=0.0, grad_scale=1.0, seed=0):
        """From now on every step updates w by one step of ``opt`` (an AdamW
        whose gradients are slices of gradient(), in the places that its w have
        in the w of step) instead of by SGD; None: by SGD again."""
        hyper = AdamWHyper(lr, beta1, beta2, eps, grad_scale, max_norm, int(seed) & 0xFFFFFFFF)
        plan = opt._open() if opt is not None else None   # (a closed plan's NULL would mean SGD)
        self._check(self.lib.dbw_set_adamw(self.h, plan, ctypes.byref(hyper)),
                    "dbw_set_adamw")
        self._adamw = opt            # the plan outlives its use

    def step_outputs(self):
        """Copies of the buffers the last step wrote (torch tensors)."""
        torch = _torch()
        c = self.cfg
        bufs = StepBuffers()
        self._check(self.lib.dbw_step_outputs(self.h, ctypes.byref(bufs)), "dbw_step_outputs")
        spec = {"G": ((c.n, self.P), torch.float32), "loss": ((c.n,), torch.float32),
                "g": ((self.P,), torch.float32), "mask": ((c.n,), torch.uint8),
                "sqnorm": ((c.n,), torch.float32), "stats": ((4,), torch.float64),
                "T_hat": ((c.n,), torch.float64), "objective": ((c.n,), torch.float64),
                "k": ((1,), torch.int32), "b": ((1,), torch.int32)}
        hip = _hip_runtime()
        out = {}
        for name, (shape, dtype) in spec.items():
            t = self._empty(shape, dtype)
            nbytes = t.numel() * t.element_size()
            e = hip.hipMemcpyAsync(c_void_p(t.data_ptr()), c_void_p(getattr(bufs, name)), nbytes,
                                   HIP_MEMCPY_D2D, c_void_p(self.stream.cuda_stream))
            if e != 0:
                raise DBWError(DBW_EHIP, f"hipMemcpyAsync of {name} failed ({e})")
            out[name] = t
        return out

    def sync(self):
        self._check(self.lib.dbw_sync(self.h), "dbw_sync")

    # -- state -------------------------------------------------------------------
    def export_state(self) -> dict:
        s = EstimatorState()
        self._check(self.lib.dbw_state_export(self.h, ctypes.byref(s)), "dbw_state_export")
        return {"t": s.t, "k_prev": s.k_prev, "hV": list(s.hV[:s.nV]), "hN": list(s.hN[:s.nV]),
                "hL": list(s.hL[:s.nL]), "nF": s.nF, "F_prev": s.F_prev, "F_prev2": s.F_prev2}

    def import_state(self, st: dict):
        s = EstimatorState()
        s.t = int(st["t"])
        s.k_prev = int(st["k_prev"])
        hV, hN, hL = list(st["hV"]), list(st["hN"]), list(st["hL"])
        if len(hV) != len(hN):
            raise ValueError("hV and hN must have the same length")
        s.nV, s.nL, s.nF = len(hV), len(hL), int(st["nF"])
        for i, v in enumerate(hV):
            s.hV[i] = v
        for i, v in enumerate(hN):
            s.hN[i] = v
        for i, v in enumerate(hL):
            s.hL[i] = v
        s.F_prev = float(st.get("F_prev", 0.0))
        s.F_prev2 = float(st.get("F_prev2", 0.0))
        self._check(self.lib.dbw_state_import(self.h, ctypes.byref(s)), "dbw_state_import")

    def export_samples(self):
        n = self.cfg.n
        cnt = np.zeros((n, n), np.int64)
        tsum = np.zeros((n, n), np.int64)
        clock = c_int64(0)
        self._check(self.lib.dbw_samples_export(self.h, cnt.ctypes.data_as(POINTER(c_int64)),
                                                tsum.ctypes.data_as(POINTER(c_int64)), ctypes.byref(clock)),
                    "dbw_samples_export")
        return cnt, tsum, int(clock.value)

    def export_busy(self) -> np.ndarray:
        """Push & Wait: the time each worker becomes free (ticks)."""
        out = np.empty(self.cfg.n, dtype=np.int64)
        self._check(self.lib.dbw_busy_export(self.h, out.ctypes.data_as(POINTER(c_int64))), "dbw_busy_export")
        return out

    def import_busy(self, busy):
        b = np.ascontiguousarray(busy, dtype=np.int64)
        if b.shape != (self.cfg.n,):
            raise ValueError(f"busy must have shape ({self.cfg.n},)")
        self._check(self.lib.dbw_busy_import(self.h, b.ctypes.data_as(POINTER(c_int64))), "dbw_busy_import")

    def import_samples(self, cnt, tsum, clock: int = 0):
        cnt = np.ascontiguousarray(cnt, dtype=np.int64)
        tsum = np.ascontiguousarray(tsum, dtype=np.int64)
        self._check(self.lib.dbw_samples_import(self.h, cnt.ctypes.data_as(POINTER(c_int64)),
                                                tsum.ctypes.data_as(POINTER(c_int64)), int(clock)),
                    "dbw_samples_import")

    # -- timing --------------------------------------------------------------------
    def profile(self, on=True):
        """True/1: device events and host timers; 2: host timers only; False/0: off."""
        mode = 1 if on is True else (0 if on is False else int(on))
        self._check(self.lib.dbw_profile_enable(self.h, mode), "dbw_profile_enable")

    def profile_reset(self):
        self._check(self.lib.dbw_profile_reset(self.h), "dbw_profile_reset")

    def kernel_time(self, group: int):
        ms, n = c_double(0.0), c_int64(0)
        self._check(self.lib.dbw_kernel_time(self.h, int(group), ctypes.byref(ms), ctypes.byref(n)),
                    "dbw_kernel_time")
        return float(ms.value), int(n.value)
