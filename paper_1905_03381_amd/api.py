"""Thin ctypes binding of libautoassist.so (include/autoassist.h).

Argument marshalling only: every step of the path runs in the HIP kernels.
Tensors are torch CUDA tensors (device memory and streams come from PyTorch);
each function takes the same arguments as the C entry point of the same name
and launches on torch's current stream.  There is no CPU fallback: if the
library is missing or fails to load, every call raises.
"""
import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libautoassist.so")

AA_OK = 0
AA_DENSE, AA_CSR = 0, 1
DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}   # AA_F32, AA_BF16, AA_F16
SCORES = {"softmax": 0, "sigmoid": 1}
ACTIVATIONS = {"none": 0, "relu": 1, "gated": 2}
DENSE_ACTIVATIONS = dict(ACTIVATIONS, silu=3, gelu=4)   # of linear and linear_grad

SYMBOLS = [
    "aa_version", "aa_status_string", "aa_workspace_bytes", "aa_workspace_init", "aa_profile_hook",
    "aa_profile_hooks",
    "aa_assistant_score", "aa_shrink", "aa_score_shrink", "aa_shrink_threshold", "aa_gather",
    "aa_gather_csr", "aa_svm_sgd_step", "aa_assistant_update", "aa_boss_assistant_step",
    "aa_fused_step", "aa_sk_step", "aa_train_epoch", "aa_threshold_update",
    "aa_threshold_assistant_update", "aa_bucket_batches",
    "aa_pipeline_workspace_bytes", "aa_train_epoch_stale", "aa_sk_epoch",
    "aa_static_scratch_bytes", "aa_fused_step_static",
    "aa_expert_workspace_bytes", "aa_route", "aa_route_grad", "aa_expert_plan", "aa_expert_forward",
    "aa_expert_grad_input", "aa_expert_grad_weight", "aa_expert_combine", "aa_expert_combine_grad",
    "aa_dropout",
    "aa_layer_workspace_bytes", "aa_layer_norm", "aa_layer_norm_grad", "aa_linear", "aa_linear_grad", "aa_balance", "aa_balance_grad",
    "aa_adamw_chunks", "aa_adamw_table_bytes", "aa_adamw_table", "aa_grad_norm", "aa_adamw_step",
]


class AAError(RuntimeError):
    pass


class aa_features(C.Structure):
    _fields_ = [("layout", C.c_int32), ("d", C.c_int32), ("n", C.c_int64),
                ("x", C.c_void_p), ("ld", C.c_int64),
                ("rowptr", C.c_void_p), ("col", C.c_void_p), ("val", C.c_void_p)]


class aa_step_config(C.Structure):
    _fields_ = [("gamma", C.c_float), ("lambda_", C.c_float), ("lr", C.c_float),
                ("lr_a", C.c_float), ("l2_a", C.c_float), ("reserved", C.c_int32),
                ("seed", C.c_uint64), ("step", C.c_uint64), ("T", C.c_void_p)]


class aa_route_config(C.Structure):
    _fields_ = [("score", C.c_int32), ("top_k", C.c_int32), ("n_groups", C.c_int32),
                ("top_groups", C.c_int32), ("group_best", C.c_int32), ("renormalise", C.c_int32),
                ("scale", C.c_float), ("reserved", C.c_int32)]


class aa_adamw_tensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("copy", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p),
                ("m_scale", C.c_void_p), ("v_scale", C.c_void_p), ("n", C.c_int64), ("grad_dtype", C.c_int32),
                ("copy_dtype", C.c_int32), ("state_bits", C.c_int32), ("decay", C.c_float)]


class aa_adamw_config(C.Structure):
    _fields_ = [("lr", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float),
                ("weight_decay", C.c_float), ("reserved", C.c_int32), ("seed", C.c_uint64)]


_lib = None


def lib():
    """Load the HIP library built in-tree (build with `python -m paper_1905_03381_amd.build`)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise AAError(f"{LIB_PATH} is missing: build it with paper_1905_03381_amd/build.py; "
                      "there is no CPU fallback")
    L = C.CDLL(LIB_PATH)
    vp, i32, i64, u64, f32, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64, C.c_float, C.c_size_t
    FP, CP, RP = C.POINTER(aa_features), C.POINTER(aa_step_config), C.POINTER(aa_route_config)
    TP, AP = C.POINTER(aa_adamw_tensor), C.POINTER(aa_adamw_config)
    sig = {
        "aa_version": (i32, []),
        "aa_status_string": (C.c_char_p, [i32]),
        "aa_workspace_bytes": (sz, [i32, i32]),
        "aa_workspace_init": (i32, [vp, sz, vp]),
        "aa_profile_hook": (i32, [vp, vp]),
        "aa_profile_hooks": (i32, [vp, vp, i32]),
        "aa_assistant_score": (i32, [FP, vp, i32, vp, vp, vp, vp, vp]),
        "aa_shrink": (i32, [vp, i32, f32, u64, u64, vp, vp, vp, vp, sz, vp]),
        "aa_score_shrink": (i32, [FP, vp, i32, vp, vp, f32, u64, u64, vp, vp, vp, vp, vp, vp, sz, vp]),
        "aa_shrink_threshold": (i32, [vp, i32, vp, vp, vp, vp, vp, sz, vp]),
        "aa_gather": (i32, [vp, i64, vp, vp, vp, i32, vp, vp, vp]),
        "aa_gather_csr": (i32, [FP, vp, vp, vp, i32, vp, vp, vp, i64, vp, sz, vp]),
        "aa_svm_sgd_step": (i32, [FP, vp, vp, vp, i32, vp, f32, f32, f32, vp, vp, sz, vp]),
        "aa_assistant_update": (i32, [FP, vp, vp, i32, vp, vp, vp, vp, f32, f32, vp, sz, vp]),
        "aa_boss_assistant_step": (i32, [FP, vp, vp, vp, i32, vp, vp, vp, CP, vp, vp, sz, vp]),
        "aa_fused_step": (i32, [FP, vp, vp, i32, vp, vp, vp, CP, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
        "aa_static_scratch_bytes": (sz, []),
        "aa_fused_step_static": (i32, [FP, vp, vp, i32, vp, vp, vp, CP, vp, vp, vp, vp, vp, vp, vp, vp]),
        "aa_sk_step": (i32, [FP, vp, vp, i32, vp, vp, f32, f32, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
        "aa_train_epoch": (i32, [FP, vp, vp, i64, i32, vp, vp, vp, CP, vp, vp, vp, vp, vp, sz, vp]),
        "aa_sk_epoch": (i32, [FP, vp, vp, i64, i32, vp, vp, f32, f32, vp, vp, vp, vp, vp, sz, vp]),
        "aa_threshold_update": (i32, [vp, vp, i32, f32, vp, vp, vp]),
        "aa_threshold_assistant_update": (i32, [FP, vp, vp, i32, vp, f32, vp, vp, vp, vp, f32, f32, vp, sz, vp]),
        "aa_pipeline_workspace_bytes": (sz, [i32, i32, i32]),
        "aa_train_epoch_stale": (i32, [FP, vp, vp, i64, i32, i32, vp, vp, vp, CP, vp, vp, vp, vp, sz, vp, vp]),
        "aa_bucket_batches": (i32, [vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, vp, vp, sz, vp]),
        "aa_expert_workspace_bytes": (sz, [i32, i32, i32]),
        "aa_route": (i32, [vp, i32, i64, vp, i32, i32, vp, RP, vp, vp, vp, vp, vp, vp, sz, vp]),
        "aa_route_grad": (i32, [vp, i32, i64, vp, i32, i32, RP, vp, vp, vp, i64, vp]),
        "aa_expert_plan": (i32, [vp, vp, i32, i32, i32, vp, vp, vp, vp, sz, vp]),
        "aa_expert_forward": (i32, [vp, i32, i64, vp, i32, vp, i32, i32, i32, i32, vp, i32, vp, i64, vp, i64, vp]),
        "aa_expert_grad_input": (i32, [vp, i32, i64, vp, i32, i32, i32, i32, vp, i32, vp, i64, vp, i64, vp]),
        "aa_expert_grad_weight": (i32, [vp, i32, i64, vp, i64, vp, i32, vp, i32, i32, i32, i32, vp, i32, i32, vp,
                                        sz, vp]),
        "aa_expert_combine": (i32, [vp, i32, i64, vp, vp, vp, i32, i32, i32, vp, i64, f32, u64, u64, vp, i64, vp]),
        "aa_expert_combine_grad": (i32, [vp, i32, i64, vp, i64, vp, vp, vp, i32, i32, i32, f32, u64, u64, vp, i64,
                                         vp, vp]),
        "aa_dropout": (i32, [vp, i32, i64, vp, i32, i32, vp, i64, f32, u64, u64, vp, i64, vp]),
        "aa_layer_workspace_bytes": (sz, [i32]),
        "aa_layer_norm": (i32, [vp, i32, i64, vp, i32, i32, vp, vp, f32, vp, i64, vp, vp, vp]),
        "aa_layer_norm_grad": (i32, [vp, i32, i64, vp, i64, vp, i32, i32, vp, vp, vp, vp, i64, vp, i64, vp, vp, i32,
                                     vp, sz, vp]),
        "aa_linear": (i32, [vp, i32, i64, vp, i32, i32, i32, vp, vp, i32, vp, i64, vp, i64, vp, i64, vp]),
        "aa_linear_grad": (i32, [vp, i32, i64, vp, i32, i32, i32, vp, i64, vp, i64, vp, i32, vp, sz, vp]),
        "aa_balance": (i32, [vp, i32, i64, vp, i32, i32, RP, vp, f32, f32, vp, vp, vp, vp, sz, vp]),
        "aa_balance_grad": (i32, [vp, i32, i64, vp, i32, i32, RP, vp, vp, vp, f32, f32, vp, vp, i64, vp]),
        "aa_adamw_chunks": (i64, [TP, i32]),
        "aa_adamw_table_bytes": (sz, [i32, i64]),
        "aa_adamw_table": (i32, [TP, i32, vp, sz, vp]),
        "aa_grad_norm": (i32, [vp, sz, i32, i64, f32, vp, vp, vp]),
        "aa_adamw_step": (i32, [vp, sz, i32, i64, AP, vp, vp, vp, vp, vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)
        fn.restype, fn.argtypes = res, args
    _lib = L
    return L


def status_string(rc):
    return lib().aa_status_string(rc).decode()


def _check(rc, what):
    if rc != AA_OK:
        raise AAError(f"{what}: {status_string(rc)} ({rc})")


def _ptr(t):
    return None if t is None else t.data_ptr()


# The handle itself, as torch's own generated code asks for it: building the Stream object around it
# took 2.8 us of the 11.4 us a fused_step call spends on the host, this 0.2 us.  Both names are
# private to torch: one that lacks them is asked for the Stream object.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream():
    if _raw_stream is None or _device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_device())


class Features:
    """Device feature matrix handle: Features.dense(x[, d]) or Features.csr(rowptr, col, val, d)."""

    def __init__(self, c, keep):
        self.c, self._keep = c, keep

    @classmethod
    def dense(cls, x, d=None):
        assert x.is_cuda and x.dtype == torch.float32 and x.dim() == 2 and x.stride(1) == 1
        c = aa_features(AA_DENSE, x.shape[1] if d is None else d, x.shape[0], x.data_ptr(),
                        x.stride(0), None, None, None)
        return cls(c, [x])

    @classmethod
    def csr(cls, rowptr, col, val, d):
        assert rowptr.is_cuda and rowptr.dtype == torch.int64 and col.dtype == torch.int32
        assert val is None or val.dtype == torch.float32
        c = aa_features(AA_CSR, d, rowptr.shape[0] - 1, None, 0, rowptr.data_ptr(),
                        col.data_ptr(), _ptr(val))
        return cls(c, [rowptr, col, val])

    @property
    def d(self):
        return self.c.d

    def ref(self):
        return C.byref(self.c)


class Workspace:
    """Device scratch for pools up to P_max candidates and d_max features."""

    def __init__(self, P_max, d_max, device="cuda", staleness=None):
        """staleness: size the workspace for aa_train_epoch_stale with up to that staleness."""
        if staleness is None:
            self.bytes = int(lib().aa_workspace_bytes(P_max, d_max))
        else:
            self.bytes = int(lib().aa_pipeline_workspace_bytes(P_max, d_max, staleness))
        self.buf = torch.empty(self.bytes + 256, dtype=torch.uint8, device=device)
        off = (-self.buf.data_ptr()) % 256
        self.ptr = self.buf.data_ptr() + off
        _check(lib().aa_workspace_init(self.ptr, self.bytes, _stream()), "aa_workspace_init")


def step_config(gamma, lam, lr, lr_a, l2_a, seed, step, T):
    """T: 1-element float32 CUDA tensor (device scalar).  The returned structure holds a
    reference to it, so the address stays valid as long as the configuration lives."""
    cfg = aa_step_config(gamma, lam, lr, lr_a, l2_a, 0, seed, step, T.data_ptr())
    cfg._threshold = T
    return cfg


def version():
    return int(lib().aa_version())


def workspace_bytes(P_max, d_max):
    return int(lib().aa_workspace_bytes(P_max, d_max))


def profile_hook(event_before, event_after):
    """Raw hipEvent_t handles (ints) or two Nones to disarm."""
    _check(lib().aa_profile_hook(event_before, event_after), "aa_profile_hook")


def profile_hooks(events_before, events_after):
    """Lists of raw hipEvent_t handles: pair i receives the start and stop time stamps of the i-th
    row-pass launch from now on.
    Returns the two ctypes arrays, which the caller keeps alive until those launches are issued."""
    n = len(events_before)
    assert n == len(events_after)
    arr_b = (C.c_void_p * max(n, 1))(*events_before)
    arr_a = (C.c_void_p * max(n, 1))(*events_after)
    _check(lib().aa_profile_hooks(arr_b, arr_a, n), "aa_profile_hooks")
    return arr_b, arr_a


def assistant_score(F, idx, P, phi, bias, logit, prob):
    _check(lib().aa_assistant_score(F.ref(), _ptr(idx), P, _ptr(phi), _ptr(bias), _ptr(logit),
                                    _ptr(prob), _stream()), "aa_assistant_score")


def shrink(prob, P, gamma, seed, step, keep, kept_pos, kept_count, ws):
    _check(lib().aa_shrink(_ptr(prob), P, gamma, seed, step, _ptr(keep), _ptr(kept_pos),
                           _ptr(kept_count), ws.ptr, ws.bytes, _stream()), "aa_shrink")


def shrink_threshold(crit, P, T, keep, kept_pos, kept_count, ws):
    _check(lib().aa_shrink_threshold(_ptr(crit), P, _ptr(T), _ptr(keep), _ptr(kept_pos),
                                     _ptr(kept_count), ws.ptr, ws.bytes, _stream()),
           "aa_shrink_threshold")


def score_shrink(F, idx, P, phi, bias, gamma, seed, step, logit, prob, keep, kept_pos, kept_count,
                 ws):
    _check(lib().aa_score_shrink(F.ref(), _ptr(idx), P, _ptr(phi), _ptr(bias), gamma, seed, step,
                                 _ptr(logit), _ptr(prob), _ptr(keep), _ptr(kept_pos),
                                 _ptr(kept_count), ws.ptr, ws.bytes, _stream()), "aa_score_shrink")


def gather(src, row_bytes, idx, kept_pos, kept_count, max_rows, dst, kept_ids):
    _check(lib().aa_gather(_ptr(src), row_bytes, _ptr(idx), _ptr(kept_pos), _ptr(kept_count),
                           max_rows, _ptr(dst), _ptr(kept_ids), _stream()), "aa_gather")


def gather_csr(F, idx, kept_pos, kept_count, max_rows, out_rowptr, out_col, out_val, out_nnz_cap,
               ws):
    _check(lib().aa_gather_csr(F.ref(), _ptr(idx), _ptr(kept_pos), _ptr(kept_count), max_rows,
                               _ptr(out_rowptr), _ptr(out_col), _ptr(out_val), out_nnz_cap,
                               ws.ptr, ws.bytes, _stream()), "aa_gather_csr")


def svm_sgd_step(F, y, rows, m_dev, m_max, w, lam, lr, radius, loss, ws):
    _check(lib().aa_svm_sgd_step(F.ref(), _ptr(y), _ptr(rows), _ptr(m_dev), m_max, _ptr(w), lam,
                                 lr, radius, _ptr(loss), ws.ptr, ws.bytes, _stream()),
           "aa_svm_sgd_step")


def assistant_update(F, rows, m_dev, m_max, loss, T, phi, bias, lr_a, l2_a, ws):
    _check(lib().aa_assistant_update(F.ref(), _ptr(rows), _ptr(m_dev), m_max, _ptr(loss), _ptr(T),
                                     _ptr(phi), _ptr(bias), lr_a, l2_a, ws.ptr, ws.bytes,
                                     _stream()), "aa_assistant_update")


def boss_assistant_step(F, y, rows, m_dev, m_max, w, phi, bias, cfg, loss, ws):
    _check(lib().aa_boss_assistant_step(F.ref(), _ptr(y), _ptr(rows), _ptr(m_dev), m_max, _ptr(w),
                                        _ptr(phi), _ptr(bias), C.byref(cfg), _ptr(loss), ws.ptr,
                                        ws.bytes, _stream()), "aa_boss_assistant_step")


def fused_step(F, y, idx, P, w, phi, bias, cfg, logit, prob, keep, kept_pos, kept_ids, loss,
               kept_count, ws):
    _check(lib().aa_fused_step(F.ref(), _ptr(y), _ptr(idx), P, _ptr(w), _ptr(phi), _ptr(bias),
                               C.byref(cfg), _ptr(logit), _ptr(prob), _ptr(keep), _ptr(kept_pos),
                               _ptr(kept_ids), _ptr(loss), _ptr(kept_count), ws.ptr, ws.bytes,
                               _stream()), "aa_fused_step")


def static_scratch_bytes():
    return int(lib().aa_static_scratch_bytes())


def fused_step_static(F, y, idx, P, w, phi, bias, cfg, logit, prob, keep, kept_pos, kept_ids, loss,
                      kept_count):
    _check(lib().aa_fused_step_static(F.ref(), _ptr(y), _ptr(idx), P, _ptr(w), _ptr(phi),
                                      _ptr(bias), C.byref(cfg), _ptr(logit), _ptr(prob), _ptr(keep),
                                      _ptr(kept_pos), _ptr(kept_ids), _ptr(loss), _ptr(kept_count),
                                      _stream()), "aa_fused_step_static")


def sk_step(F, y, idx, P, w, T, lam, lr, loss_pool, keep, kept_pos, kept_ids, loss, kept_count, ws):
    _check(lib().aa_sk_step(F.ref(), _ptr(y), _ptr(idx), P, _ptr(w), _ptr(T), lam, lr,
                            _ptr(loss_pool), _ptr(keep), _ptr(kept_pos), _ptr(kept_ids), _ptr(loss),
                            _ptr(kept_count), ws.ptr, ws.bytes, _stream()), "aa_sk_step")


def train_epoch(F, y, perm, n_perm, P, w, phi, bias, cfg, t_upd, kept_hist, ws, kept_ids_hist=None,
                loss_hist=None):
    _check(lib().aa_train_epoch(F.ref(), _ptr(y), _ptr(perm), n_perm, P, _ptr(w), _ptr(phi),
                                _ptr(bias), C.byref(cfg), _ptr(t_upd), _ptr(kept_hist),
                                _ptr(kept_ids_hist), _ptr(loss_hist), ws.ptr, ws.bytes, _stream()),
           "aa_train_epoch")


def sk_epoch(F, y, perm, n_perm, P, w, T, lam, lr0, t_upd, kept_hist, ws, kept_ids_hist=None,
             loss_hist=None):
    _check(lib().aa_sk_epoch(F.ref(), _ptr(y), _ptr(perm), n_perm, P, _ptr(w), _ptr(T), lam, lr0,
                             _ptr(t_upd), _ptr(kept_hist), _ptr(kept_ids_hist), _ptr(loss_hist),
                             ws.ptr, ws.bytes, _stream()), "aa_sk_epoch")


def train_epoch_stale(F, y, perm, n_perm, P, staleness, w, phi, bias, cfg, t_upd, kept_hist,
                      kept_ids_hist, ws, stream_gen):
    """stream_gen: a torch.cuda.Stream other than the current one (the Boss runs on the current)."""
    _check(lib().aa_train_epoch_stale(F.ref(), _ptr(y), _ptr(perm), n_perm, P, staleness, _ptr(w),
                                      _ptr(phi), _ptr(bias), C.byref(cfg), _ptr(t_upd),
                                      _ptr(kept_hist), _ptr(kept_ids_hist), ws.ptr, ws.bytes,
                                      _stream(), stream_gen.cuda_stream), "aa_train_epoch_stale")


def threshold_update(loss, m_dev, m_max, momentum, T, initialised):
    _check(lib().aa_threshold_update(_ptr(loss), _ptr(m_dev), m_max, momentum, _ptr(T),
                                     _ptr(initialised), _stream()), "aa_threshold_update")


def threshold_assistant_update(F, rows, m_dev, m_max, loss, momentum, T, initialised, phi, bias, lr_a,
                               l2_a, ws):
    _check(lib().aa_threshold_assistant_update(F.ref(), _ptr(rows), _ptr(m_dev), m_max, _ptr(loss),
                                               momentum, _ptr(T), _ptr(initialised), _ptr(phi),
                                               _ptr(bias), lr_a, l2_a, ws.ptr, ws.bytes, _stream()),
           "aa_threshold_assistant_update")


def bucket_batches(len_s, len_t, m_dev, m_max, width, n_buckets, token_budget, order, bucket_start,
                   batch_of, n_batches, ws):
    _check(lib().aa_bucket_batches(_ptr(len_s), _ptr(len_t), _ptr(m_dev), m_max, width, n_buckets,
                                   token_budget, _ptr(order), _ptr(bucket_start), _ptr(batch_of),
                                   _ptr(n_batches), ws.ptr, ws.bytes, _stream()), "aa_bucket_batches")


# ---- a Boss block of experts: routing, ragged products, combination, dropout ----
#
# Sizes, types and strides are read off the tensors: matrices are 2-d with neighbouring columns in
# neighbouring elements (any row stride), matrices of all experts are contiguous [E, rows, columns],
# index arrays are contiguous int32.


def _require(ok, what):
    if not ok:
        raise AAError(what)


# A call of a few rows takes as long as the host needs for it (about 8 us), so the checks look at each property once and
# put their messages together only where they fail.


def _matrix(t, name, dtype=None, width=None, rows=0):
    """(pointer, row stride) of a 2-d CUDA tensor of the given type, width and number of rows (at least)."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dim() == 2):
        raise AAError(f"{name}: a 2-d CUDA tensor is needed")
    n, d = t.shape
    if dtype is not None and t.dtype != dtype:
        raise AAError(f"{name}: {t.dtype} where {dtype} is needed")
    if width is not None and d != width:
        raise AAError(f"{name}: {d} columns where {width} are needed")
    if n < rows:
        raise AAError(f"{name}: {n} rows where {rows} are needed")
    ld, step = t.stride()
    if step != 1 and d > 1:
        raise AAError(f"{name}: neighbouring columns must be neighbours in memory")
    return t.data_ptr(), ld if n > 1 else d   # (a tensor of one row may state any stride)


def _array(t, name, dtype, shape=None, least=0):
    """Pointer of a contiguous CUDA tensor; None stays None."""
    if t is None:
        return None
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise AAError(f"{name}: a contiguous {dtype} CUDA tensor is needed")
    if shape is not None and t.shape != shape:
        raise AAError(f"{name}: shape {tuple(t.shape)}, not {tuple(shape)}")
    if least and t.numel() < least:
        raise AAError(f"{name}: {t.numel()} entries where {least} are needed")
    return t.data_ptr()


def _type(t, name, products=False):
    """The type's code; products: of 16 bits."""
    code = DTYPES.get(t.dtype) if isinstance(t, torch.Tensor) else None
    if code is None or (products and code == 0):
        raise AAError(f"{name}: its type is not one this call takes")
    return code


def _name_of(table, name, what):
    code = table.get(name) if isinstance(name, str) else None
    if code is None:
        raise AAError(f"{what}: {name!r} is none of {sorted(table)}")
    return code


def _all_weights(w, what):
    """E, rows, columns of the experts' matrices."""
    if not (isinstance(w, torch.Tensor) and w.dim() == 3):
        raise AAError(what)
    return w.shape


class ExpertWorkspace:
    """Device scratch of route / expert_plan (with a plan) and expert_grad_weight."""

    def __init__(self, n_max, top_k, n_experts, device="cuda"):
        _take(self, int(lib().aa_expert_workspace_bytes(n_max, top_k, n_experts)), device)


def _take(ws, size, device):
    """Prepared scratch of `size` bytes for the workspace object ws."""
    ws.bytes = size
    ws.buf = torch.empty(size + 256, dtype=torch.uint8, device=device)
    ws.ptr = ws.buf.data_ptr() + (-ws.buf.data_ptr()) % 256
    _check(lib().aa_workspace_init(ws.ptr, ws.bytes, _stream()), "aa_workspace_init")


def _scratch(ws, kind="an ExpertWorkspace"):
    if ws is None:
        raise AAError(f"ws: {kind} is needed")
    return ws.ptr, ws.bytes


def route_config(score, top_k, n_groups=1, top_groups=1, group_best=1, renormalise=False, scale=1.0):
    """score: "softmax" or "sigmoid"."""
    return aa_route_config(_name_of(SCORES, score, "score"), top_k, n_groups, top_groups, group_best,
                           int(bool(renormalise)), scale, 0)


def _plan_pointers(plan, n, k, n_experts):
    offsets, order, slot = plan
    _require(offsets is not None and order is not None and slot is not None, "plan: offsets, order and slot")
    return (_array(offsets, "offsets", torch.int32, (n_experts + 1,)), _array(order, "order", torch.int32, least=n * k),
            _array(slot, "slot", torch.int32, (n, k)))


def route(logits, count, bias, cfg, ids, weights, plan=None, ws=None):
    """plan: (offsets[E + 1], order[n * top_k], slot[n, top_k]) to be made in the same call; ws then an ExpertWorkspace."""
    dt = _type(logits, "logits")
    x, ld = _matrix(logits, "logits")
    n, E = logits.shape
    p = (None, None, None) if plan is None else _plan_pointers(plan, n, cfg.top_k, E)
    _check(lib().aa_route(x, dt, ld, _array(count, "count", torch.int32, least=1), n, E,
                          _array(bias, "bias", torch.float32, (E,)), C.byref(cfg),
                          _array(ids, "ids", torch.int32, (n, cfg.top_k)),
                          _array(weights, "weights", torch.float32, (n, cfg.top_k)), *p,
                          ws.ptr if ws else None, ws.bytes if ws else 0, _stream()), "aa_route")


def route_grad(logits, count, cfg, ids, dweights, dlogits):
    dt = _type(logits, "logits")
    x, ld = _matrix(logits, "logits")
    n, E = logits.shape
    out, ld_out = _matrix(dlogits, "dlogits", logits.dtype, E, n)
    _check(lib().aa_route_grad(x, dt, ld, _array(count, "count", torch.int32, least=1), n, E, C.byref(cfg),
                               _array(ids, "ids", torch.int32, (n, cfg.top_k)),
                               _array(dweights, "dweights", torch.float32, (n, cfg.top_k)), out, ld_out,
                               _stream()), "aa_route_grad")


def expert_plan(ids, count, n_experts, offsets, order, slot, ws):
    _require(isinstance(ids, torch.Tensor) and ids.dim() == 2, "ids: a 2-d tensor")
    n, k = ids.shape
    p = _plan_pointers((offsets, order, slot), n, k, n_experts)
    _check(lib().aa_expert_plan(_array(ids, "ids", torch.int32), _array(count, "count", torch.int32, least=1), n, k,
                                n_experts, *p, *_scratch(ws), _stream()), "aa_expert_plan")


def _grouped_rows(x, order, top_k, rows, name):
    """Rows that a product over `rows` places may read must be there."""
    n = x.shape[0]
    if order is None:
        if n < rows:
            raise AAError(f"{name}: {n} rows where {rows} are needed")
        return None
    if top_k < 1 or n * top_k < rows:
        raise AAError(f"{name}: {n} rows for {rows} pairs")
    return _array(order, "order", torch.int32, None, rows)


def expert_forward(x, order, top_k, offsets, w, act, out, pre=None):
    """Places 0 .. out.shape[0] - 1 at most; order None: place q reads row q of x (top_k is then not used)."""
    dt, a = _type(x, "x", True), _name_of(ACTIVATIONS, act, "act")
    E, d_out, d_in = _all_weights(w, "w: [E, rows, d_in]")
    if a == 2:
        _require(d_out % 2 == 0, "w: [E, rows, d_in]")
        d_out //= 2
    dtype = x.dtype
    xp, ldx = _matrix(x, "x", None, d_in)
    op, ldo = _matrix(out, "out", dtype, d_out)
    rows = out.shape[0]
    pp, ldp = (None, 0) if pre is None else _matrix(pre, "pre", dtype, 2 * d_out, rows)
    ordp = _grouped_rows(x, order, top_k, rows, "x")
    _check(lib().aa_expert_forward(xp, dt, ldx, ordp, top_k, _array(offsets, "offsets", torch.int32, (E + 1,)), rows, E,
                                   d_in, d_out, _array(w, "w", dtype), a, op, ldo, pp, ldp, _stream()),
           "aa_expert_forward")


def expert_grad_input(dout, offsets, w, act, saved, dx):
    dt, a = _type(dout, "dout", True), _name_of(ACTIVATIONS, act, "act")
    E, d_out, d_in = _all_weights(w, "w: [E, d_out, d_in]")
    dtype, wide = dout.dtype, 2 * d_in if a == 2 else d_in
    xp, ldx = _matrix(dx, "dx", dtype, wide)
    rows = dx.shape[0]
    gp, ldg = _matrix(dout, "dout", None, d_out, rows)
    sp, lds = (None, 0) if a == 0 else _matrix(saved, "saved", dtype, wide, rows)
    _check(lib().aa_expert_grad_input(gp, dt, ldg, _array(offsets, "offsets", torch.int32, (E + 1,)), rows, E, d_in,
                                      d_out, _array(w, "w", dtype), a, sp, lds, xp, ldx, _stream()),
           "aa_expert_grad_input")


def expert_grad_weight(dout, x, order, top_k, offsets, dw, accumulate, ws):
    dt = _type(dout, "dout", True)
    E, d_out, d_in = _all_weights(dw, "dw: [E, d_out, d_in] of dout's type or float32")
    _require(dw.dtype in (dout.dtype, torch.float32), "dw: [E, d_out, d_in] of dout's type or float32")
    gp, ldg = _matrix(dout, "dout", None, d_out)
    rows = dout.shape[0]
    xp, ldx = _matrix(x, "x", dout.dtype, d_in)
    ordp = _grouped_rows(x, order, top_k, rows, "x")
    _check(lib().aa_expert_grad_weight(gp, dt, ldg, xp, ldx, ordp, top_k,
                                       _array(offsets, "offsets", torch.int32, (E + 1,)), rows, E, d_in, d_out,
                                       _array(dw, "dw", dw.dtype), DTYPES[dw.dtype], int(bool(accumulate)),
                                       *_scratch(ws), _stream()), "aa_expert_grad_weight")


def dropout(x, count, residual, p, seed, step, out):
    dt = _type(x, "x")
    xp, ldx = _matrix(x, "x")
    n, d = x.shape
    rp, ldr = (None, 0) if residual is None else _matrix(residual, "residual", x.dtype, d, n)
    op, ldo = _matrix(out, "out", x.dtype, d, n)
    _check(lib().aa_dropout(xp, dt, ldx, _array(count, "count", torch.int32, least=1), n, d, rp, ldr, p, seed, step,
                            op, ldo, _stream()), "aa_dropout")


def expert_combine(y, slot, weights, count, residual, p, seed, step, out):
    dt = _type(y, "y")
    _require(isinstance(slot, torch.Tensor) and slot.dim() == 2, "slot: a 2-d tensor")
    n, k = slot.shape
    yp, ldy = _matrix(y, "y")
    d = y.shape[1]
    rp, ldr = (None, 0) if residual is None else _matrix(residual, "residual", y.dtype, d, n)
    op, ldo = _matrix(out, "out", y.dtype, d, n)
    _check(lib().aa_expert_combine(yp, dt, ldy, _array(slot, "slot", torch.int32),
                                   _array(weights, "weights", torch.float32, (n, k)),
                                   _array(count, "count", torch.int32, least=1), n, k, d, rp, ldr, p, seed, step, op,
                                   ldo, _stream()), "aa_expert_combine")


def expert_combine_grad(dout, y, slot, weights, count, p, seed, step, dy, dweights):
    """y is only read for dweights: both may be None."""
    dt = _type(dout, "dout")
    _require(isinstance(slot, torch.Tensor) and slot.dim() == 2, "slot: a 2-d tensor")
    n, k = slot.shape
    gp, ldg = _matrix(dout, "dout", rows=n)
    d = dout.shape[1]
    _require(y is not None or dweights is None, "y: needed for dweights")
    yp, ldy = (None, d) if y is None else _matrix(y, "y", dout.dtype, d)
    dyp, lddy = _matrix(dy, "dy", dout.dtype, d)
    _check(lib().aa_expert_combine_grad(gp, dt, ldg, yp, ldy, _array(slot, "slot", torch.int32),
                                        _array(weights, "weights", torch.float32, (n, k)),
                                        _array(count, "count", torch.int32, least=1), n, k, d, p, seed, step, dyp, lddy,
                                        _array(dweights, "dweights", torch.float32, (n, k)), _stream()),
           "aa_expert_combine_grad")


# ---- around a Boss block of experts: layer norm, dense product, balance loss, optimizer ----


class LayerWorkspace:
    """Device scratch of layer_norm_grad, linear_grad and balance for rows of up to d_max columns (gated layers: twice d_out;
    balance: the experts)."""

    def __init__(self, d_max, device="cuda"):
        _take(self, int(lib().aa_layer_workspace_bytes(d_max)), device)


_current = _device or torch.cuda.current_device
_stream_on = _raw_stream or (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _here(t, name, device):
    """A GPU tensor is on the device that the call's stream is of."""
    if isinstance(t, torch.Tensor) and t.is_cuda and t.get_device() != device:
        raise AAError(f"{name}: on device {t.get_device()}, the call's is {device}")


def _flat(t, name, device, dtype, shape=None, least=0):
    """_array of a tensor on the call's device."""
    if t is None:
        return None
    _here(t, name, device)
    return _array(t, name, dtype, shape, least)


def _layer_scratch(ws, device):
    scratch = _scratch(ws, "a LayerWorkspace")
    _here(ws.buf, "ws", device)
    return scratch


# (Calls of a row or a few take as long as the host: each of these asks a tensor for six things where _matrix and _array ask for
# ten.  What is unusual goes to those, for their messages.)
_F32, _I32, _Tensor = torch.float32, torch.int32, torch.Tensor


def _scalar(t, name, device, dtype=_F32):
    """Pointer of one value; None stays None."""
    if t is None:
        return None
    if type(t) is _Tensor and t.dtype is dtype and t.get_device() == device and t.shape == (1,):
        return t.data_ptr()
    return _flat(t, name, device, dtype, least=1)


def _count(count, device):
    return _scalar(count, "count", device, _I32)


def _vector(t, name, device, n):
    """Pointer of n neighbouring float32 values; None stays None."""
    if t is None:
        return None
    if type(t) is _Tensor and t.dtype is _F32 and t.get_device() == device and t.shape == (n,) and t.is_contiguous():
        return t.data_ptr()
    return _flat(t, name, device, _F32, (n,))


def _rows_like(t, name, device, dtype, n, d):
    """(pointer, row stride) of n rows of d neighbouring columns of the given type (or more rows)."""
    if type(t) is _Tensor and t.dtype is dtype and t.get_device() == device and t.shape == (n, d):
        ld, step = t.stride()
        if step == 1:
            return t.data_ptr(), ld if n > 1 else d
    _here(t, name, device)
    return _matrix(t, name, dtype, d, n)


def _first_rows(t, name, types):
    """(device, type code, pointer, row stride, rows, columns) of the matrix that a call's device, sizes and type come from."""
    if type(t) is _Tensor and t.is_cuda and t.dim() == 2:
        device, code = _current(), types.get(t.dtype)
        n, d = t.shape
        ld, step = t.stride()
        if code is not None and step == 1 and t.get_device() == device:
            return device, code, t.data_ptr(), ld if n > 1 else d, n, d
        _here(t, name, device)
    code = _type(t, name, types is _HALVES)
    p, ld = _matrix(t, name)
    device = _current()
    _here(t, name, device)
    return device, code, p, ld, t.shape[0], t.shape[1]


_HALVES = {t: c for t, c in DTYPES.items() if t is not _F32}


def layer_norm(x, gamma, beta, eps, count, out, mean=None, rstd=None):
    """gamma, beta: float32 [d] or None (1 and 0); mean, rstd: float32 [n], for the backward pass."""
    dev, dt, xp, ldx, n, d = _first_rows(x, "x", DTYPES)
    op, ldo = _rows_like(out, "out", dev, x.dtype, n, d)
    _check(lib().aa_layer_norm(xp, dt, ldx, _count(count, dev), n, d, _vector(gamma, "gamma", dev, d),
                               _vector(beta, "beta", dev, d), eps, op, ldo, _vector(mean, "mean", dev, n),
                               _vector(rstd, "rstd", dev, n), _stream_on(dev)), "aa_layer_norm")


def layer_norm_grad(dout, x, gamma, mean, rstd, residual, count, dx, dgamma, dbeta, accumulate, ws):
    """residual: what is added to dx, or None; dgamma, dbeta: either may be None, and ws where both are."""
    dev, dt, gp, ldg, n, d = _first_rows(dout, "dout", DTYPES)
    xp, ldx = _rows_like(x, "x", dev, dout.dtype, n, d)
    rp, ldr = (None, 0) if residual is None else _rows_like(residual, "residual", dev, dout.dtype, n, d)
    op, ldo = _rows_like(dx, "dx", dev, dout.dtype, n, d)
    scratch = (None, 0) if dgamma is None and dbeta is None else _layer_scratch(ws, dev)
    _check(lib().aa_layer_norm_grad(gp, dt, ldg, xp, ldx, _count(count, dev), n, d,
                                    _vector(gamma, "gamma", dev, d), _vector(mean, "mean", dev, n),
                                    _vector(rstd, "rstd", dev, n), rp, ldr, op, ldo,
                                    _vector(dgamma, "dgamma", dev, d), _vector(dbeta, "dbeta", dev, d),
                                    int(bool(accumulate)), *scratch, _stream_on(dev)), "aa_layer_norm_grad")


def linear(x, w, bias, act, residual, count, out, pre=None):
    """w [d_out, d_in] (gated: [2 d_out, d_in]) and bias (float32, or None) for all rows; pre: what the activation is taken
    of, for the backward pass."""
    a = _name_of(DENSE_ACTIVATIONS, act, "act")
    dev, dt, xp, ldx, n, d_in = _first_rows(x, "x", _HALVES)
    _require(isinstance(w, torch.Tensor) and w.dim() == 2 and w.shape[1] == d_in, "w: [rows, d_in]")
    wide, dtype = w.shape[0], x.dtype
    _require(a != 2 or wide % 2 == 0, "w: [rows, d_in]")
    d_out = wide // 2 if a == 2 else wide
    op, ldo = _rows_like(out, "out", dev, dtype, n, d_out)
    rp, ldr = (None, 0) if residual is None else _rows_like(residual, "residual", dev, dtype, n, d_out)
    pp, ldp = (None, 0) if pre is None else _rows_like(pre, "pre", dev, dtype, n, wide)
    _check(lib().aa_linear(xp, dt, ldx, _count(count, dev), n, d_in, d_out, _flat(w, "w", dev, dtype),
                           _vector(bias, "bias", dev, wide), a, rp, ldr, op, ldo, pp, ldp, _stream_on(dev)),
           "aa_linear")


def linear_grad(dout, act, pre, count, dpre, dbias, accumulate, ws):
    """pre: not needed without an activation; dpre or dbias may be None, and ws where dbias is."""
    a = _name_of(DENSE_ACTIVATIONS, act, "act")
    dev, dt, gp, ldg, n, d = _first_rows(dout, "dout", _HALVES)
    dtype = dout.dtype
    wide = 2 * d if a == 2 else d
    pp, ldp = (None, 0) if a == 0 else _rows_like(pre, "pre", dev, dtype, n, wide)
    op, ldo = (None, 0) if dpre is None else _rows_like(dpre, "dpre", dev, dtype, n, wide)
    scratch = (None, 0) if dbias is None else _layer_scratch(ws, dev)
    _check(lib().aa_linear_grad(gp, dt, ldg, _count(count, dev), n, d, a, pp, ldp, op, ldo,
                                _vector(dbias, "dbias", dev, wide), int(bool(accumulate)), *scratch,
                                _stream_on(dev)), "aa_linear_grad")


def balance(logits, count, cfg, ids, coef, z_coef, counts, share, loss, ws):
    """counts: int32 [E]; share: float32 [E] or None; loss: float32 [2] or None; ws: a LayerWorkspace of E columns."""
    dev, dt, x, ld, n, E = _first_rows(logits, "logits", DTYPES)
    _require(counts is not None, "counts: needed")
    _check(lib().aa_balance(x, dt, ld, _count(count, dev), n, E, C.byref(cfg),
                            _flat(ids, "ids", dev, torch.int32, (n, cfg.top_k)), coef, z_coef,
                            _flat(counts, "counts", dev, torch.int32, (E,)), _vector(share, "share", dev, E), _vector(loss, "loss", dev, 2),
                            *_layer_scratch(ws, dev), _stream_on(dev)), "aa_balance")


def balance_grad(logits, count, cfg, ids, dweights, counts, coef, z_coef, dloss, dlogits):
    """dweights None: the balance loss alone (ids is then not read and may be None); dloss: a float32 tensor of one, or None."""
    dev, dt, x, ld, n, E = _first_rows(logits, "logits", DTYPES)
    out, ld_out = _rows_like(dlogits, "dlogits", dev, logits.dtype, n, E)
    _check(lib().aa_balance_grad(x, dt, ld, _count(count, dev), n, E, C.byref(cfg),
                                 _flat(ids, "ids", dev, torch.int32, (n, cfg.top_k)),
                                 _flat(dweights, "dweights", dev, torch.float32, (n, cfg.top_k)),
                                 _flat(counts, "counts", dev, torch.int32, (E,)), coef, z_coef,
                                 _flat(dloss, "dloss", dev, torch.float32, least=1), out, ld_out, _stream_on(dev)),
           "aa_balance_grad")


STATE_BLOCK = 256   # AA_STATE_BLOCK


def adamw_tensor(param, grad, m, v, copy=None, m_scale=None, v_scale=None, decay=1.0):
    """One tensor of an update.  param float32, grad of any of the three types, copy bfloat16 or float16; all of the same number of
    elements, contiguous.  m, v: float32, or float8_e4m3fn with m_scale, v_scale float32 (one for 256 neighbours)."""
    _require(isinstance(param, torch.Tensor), "param: a tensor")
    n, bits8 = param.numel(), isinstance(m, torch.Tensor) and m.dtype == torch.float8_e4m3fn
    code = _type(grad, "grad")
    state, device = torch.float8_e4m3fn if bits8 else torch.float32, param.get_device()

    def flat(t, name, dtype, size=n):
        p = _flat(t, name, device, dtype)
        _require(p is not None and t.numel() == size, f"{name}: {size} elements are needed")
        return p

    copy_code = 0 if copy is None else _type(copy, "copy", products=True)
    blocks = -(-n // STATE_BLOCK)
    out = aa_adamw_tensor(
        flat(param, "param", torch.float32), flat(grad, "grad", grad.dtype),
        None if copy is None else flat(copy, "copy", copy.dtype), flat(m, "m", state), flat(v, "v", state),
        flat(m_scale, "m_scale", torch.float32, blocks) if bits8 else None,
        flat(v_scale, "v_scale", torch.float32, blocks) if bits8 else None,
        n, code, copy_code, 8 if bits8 else 32, decay)
    out._tensors = (param, grad, copy, m, v, m_scale, v_scale)
    return out


class AdamWTable:
    """The tensors of an optimizer's steps, listed on the device once.  Holds references to them: they stay where they are."""

    def __init__(self, tensors, device="cuda"):
        self._tensors = [t._tensors for t in tensors]
        self.n = len(tensors)
        _require(self.n > 0, "tensors: at least one")
        listed = (aa_adamw_tensor * self.n)(*tensors)
        self.chunks = int(lib().aa_adamw_chunks(listed, self.n))
        _check(min(self.chunks, 0), "aa_adamw_chunks")
        self.bytes = int(lib().aa_adamw_table_bytes(self.n, self.chunks))
        self.buf = torch.empty(self.bytes + 256, dtype=torch.uint8, device=device)
        self.ptr = self.buf.data_ptr() + (-self.buf.data_ptr()) % 256
        dev = self.device = _current()
        for t in [self.buf] + [t[0] for t in self._tensors]:
            _here(t, "tensors", dev)
        _check(lib().aa_adamw_table(listed, self.n, self.ptr, self.bytes, _stream_on(dev)), "aa_adamw_table")


def adamw_config(lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, seed=0):
    return aa_adamw_config(lr, beta1, beta2, eps, weight_decay, 0, seed)


def grad_norm(table, max_norm, scale, out):
    """out: float32 [2], the norm of all gradients and the factor for adamw_step; scale: a float32 tensor of one, or None."""
    _require(out is not None, "out: needed")
    dev = _current()
    _require(table.device == dev, "table: on another device than the current one")
    _check(lib().aa_grad_norm(table.ptr, table.bytes, table.n, table.chunks, max_norm, _scalar(scale, "scale", dev),
                              _flat(out, "out", dev, torch.float32, least=2), _stream_on(dev)), "aa_grad_norm")


def adamw_step(table, cfg, lr_factor, grad_factor, count, t):
    """lr_factor, grad_factor: float32 tensors of one, or None (1); count: an int32 tensor of one, or None; t: the int32 tensor of
    one that counts the updates."""
    _require(t is not None, "t: needed")
    dev = _current()
    _require(table.device == dev, "table: on another device than the current one")
    _check(lib().aa_adamw_step(table.ptr, table.bytes, table.n, table.chunks, C.byref(cfg),
                               _scalar(lr_factor, "lr_factor", dev), _scalar(grad_factor, "grad_factor", dev), _count(count, dev),
                               _scalar(t, "t", dev, torch.int32), _stream_on(dev)), "aa_adamw_step")
