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
        self.bytes = int(lib().aa_expert_workspace_bytes(n_max, top_k, n_experts))
        self.buf = torch.empty(self.bytes + 256, dtype=torch.uint8, device=device)
        self.ptr = self.buf.data_ptr() + (-self.buf.data_ptr()) % 256
        _check(lib().aa_workspace_init(self.ptr, self.bytes, _stream()), "aa_workspace_init")


def _scratch(ws):
    if ws is None:
        raise AAError("ws: an ExpertWorkspace is needed")
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
