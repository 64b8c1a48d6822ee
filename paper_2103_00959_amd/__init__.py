"""MI355X-native GNN message-passing operators of the CogDL paper (arxiv 2103.00959, section 2.2).

Thin ctypes binding over ``libcogdl_mi355.so`` (see ``include/cogdl.h``):
argument marshalling only.  Every step runs in the library's HIP kernels on
the current torch stream; torch is used for device memory and streams.  The
binding fails loudly when the library or a GPU is missing: there is no CPU
fallback.

    spmm(rowptr, col, val, X, plan=None, out_dtype=None)          -> Y = A X
    gspmm(rowptr, col, val, X, reduce, compute=..., ...)          -> Eq. 1 with sum/mean/max, mul/add/sub/copy
    csr_to_csc(rowptr, col, val, n_cols)                          -> colptr, row_t, val_t, perm
    spmm_t(colptr, row_t, val_t, G, plan_t=None, out_dtype=None)  -> dX = A^T G
    sddmm_edge_softmax(rowptr, col, s_dst, s_src, slope, plan)    -> alpha [nnz, H]
    gat_aggregate(rowptr, col, s_dst, s_src, X, slope, ...)       -> Y [n, H, D] (, alpha)
    sddmm_dot(rowptr, col, P, Q)                                  -> <P[i,h], Q[j,h]> per edge
    gat_backward(rowptr, col, colptr, row_t, perm, ..., dY)       -> dX, dalpha, dscore, ds_dst, ds_src
    linear(X, W, bias, act)                                       -> Y = act(X W^T + b)
    grouped_linear(X, W, offsets, bias, act, save=False)          -> Y, rows of group g by W[g] (, checkpoint of X)
    grouped_linear_backward(dY, W, offsets, X | codes, exps, ...) -> dX, dW, db
    act_checkpoint(A) / act_restore(codes, exps)                  -> activations in 8 bits and back
    embedding(table, index, scale)                                -> Y = scale table[index]
    embedding_backward(dY, index, V, scale)                       -> the table's gradient, by sorted tokens
    linear_cross_entropy(X, W, target, bias)                      -> loss, lse of the logits X W^T + b, never kept
    linear_cross_entropy_backward(dloss, X, W, target, loss, lse) -> dX, dW, db
    linear_distill(X, W, index, teacher, bias, temperature)       -> loss, lse, logp against a teacher's top logits
    linear_distill_backward(dloss, X, W, index, teacher, ...)     -> dX, dW, db
    Plan(rowptr, nnz, max_feat, max_heads, mode, group_size)      -> the workload balancer
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import operator
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libcogdl_mi355.so")

COGDL_F32, COGDL_BF16, COGDL_F16 = 0, 1, 2
BALANCE = {"auto": 0, "row_split": 1, "neighbor_group": 2}
MODE_NAMES = {1: "row_split", 2: "neighbor_group"}
MAX_HEADS = 64
MAX_NNZ = 2**31 - 4097     # COGDL_MAX_NNZ: int32 edge ids with room for one batch past the end

_lib = None


class CogdlError(RuntimeError):
    pass


class _PlanInfo(ctypes.Structure):
    _fields_ = [("n_rows", ctypes.c_int32), ("nnz", ctypes.c_int64), ("group_size", ctypes.c_int32),
                ("max_feat", ctypes.c_int32), ("max_heads", ctypes.c_int32), ("mode", ctypes.c_int32),
                ("n_units", ctypes.c_int32), ("n_long_units", ctypes.c_int32),
                ("n_split_rows", ctypes.c_int32),
                ("n_partials", ctypes.c_int32), ("device_bytes", ctypes.c_int64)]


def lib():
    """Load the HIP library (after torch, so both share one HIP runtime)."""
    global _lib
    if _lib is not None:
        return _lib
    import torch  # noqa: F401  (loads the HIP runtime the library binds to)
    if not os.path.exists(LIB_PATH):
        raise CogdlError(f"{LIB_PATH} is missing: build it with `python -m paper_2103_00959_amd.build`")
    L = ctypes.CDLL(LIB_PATH)
    P, i32, i64, f32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
    L.cogdl_status_string.restype = ctypes.c_char_p
    L.cogdl_status_string.argtypes = [ctypes.c_int]
    L.cogdl_version.restype = i32
    L.cogdl_plan_create.argtypes = [i32, i64, P, i32, i32, ctypes.c_int, i32, P, ctypes.POINTER(P)]
    L.cogdl_plan_rebuild.argtypes = [P, P, P]
    L.cogdl_plan_create_sliced.argtypes = [i32, i64, P, P, i32, i32, i32, ctypes.c_int, i32, i32, P,
                                           ctypes.POINTER(P)]
    L.cogdl_plan_rebuild_sliced.argtypes = [P, P, P, P]
    L.cogdl_plan_destroy.argtypes = [P]
    L.cogdl_plan_query.argtypes = [P, P, ctypes.POINTER(_PlanInfo)]
    L.cogdl_plan_units.argtypes = [P, P, i64, P]
    L.cogdl_spmm.argtypes = [i32, i32, i64, P, P, P, i32, P, ctypes.c_int, P, ctypes.c_int, P, P]
    L.cogdl_gspmm.argtypes = [i32, i32, i64, P, P, P, i32, P, ctypes.c_int, P, ctypes.c_int,
                              ctypes.c_int, ctypes.c_int, P, ctypes.c_int, P, P, P]
    L.cogdl_gat_aggregate_act.argtypes = [i32, i32, i64, P, P, i32, i32, P, P, f32, P, P,
                                          ctypes.c_int, P, ctypes.c_int, P, P, ctypes.c_int, P, P]
    L.cogdl_gat_aggregate_proj.argtypes = [i32, i32, i64, P, P, i32, i32, P, P, f32, P, ctypes.c_int, P,
                                           ctypes.c_int, P, ctypes.c_int, P, P]
    L.cogdl_gat_aggregate_stats.argtypes = [i32, i32, i64, P, P, i32, i32, P, P, P, f32, P, ctypes.c_int, P,
                                            ctypes.c_int, P, P, ctypes.c_int, P, P]
    L.cogdl_linear.argtypes = [i64, i32, i32, P, P, ctypes.c_int, P, ctypes.c_int, P, ctypes.c_int, P]
    L.cogdl_head_scores.argtypes = [i64, i32, i32, P, ctypes.c_int, P, P, P, P, P]
    L.cogdl_act_codec_size.argtypes = [i64, i32, i32, i32, ctypes.POINTER(i64), ctypes.POINTER(i64)]
    L.cogdl_act_compress.argtypes = [i64, i32, P, ctypes.c_int, i32, i32, ctypes.c_uint64, P, P, P]
    L.cogdl_act_decompress.argtypes = [i64, i32, i32, i32, P, P, P, ctypes.c_int, P]
    L.cogdl_act_checkpoint.argtypes = [i64, i32, P, ctypes.c_int, P, P, P]
    L.cogdl_act_restore.argtypes = [i64, i32, P, P, P, ctypes.c_int, P]
    L.cogdl_grouped_linear.argtypes = [i64, i32, i32, i32, P, P, P, ctypes.c_int, P, ctypes.c_int, P,
                                       ctypes.c_int, P, P, P]
    L.cogdl_grouped_linear_backward_workspace.argtypes = [i64, i32, i32, i32, ctypes.POINTER(sz)]
    L.cogdl_grouped_linear_backward.argtypes = [i64, i32, i32, i32, P, P, P, P, P, P, ctypes.c_int, P,
                                                ctypes.c_int, P, P, ctypes.c_int, P, P, sz, P]
    L.cogdl_embedding.argtypes = [i64, i32, i32, P, ctypes.c_int, P, f32, P, ctypes.c_int, P]
    L.cogdl_embedding_backward_workspace.argtypes = [i64, i32, i32, ctypes.POINTER(sz)]
    L.cogdl_embedding_backward.argtypes = [i64, i32, i32, P, ctypes.c_int, P, f32, P, ctypes.c_int, i32, P, sz, P]
    L.cogdl_linear_loss_workspace.argtypes = [i64, i32, i32, i32, ctypes.POINTER(sz)]
    L.cogdl_linear_loss_backward_workspace.argtypes = L.cogdl_linear_loss_workspace.argtypes
    L.cogdl_linear_cross_entropy.argtypes = [i64, i32, i32, P, P, ctypes.c_int, P, P, P, P, P, sz, P]
    L.cogdl_linear_cross_entropy_backward.argtypes = [i64, i32, i32, P, P, P, ctypes.c_int, P, P, P, P, P, P, P, P,
                                                      sz, P]
    L.cogdl_linear_distill.argtypes = [i64, i32, i32, i32, P, P, ctypes.c_int, P, P, P, f32, P, P, P, P, sz, P]
    L.cogdl_linear_distill_backward.argtypes = [i64, i32, i32, i32, P, P, P, ctypes.c_int, P, P, P, f32, P, P, P, P,
                                                P, P, sz, P]
    L.cogdl_spmm_t.argtypes = [i32, i32, i64, P, P, P, i32, P, ctypes.c_int, P, ctypes.c_int, P, P]
    L.cogdl_csr_to_csc_workspace.argtypes = [i32, i32, i64, ctypes.POINTER(sz)]
    L.cogdl_csr_to_csc.argtypes = [i32, i32, i64, P, P, P, P, P, P, P, P, sz, P]
    L.cogdl_csr_to_csc_noalloc.argtypes = [i32, i32, i64, P, P, P, P, P, P, P, P]
    L.cogdl_sddmm_edge_softmax.argtypes = [i32, i32, i64, P, P, i32, P, P, f32, P, P, P]
    L.cogdl_gat_aggregate.argtypes = [i32, i32, i64, P, P, i32, i32, P, P, f32, P, P, ctypes.c_int,
                                      P, ctypes.c_int, P, P, P]
    L.cogdl_sddmm_dot.argtypes = [i32, i32, i64, P, P, i32, i32, P, ctypes.c_int, P, ctypes.c_int,
                                  P, P, P]
    L.cogdl_gat_backward.argtypes = [i32, i32, i64, P, P, P, P, P, i32, i32, P, P, f32, P, P,
                                     ctypes.c_int, P, ctypes.c_int, P, ctypes.c_int, P, P, P, P, P,
                                     P, P, P]
    L.cogdl_gat_backward_stats.argtypes = L.cogdl_gat_backward.argtypes
    L.cogdl_trace_enable.argtypes = [i32]
    L.cogdl_trace_filter.argtypes = [ctypes.c_char_p]
    L.cogdl_trace_count.restype = i32
    L.cogdl_trace_get.argtypes = [i32, ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(f32)]
    for name in ("cogdl_trace_enable", "cogdl_trace_filter", "cogdl_trace_reset", "cogdl_trace_get", "cogdl_plan_create", "cogdl_plan_rebuild", "cogdl_plan_create_sliced", "cogdl_plan_rebuild_sliced", "cogdl_plan_destroy", "cogdl_plan_query",
                 "cogdl_plan_units", "cogdl_spmm", "cogdl_gspmm", "cogdl_spmm_t", "cogdl_csr_to_csc_workspace",
                 "cogdl_csr_to_csc", "cogdl_csr_to_csc_noalloc", "cogdl_sddmm_edge_softmax",
                 "cogdl_gat_aggregate",
                 "cogdl_sddmm_dot", "cogdl_gat_backward", "cogdl_gat_backward_stats",
                 "cogdl_gat_aggregate_act", "cogdl_gat_aggregate_proj", "cogdl_gat_aggregate_stats",
                 "cogdl_linear",
                 "cogdl_head_scores", "cogdl_act_codec_size", "cogdl_act_compress",
                 "cogdl_act_decompress", "cogdl_act_checkpoint", "cogdl_act_restore", "cogdl_grouped_linear",
                 "cogdl_grouped_linear_backward_workspace", "cogdl_grouped_linear_backward", "cogdl_embedding",
                 "cogdl_embedding_backward_workspace", "cogdl_embedding_backward", "cogdl_linear_loss_workspace",
                 "cogdl_linear_loss_backward_workspace", "cogdl_linear_cross_entropy",
                 "cogdl_linear_cross_entropy_backward", "cogdl_linear_distill", "cogdl_linear_distill_backward"):
        getattr(L, name).restype = ctypes.c_int
    _lib = L
    return L


def _check(status: int, what: str):
    if status != 0:
        msg = lib().cogdl_status_string(status).decode()
        raise CogdlError(f"{what}: {msg} (status {status})")


def _dtype_code(t) -> int:
    import torch
    codes = {torch.float32: COGDL_F32, torch.bfloat16: COGDL_BF16, torch.float16: COGDL_F16}
    if t.dtype not in codes:
        raise CogdlError(f"unsupported feature dtype {t.dtype}")
    return codes[t.dtype]


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream():
    import torch
    # (the handle itself: a Stream object around it takes 3 us)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _dev(t, name, dtype=None):
    import torch
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise CogdlError(f"{name} must be a CUDA (HIP) tensor")
    if dtype is not None and t.dtype != dtype:
        raise CogdlError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise CogdlError(f"{name} must be contiguous")
    return t


# Size checks.  The C ABI receives bare pointers and cannot see how large a
# tensor is, so every size the library will read or write through is checked
# here, before any device check and before anything is launched: a tensor of
# the wrong size would otherwise be read or written out of bounds on the GPU.
def _tensor(t, name):
    import torch
    if not isinstance(t, torch.Tensor):
        raise CogdlError(f"{name} must be a torch tensor, got {type(t).__name__}")
    return t


def _dims(t, name, ndim):
    _tensor(t, name)
    if t.dim() != ndim:
        raise CogdlError(f"{name} must have {ndim} dimensions, got shape {tuple(t.shape)}")
    return tuple(t.shape)


def _numel(t, name, n):
    """t is None, or a tensor of exactly n elements."""
    if t is None:
        return
    _tensor(t, name)
    if t.numel() != n:
        raise CogdlError(f"{name} has {t.numel()} elements, expected {n}")


def _at_least(t, name, n):
    if t is None:
        return
    _tensor(t, name)
    if t.numel() < n:
        raise CogdlError(f"{name} has {t.numel()} elements, needs at least {n}")


def _index_array(t, name):
    """A 1-D int32 index array (rowptr, col, ...): its element count."""
    _dims(t, name, 1)
    return t.numel()


def _rowptr_rows(rowptr, name="rowptr"):
    n = _index_array(rowptr, name)
    if n < 1:
        raise CogdlError(f"{name} needs at least one entry (n_rows + 1)")
    return n - 1


def _feat2(X, name):
    """(rows, width) of a feature matrix given as [rows, F] or [rows]."""
    _tensor(X, name)
    if X.dim() == 2:
        return X.shape[0], X.shape[1]
    if X.dim() == 1:
        return X.shape[0], 1
    raise CogdlError(f"{name} must be [rows, F] or [rows], got shape {tuple(X.shape)}")


def _plan_matches(plan, n_rows, nnz, name="plan"):
    if plan is not None and (plan.n_rows != n_rows or plan.nnz != nnz):
        raise CogdlError(f"{name} was built for {plan.n_rows} rows and {plan.nnz} nonzeros, "
                         f"the call has {n_rows} rows and {nnz} nonzeros")


class Plan:
    """The data-aware workload balancer (section 2.2): run once per graph."""

    def __init__(self, rowptr, nnz: int, max_feat: int, max_heads: int = 0, mode: str = "auto",
                 group_size: int = 0, col=None, n_cols: int | None = None, slice_min: int = 0):
        """With `col` (and `n_cols`), a column-sliced plan (cogdl_plan_create_sliced): long rows
        are also cut at 8 column-range boundaries and each range's units run on one XCD."""
        import torch
        self._h = None
        n_rows = _rowptr_rows(rowptr)
        if mode not in BALANCE:
            raise CogdlError(f"mode must be one of {sorted(BALANCE)}")
        self.sliced = col is not None
        if self.sliced:
            _index_array(col, "col")
            _numel(col, "col", int(nnz))
            if n_cols is None:
                raise CogdlError("a sliced plan needs n_cols")
        _dev(rowptr, "rowptr", torch.int32)
        self.rowptr = rowptr
        self.n_rows = n_rows
        self.nnz = int(nnz)
        h = ctypes.c_void_p()
        if self.sliced:
            _dev(col, "col", torch.int32)
            self.col = col
            _check(lib().cogdl_plan_create_sliced(self.n_rows, self.nnz, _ptr(rowptr), _ptr(col), int(n_cols),
                                                  int(max_feat), int(max_heads), BALANCE[mode], int(group_size),
                                                  int(slice_min), _stream(), ctypes.byref(h)),
                   "cogdl_plan_create_sliced")
        else:
            _check(lib().cogdl_plan_create(self.n_rows, self.nnz, _ptr(rowptr), int(max_feat),
                                           int(max_heads), BALANCE[mode], int(group_size), _stream(),
                                           ctypes.byref(h)), "cogdl_plan_create")
        self._h = h

    @property
    def handle(self):
        if self._h is None:
            raise CogdlError("plan destroyed")
        return self._h

    def rebuild(self, rowptr=None, col=None):
        import torch
        if rowptr is not None:
            _numel(rowptr, "rowptr", self.n_rows + 1)
            _index_array(rowptr, "rowptr")
        if col is not None:
            if not self.sliced:
                raise CogdlError("only a sliced plan is rebuilt with col")
            _numel(col, "col", self.nnz)
            _index_array(col, "col")
        if rowptr is not None:
            _dev(rowptr, "rowptr", torch.int32)
            self.rowptr = rowptr
        if self.sliced:
            if col is not None:
                _dev(col, "col", torch.int32)
                self.col = col
            _check(lib().cogdl_plan_rebuild_sliced(self.handle, _ptr(self.rowptr), _ptr(self.col), _stream()),
                   "cogdl_plan_rebuild_sliced")
        else:
            _check(lib().cogdl_plan_rebuild(self.handle, _ptr(self.rowptr), _stream()), "cogdl_plan_rebuild")

    def info(self) -> dict:
        inf = _PlanInfo()
        _check(lib().cogdl_plan_query(self.handle, _stream(), ctypes.byref(inf)), "cogdl_plan_query")
        d = {f: getattr(inf, f) for f, _ in _PlanInfo._fields_}
        d["mode_name"] = MODE_NAMES.get(d["mode"], "?")
        return d

    def units(self):
        import torch
        n = self.info()["n_units"]
        out = torch.empty((max(n, 1), 4), dtype=torch.int32, device="cuda")
        _check(lib().cogdl_plan_units(self.handle, _ptr(out), n, _stream()), "cogdl_plan_units")
        return out[:n]

    def close(self):
        if getattr(self, "_h", None) is not None:
            lib().cogdl_plan_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def trace_enable(capacity: int = 4096):
    """Record HIP events around every library kernel launch (0 disables)."""
    _check(lib().cogdl_trace_enable(int(capacity)), "cogdl_trace_enable")


def trace_filter(names=None):
    """Record only the launches with these names (an iterable of str); None: all."""
    arg = None if names is None else ",".join(names).encode()
    _check(lib().cogdl_trace_filter(arg), "cogdl_trace_filter")


def trace_reset():
    _check(lib().cogdl_trace_reset(), "cogdl_trace_reset")


def trace_read() -> list:
    """[(kernel name, milliseconds)] of the launches recorded since the last reset."""
    L = lib()
    out = []
    for i in range(L.cogdl_trace_count()):
        name, ms = ctypes.c_char_p(), ctypes.c_float()
        _check(L.cogdl_trace_get(i, ctypes.byref(name), ctypes.byref(ms)), "cogdl_trace_get")
        out.append((name.value.decode(), ms.value))
    return out


def _plan_handle(plan):
    return None if plan is None else plan.handle


def _graph(rowptr, col, val=None, val_name="val"):
    """(n_rows, nnz) of a CSR (or CSC) graph, with the sizes of its arrays checked."""
    n_rows = _rowptr_rows(rowptr)
    nnz = _index_array(col, "col")
    _numel(val, val_name, nnz)
    return n_rows, nnz


def spmm(rowptr, col, val, X, plan: Plan | None = None, out_dtype=None, out=None):
    """Y[i] = sum_k val[k] * X[col[k]] over row i (Eq. 1, sum of products)."""
    import torch
    n_rows, nnz = _graph(rowptr, col, val)
    n_cols, F = _feat2(X, "X")
    _numel(out, "out", n_rows * F)
    _plan_matches(plan, n_rows, nnz)
    _dev(rowptr, "rowptr", torch.int32), _dev(col, "col", torch.int32)
    _dev(val, "val", torch.float32), _dev(X, "X")
    if out is None:
        out = torch.empty((n_rows, F), dtype=out_dtype or X.dtype, device=X.device)
    _dev(out, "out")
    _check(lib().cogdl_spmm(n_rows, n_cols, nnz, _ptr(rowptr), _ptr(col), _ptr(val), F,
                            _ptr(X), _dtype_code(X), _ptr(out), _dtype_code(out), _plan_handle(plan),
                            _stream()), "cogdl_spmm")
    return out


REDUCE = {"sum": 0, "mean": 1, "max": 2}
COMPUTE = {"mul": 0, "add": 1, "sub": 2, "copy": 3}
ACT = {"none": 0, "relu": 1, "elu": 2}


def gspmm(rowptr, col, val, X, reduce: str = "sum", plan: Plan | None = None, out_dtype=None,
          out=None, return_arg: bool = False, arg=None, compute: str = "mul", bias=None,
          act: str = "none"):
    """Eq. 1 with reduce = sum, mean or max over the edges k of row i of the
    message val[k] * x (compute "mul"), x + val[k] ("add"), x - val[k] ("sub")
    or x ("copy"), x = X[col[k]]; then act(. + bias) (bias fp32 [F] or None).

    For max, ``return_arg`` also returns the int32 edge id of the first edge
    attaining each output (-1 on empty rows); max keeps X's dtype or fp32."""
    import torch
    if reduce not in REDUCE:
        raise ValueError(f"reduce must be one of {sorted(REDUCE)}")
    if compute not in COMPUTE:
        raise ValueError(f"compute must be one of {sorted(COMPUTE)}")
    if act not in ACT:
        raise ValueError(f"act must be one of {sorted(ACT)}")
    if (return_arg or arg is not None) and reduce != "max":
        raise ValueError("return_arg / arg need reduce='max'")
    n_rows, nnz = _graph(rowptr, col, val)
    n_cols, F = _feat2(X, "X")
    _numel(out, "out", n_rows * F)
    _numel(arg, "arg", n_rows * F)
    _numel(bias, "bias", F)
    _plan_matches(plan, n_rows, nnz)
    _dev(bias, "bias", torch.float32)
    _dev(rowptr, "rowptr", torch.int32), _dev(col, "col", torch.int32)
    _dev(val, "val", torch.float32), _dev(X, "X")
    if out is None:
        out = torch.empty((n_rows, F), dtype=out_dtype or X.dtype, device=X.device)
    _dev(out, "out")
    if return_arg and arg is None:
        arg = torch.empty((n_rows, F), dtype=torch.int32, device=X.device)
    _dev(arg, "arg", torch.int32)
    _check(lib().cogdl_gspmm(n_rows, n_cols, nnz, _ptr(rowptr), _ptr(col), _ptr(val), F,
                             _ptr(X), _dtype_code(X), _ptr(out), _dtype_code(out), REDUCE[reduce],
                             COMPUTE[compute], _ptr(bias), ACT[act], _ptr(arg), _plan_handle(plan),
                             _stream()), "cogdl_gspmm")
    return (out, arg) if return_arg else out


def csr_to_csc_workspace(n_rows: int, n_cols: int, nnz: int) -> int:
    b = ctypes.c_size_t()
    _check(lib().cogdl_csr_to_csc_workspace(n_rows, n_cols, nnz, ctypes.byref(b)),
           "cogdl_csr_to_csc_workspace")
    return b.value


def csr_to_csc(rowptr, col, val, n_cols: int, workspace=None, with_perm: bool = True):
    """Stable transpose: (colptr, row_t, val_t, perm); inside a column edges keep CSR order."""
    import torch
    n_rows, nnz = _graph(rowptr, col, val)
    n_cols = int(n_cols)
    if n_cols < 0:
        raise CogdlError("n_cols must be >= 0")
    if workspace is not None:
        _dims(workspace, "workspace", 1)
    _dev(rowptr, "rowptr", torch.int32), _dev(col, "col", torch.int32), _dev(val, "val", torch.float32)
    dev = rowptr.device
    colptr = torch.empty(n_cols + 1, dtype=torch.int32, device=dev)
    row_t = torch.empty(nnz, dtype=torch.int32, device=dev)
    val_t = None if val is None else torch.empty(nnz, dtype=torch.float32, device=dev)
    perm = torch.empty(nnz, dtype=torch.int32, device=dev) if with_perm else None
    need = csr_to_csc_workspace(n_rows, n_cols, nnz)
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    _dev(workspace, "workspace")
    _check(lib().cogdl_csr_to_csc(n_rows, n_cols, nnz, _ptr(rowptr), _ptr(col), _ptr(val),
                                  _ptr(colptr), _ptr(row_t), _ptr(val_t), _ptr(perm), _ptr(workspace),
                                  workspace.numel() * workspace.element_size(), _stream()),
           "cogdl_csr_to_csc")
    return colptr, row_t, val_t, perm


def csr_to_csc_noalloc(rowptr, col, val, n_cols: int, out=None, with_perm: bool = True):
    """The transpose of csr_to_csc through cogdl_csr_to_csc_noalloc, which allocates nothing
    (its scratch is the library's static per-GPU array, so graphs up to about 1.6M edges).
    ``out`` may supply (colptr, row_t, val_t, perm); calls on one GPU must not overlap."""
    import torch
    n_rows, nnz = _graph(rowptr, col, val)
    n_cols = int(n_cols)
    if n_cols < 0:
        raise CogdlError("n_cols must be >= 0")
    if out is not None:
        colptr, row_t, val_t, perm = out
        _numel(colptr, "colptr", n_cols + 1)
        _numel(row_t, "row_t", nnz)
        _numel(val_t, "val_t", nnz)
        _numel(perm, "perm", nnz)
    need, limit = csr_to_csc_workspace(n_rows, n_cols, nnz), 64 << 20   # COGDL_NOALLOC_SCRATCH_BYTES
    if need > limit:
        raise CogdlError(f"cogdl_csr_to_csc_noalloc: a graph of {nnz} edges needs {need} bytes of "
                         f"scratch, the static scratch holds {limit}: use csr_to_csc with a workspace")
    _dev(rowptr, "rowptr", torch.int32), _dev(col, "col", torch.int32), _dev(val, "val", torch.float32)
    if out is None:
        dev = rowptr.device
        colptr = torch.empty(n_cols + 1, dtype=torch.int32, device=dev)
        row_t = torch.empty(nnz, dtype=torch.int32, device=dev)
        val_t = None if val is None else torch.empty(nnz, dtype=torch.float32, device=dev)
        perm = torch.empty(nnz, dtype=torch.int32, device=dev) if with_perm else None
    for t, name, dt in ((colptr, "colptr", torch.int32), (row_t, "row_t", torch.int32),
                        (val_t, "val_t", torch.float32), (perm, "perm", torch.int32)):
        _dev(t, name, dt)
    _check(lib().cogdl_csr_to_csc_noalloc(n_rows, n_cols, nnz, _ptr(rowptr), _ptr(col), _ptr(val),
                                          _ptr(colptr), _ptr(row_t), _ptr(val_t), _ptr(perm),
                                          _stream()), "cogdl_csr_to_csc_noalloc")
    return colptr, row_t, val_t, perm


def spmm_t(colptr, row_t, val_t, G, plan_t: Plan | None = None, out_dtype=None, out=None):
    """dX = A^T G from the CSC arrays of A; G is n_rows x F."""
    import torch
    n_cols = _rowptr_rows(colptr, "colptr")
    nnz = _index_array(row_t, "row_t")
    _numel(val_t, "val_t", nnz)
    n_rows, F = _feat2(G, "G")
    _numel(out, "out", n_cols * F)
    _plan_matches(plan_t, n_cols, nnz, "plan_t")
    _dev(colptr, "colptr", torch.int32), _dev(row_t, "row_t", torch.int32)
    _dev(val_t, "val_t", torch.float32), _dev(G, "G")
    if out is None:
        out = torch.empty((n_cols, F), dtype=out_dtype or G.dtype, device=G.device)
    _dev(out, "out")
    _check(lib().cogdl_spmm_t(n_rows, n_cols, nnz, _ptr(colptr), _ptr(row_t),
                              _ptr(val_t), F, _ptr(G), _dtype_code(G), _ptr(out), _dtype_code(out),
                              _plan_handle(plan_t), _stream()), "cogdl_spmm_t")
    return out


def _scores(t, name, rows, H):
    """A per-node score array [rows, H] (fp32)."""
    shape = _dims(t, name, 2)
    if shape != (rows, H):
        raise CogdlError(f"{name} must be [{rows}, {H}], got {shape}")


def sddmm_edge_softmax(rowptr, col, s_dst, s_src, negative_slope: float = 0.2,
                       plan: Plan | None = None, out=None):
    """alpha[k, h] = softmax over row i of LeakyReLU(s_dst[i, h] + s_src[col[k], h])."""
    import torch
    n_rows, nnz = _graph(rowptr, col)
    _dims(s_src, "s_src", 2)
    n_cols, H = s_src.shape
    _scores(s_dst, "s_dst", n_rows, H)
    _numel(out, "alpha", nnz * H)
    _plan_matches(plan, n_rows, nnz)
    _dev(rowptr, "rowptr", torch.int32), _dev(col, "col", torch.int32)
    _dev(s_dst, "s_dst", torch.float32), _dev(s_src, "s_src", torch.float32)
    if out is None:
        out = torch.empty((nnz, H), dtype=torch.float32, device=col.device)
    _dev(out, "alpha", torch.float32)
    _check(lib().cogdl_sddmm_edge_softmax(n_rows, n_cols, nnz, _ptr(rowptr),
                                          _ptr(col), H, _ptr(s_dst), _ptr(s_src),
                                          float(negative_slope), _ptr(out), _plan_handle(plan),
                                          _stream()), "cogdl_sddmm_edge_softmax")
    return out


def gat_aggregate(rowptr, col, s_dst, s_src, X, negative_slope: float = 0.2, alpha_in=None,
                  return_alpha: bool = False, plan: Plan | None = None, out_dtype=None, out=None,
                  alpha_out=None, bias=None, act: str = "none"):
    """Fused GAT aggregation.  X is [n_cols, H, D]; returns Y [n_rows, H, D] (and alpha).
    With bias (fp32 [H*D]) or act, Y = act(aggregate + bias) (cogdl_gat_aggregate_act)."""
    import torch
    if act not in ACT:
        raise ValueError(f"act must be one of {sorted(ACT)}")
    n_rows, nnz = _graph(rowptr, col)
    n_cols, H, D = _dims(X, "X", 3)
    if alpha_in is None:
        _scores(s_dst, "s_dst", n_rows, H)
        _scores(s_src, "s_src", n_cols, H)
    else:
        if s_dst is not None:
            _scores(s_dst, "s_dst", n_rows, H)
        if s_src is not None:
            _scores(s_src, "s_src", n_cols, H)
        _numel(alpha_in, "alpha_in", nnz * H)
    _numel(out, "out", n_rows * H * D)
    _numel(alpha_out, "alpha_out", nnz * H)
    _numel(bias, "bias", H * D)
    _plan_matches(plan, n_rows, nnz)
    _dev(bias, "bias", torch.float32)
    _dev(rowptr, "rowptr", torch.int32), _dev(col, "col", torch.int32), _dev(X, "X")
    _dev(s_dst, "s_dst", torch.float32), _dev(s_src, "s_src", torch.float32)
    _dev(alpha_in, "alpha_in", torch.float32)
    if out is None:
        out = torch.empty((n_rows, H, D), dtype=out_dtype or X.dtype, device=X.device)
    _dev(out, "out")
    if return_alpha and alpha_out is None:
        alpha_out = torch.empty((nnz, H), dtype=torch.float32, device=X.device)
    _dev(alpha_out, "alpha_out", torch.float32)
    if bias is None and act == "none":
        _check(lib().cogdl_gat_aggregate(n_rows, n_cols, nnz, _ptr(rowptr), _ptr(col), H, D,
                                         _ptr(s_dst), _ptr(s_src), float(negative_slope),
                                         _ptr(alpha_in), _ptr(X), _dtype_code(X), _ptr(out),
                                         _dtype_code(out), _ptr(alpha_out), _plan_handle(plan),
                                         _stream()), "cogdl_gat_aggregate")
    else:
        _check(lib().cogdl_gat_aggregate_act(n_rows, n_cols, nnz, _ptr(rowptr), _ptr(col), H, D,
                                             _ptr(s_dst), _ptr(s_src), float(negative_slope),
                                             _ptr(alpha_in), _ptr(X), _dtype_code(X), _ptr(out),
                                             _dtype_code(out), _ptr(alpha_out), _ptr(bias), ACT[act],
                                             _plan_handle(plan), _stream()), "cogdl_gat_aggregate_act")
    return (out, alpha_out) if return_alpha else out


def gat_aggregate_proj(rowptr, col, s_dst, a_src, X, negative_slope: float = 0.2,
                       plan: Plan | None = None, out_dtype=None, out=None, bias=None, act: str = "none"):
    """Fused GAT aggregation with the source scores projected from the gathered rows:
    s_src[j, h] = <X[j, h, :], a_src[h, :]> inside the kernel (cogdl_gat_aggregate_proj).
    X [n_cols, H, D] with D * itemsize a multiple of 16 bytes; a_src fp32 [H, D]."""
    import torch
    if act not in ACT:
        raise ValueError(f"act must be one of {sorted(ACT)}")
    n_rows, nnz = _graph(rowptr, col)
    n_cols, H, D = _dims(X, "X", 3)
    _scores(s_dst, "s_dst", n_rows, H)
    _numel(a_src, "a_src", H * D)
    _numel(out, "out", n_rows * H * D)
    _numel(bias, "bias", H * D)
    _plan_matches(plan, n_rows, nnz)
    _dev(bias, "bias", torch.float32), _dev(a_src, "a_src", torch.float32)
    _dev(rowptr, "rowptr", torch.int32), _dev(col, "col", torch.int32), _dev(X, "X")
    _dev(s_dst, "s_dst", torch.float32)
    if out is None:
        out = torch.empty((n_rows, H, D), dtype=out_dtype or X.dtype, device=X.device)
    _dev(out, "out")
    _check(lib().cogdl_gat_aggregate_proj(n_rows, n_cols, nnz, _ptr(rowptr), _ptr(col), H, D, _ptr(s_dst),
                                          _ptr(a_src), float(negative_slope), _ptr(X), _dtype_code(X),
                                          _ptr(out), _dtype_code(out), _ptr(bias), ACT[act],
                                          _plan_handle(plan), _stream()), "cogdl_gat_aggregate_proj")
    return out


def gat_aggregate_stats(rowptr, col, s_dst, X, s_src=None, a_src=None, negative_slope: float = 0.2,
                        plan: Plan | None = None, out_dtype=None, out=None, stats_out=None, bias=None,
                        act: str = "none"):
    """The GAT aggregation of a training step: returns (Y, row_stats), row_stats fp32
    [n_rows, 2, H] = the final (max score, 1 / normalizer) of each row's softmax per head, from
    which gat_backward(row_stats=...) rebuilds every weight instead of reading alpha.  Exactly
    one of s_src (scores given) and a_src (projected from X, as gat_aggregate_proj)."""
    import torch
    if act not in ACT:
        raise ValueError(f"act must be one of {sorted(ACT)}")
    if (s_src is None) == (a_src is None):
        raise CogdlError("give exactly one of s_src and a_src")
    n_rows, nnz = _graph(rowptr, col)
    n_cols, H, D = _dims(X, "X", 3)
    _scores(s_dst, "s_dst", n_rows, H)
    if s_src is not None:
        _scores(s_src, "s_src", n_cols, H)
    else:
        _numel(a_src, "a_src", H * D)
    _numel(out, "out", n_rows * H * D)
    _numel(stats_out, "stats_out", n_rows * 2 * H)
    _numel(bias, "bias", H * D)
    _plan_matches(plan, n_rows, nnz)
    _dev(bias, "bias", torch.float32), _dev(a_src, "a_src", torch.float32)
    _dev(rowptr, "rowptr", torch.int32), _dev(col, "col", torch.int32), _dev(X, "X")
    _dev(s_dst, "s_dst", torch.float32), _dev(s_src, "s_src", torch.float32)
    if out is None:
        out = torch.empty((n_rows, H, D), dtype=out_dtype or X.dtype, device=X.device)
    _dev(out, "out")
    if stats_out is None:
        stats_out = torch.empty((n_rows, 2, H), dtype=torch.float32, device=X.device)
    _dev(stats_out, "stats_out", torch.float32)
    _check(lib().cogdl_gat_aggregate_stats(n_rows, n_cols, nnz, _ptr(rowptr), _ptr(col), H, D, _ptr(s_dst),
                                           _ptr(s_src), _ptr(a_src), float(negative_slope), _ptr(X),
                                           _dtype_code(X), _ptr(out), _dtype_code(out), _ptr(stats_out),
                                           _ptr(bias), ACT[act], _plan_handle(plan), _stream()),
           "cogdl_gat_aggregate_stats")
    return out, stats_out


def sddmm_dot(rowptr, col, P, Q, plan: Plan | None = None, out=None):
    """out[k, h] = <P[i, h, :], Q[col[k], h, :]> for every edge k = (i, col[k]):
    the SDDMM of section 2.2 per head.  P is [n_rows, H, D], Q [n_cols, H, D]."""
    import torch
    n_rows, nnz = _graph(rowptr, col)
    pr, H, D = _dims(P, "P", 3)
    n_cols, qh, qd = _dims(Q, "Q", 3)
    if (qh, qd) != (H, D):
        raise CogdlError("P and Q must be [n, H, D] with the same H and D")
    if pr != n_rows:
        raise CogdlError(f"P has {pr} rows, the graph {n_rows}")
    _numel(out, "out", nnz * H)
    _plan_matches(plan, n_rows, nnz)
    _dev(rowptr, "rowptr", torch.int32), _dev(col, "col", torch.int32), _dev(P, "P"), _dev(Q, "Q")
    if out is None:
        out = torch.empty((nnz, H), dtype=torch.float32, device=P.device)
    _dev(out, "out", torch.float32)
    _check(lib().cogdl_sddmm_dot(n_rows, n_cols, nnz, _ptr(rowptr), _ptr(col), H, D, _ptr(P),
                                 _dtype_code(P), _ptr(Q), _dtype_code(Q), _ptr(out), _plan_handle(plan),
                                 _stream()), "cogdl_sddmm_dot")
    return out


def gat_backward(rowptr, col, colptr, row_t, perm, s_dst, s_src, alpha, X, dY,
                 negative_slope: float = 0.2, plan: Plan | None = None, plan_t: Plan | None = None,
                 dx_dtype=None, out=None, row_stats=None):
    """Gradients of gat_aggregate for dY = dL/dY.  X is [n_cols, H, D], dY [n_rows, H, D],
    alpha [nnz, H] the forward weights; (colptr, row_t, perm) the CSC from csr_to_csc.
    Returns dict(dX, dalpha, dscore, ds_dst, ds_src, edge_work); ``out`` may supply these
    tensors, and ``out={"dalpha": None, "dscore": None}`` (either or both) leaves those
    outputs out.  edge_work (fp32, 2 nnz H) is the library's scratch between its two passes:
    it ends holding the pair (alpha, dscore) of every edge and head.  With alpha None and
    row_stats (from gat_aggregate_stats) the weights are rebuilt instead of read
    (cogdl_gat_backward_stats)."""
    import torch
    n_rows, nnz = _graph(rowptr, col)
    n_cols, H, D = _dims(X, "X", 3)
    if _dims(dY, "dY", 3) != (n_rows, H, D):
        raise CogdlError(f"dY must be [{n_rows}, {H}, {D}], got {tuple(dY.shape)}")
    _numel(colptr, "colptr", n_cols + 1)
    _index_array(colptr, "colptr")
    for t, name in ((row_t, "row_t"), (perm, "perm")):
        _numel(t, name, nnz)
        _index_array(t, name)
    _scores(s_dst, "s_dst", n_rows, H)
    _scores(s_src, "s_src", n_cols, H)
    if (alpha is None) == (row_stats is None):
        raise CogdlError("give exactly one of alpha and row_stats")
    _numel(alpha, "alpha", nnz * H)
    _numel(row_stats, "row_stats", n_rows * 2 * H)
    o = dict(out or {})
    sizes = {"dX": n_cols * H * D, "dalpha": nnz * H, "dscore": nnz * H, "ds_dst": n_rows * H,
             "ds_src": n_cols * H, "edge_work": 2 * nnz * H}
    for k in o:
        if k not in sizes:
            raise CogdlError(f"unknown output {k!r}")
        if o[k] is None and k not in ("dalpha", "dscore"):
            raise CogdlError(f"output {k!r} is required")
        if o[k] is not None:
            _numel(o[k], k, sizes[k])
    _plan_matches(plan, n_rows, nnz)
    _plan_matches(plan_t, n_cols, nnz, "plan_t")
    for t, name, dt in ((rowptr, "rowptr", torch.int32), (col, "col", torch.int32),
                        (colptr, "colptr", torch.int32), (row_t, "row_t", torch.int32),
                        (perm, "perm", torch.int32), (s_dst, "s_dst", torch.float32),
                        (s_src, "s_src", torch.float32), (alpha, "alpha", torch.float32),
                        (row_stats, "row_stats", torch.float32)):
        _dev(t, name, dt)
    _dev(X, "X"), _dev(dY, "dY")
    dev = X.device
    o.setdefault("dX", torch.empty((n_cols, H, D), dtype=dx_dtype or X.dtype, device=dev))
    o.setdefault("dalpha", torch.empty((nnz, H), dtype=torch.float32, device=dev))
    o.setdefault("dscore", torch.empty((nnz, H), dtype=torch.float32, device=dev))
    o.setdefault("ds_dst", torch.empty((n_rows, H), dtype=torch.float32, device=dev))
    o.setdefault("ds_src", torch.empty((n_cols, H), dtype=torch.float32, device=dev))
    o.setdefault("edge_work", torch.empty((nnz, H, 2), dtype=torch.float32, device=dev))
    _dev(o["dX"], "dX")
    for k in ("dalpha", "dscore", "ds_dst", "ds_src", "edge_work"):
        if o[k] is not None:
            _dev(o[k], k, torch.float32)
    fn = "cogdl_gat_backward" if row_stats is None else "cogdl_gat_backward_stats"
    _check(getattr(lib(), fn)(
        n_rows, n_cols, nnz, _ptr(rowptr), _ptr(col), _ptr(colptr), _ptr(row_t), _ptr(perm), H, D,
        _ptr(s_dst), _ptr(s_src), float(negative_slope), _ptr(alpha if row_stats is None else row_stats),
        _ptr(X), _dtype_code(X), _ptr(dY), _dtype_code(dY), _ptr(o["dX"]), _dtype_code(o["dX"]),
        _ptr(o["dalpha"]), _ptr(o["dscore"]), _ptr(o["ds_dst"]), _ptr(o["ds_src"]), _ptr(o["edge_work"]),
        _plan_handle(plan), _plan_handle(plan_t), _stream()), fn)
    return o


def linear(X, W, bias=None, act: str = "none", out_dtype=None, out=None):
    """Y = act(X W^T + bias) on the matrix cores.  X [n, k] and W [m, k] (a layer's out x in
    weights) both bf16 or both fp16; bias fp32 [m] or None."""
    import torch
    if act not in ACT:
        raise ValueError(f"act must be one of {sorted(ACT)}")
    n, k = _dims(X, "X", 2)
    m, kw = _dims(W, "W", 2)
    if kw != k or X.dtype != W.dtype:
        raise CogdlError("X must be [n, k] and W [m, k] of the same dtype")
    _numel(bias, "bias", m)
    _numel(out, "out", n * m)
    _dev(X, "X"), _dev(W, "W"), _dev(bias, "bias", torch.float32)
    if out is None:
        out = torch.empty((n, m), dtype=out_dtype or X.dtype, device=X.device)
    _dev(out, "out")
    _check(lib().cogdl_linear(n, k, m, _ptr(X), _ptr(W), _dtype_code(X), _ptr(bias), ACT[act],
                              _ptr(out), _dtype_code(out), _stream()), "cogdl_linear")
    return out


def head_scores(Z, a_src, a_dst):
    """s_src[i, h] = <Z[i, h, :], a_src[h]>, s_dst likewise; Z [n, H, D], a_* fp32 [H, D].
    Either vector may be None; its scores are then not computed (returned as None)."""
    import torch
    n, H, D = _dims(Z, "Z", 3)
    if a_src is None and a_dst is None:
        raise CogdlError("head_scores needs a_src or a_dst")
    _numel(a_src, "a_src", H * D)
    _numel(a_dst, "a_dst", H * D)
    _dev(Z, "Z"), _dev(a_src, "a_src", torch.float32), _dev(a_dst, "a_dst", torch.float32)
    s_src = None if a_src is None else torch.empty((n, H), dtype=torch.float32, device=Z.device)
    s_dst = None if a_dst is None else torch.empty((n, H), dtype=torch.float32, device=Z.device)
    _check(lib().cogdl_head_scores(n, H, D, _ptr(Z), _dtype_code(Z), _ptr(a_src), _ptr(a_dst),
                                   _ptr(s_src), _ptr(s_dst), _stream()), "cogdl_head_scores")
    return s_src, s_dst


def _padded_output_layer(params, names_rows, names_cols):
    """The output layer's parameters with the output count padded to a multiple of 8 (zero
    rows / entries), prepared once per parameter dict: the aggregation then gathers
    16-byte vectors instead of single 16-bit elements of rows like 41 classes wide.  The
    padded outputs are exactly zero and are sliced away."""
    import torch
    key = "_padded_output_layer"
    if key not in params:
        C = params[names_rows[0]].shape[0]
        C8 = (C + 7) // 8 * 8
        pad = {}
        for n_ in names_rows:                     # [C, ...] -> [C8, ...]
            t = params[n_]
            z = torch.zeros((C8,) + tuple(t.shape[1:]), dtype=t.dtype, device=t.device)
            z[:C] = t
            pad[n_] = z
        for n_ in names_cols:                     # [1, C] -> [1, C8]
            t = params[n_]
            z = torch.zeros((t.shape[0], C8), dtype=t.dtype, device=t.device)
            z[:, :C] = t
            pad[n_] = z
        params[key] = (C, C8, pad)
    return params[key]


def gcn_forward(rowptr, col, val, X, params, plan: Plan | None = None):
    """2-layer GCN inference: H1 = relu(A (X W1^T) + b1), Y = A (H1 W2^T) + b2, every step a
    library kernel (dense layers on the matrix cores, aggregations with the bias and
    activation in their epilogue).  params: dict of W1 [hid, in], b1 [hid], W2 [out, hid],
    b2 [out]; activations stay in X's dtype.  Returns Y [n, out] (a view of the padded
    output when out is not a multiple of 8)."""
    C, C8, pad = _padded_output_layer(params, ("W2", "b2"), ())
    Z1 = linear(X, params["W1"])
    H1 = gspmm(rowptr, col, val, Z1, "sum", plan=plan, bias=params["b1"], act="relu")
    Z2 = linear(H1, pad["W2"])
    Y = gspmm(rowptr, col, val, Z2, "sum", plan=plan, bias=pad["b2"], act="none")
    return Y if C8 == C else Y[:, :C]


def _proj_ok(Z):
    """Whether cogdl_gat_aggregate_proj takes heads of this shape: [n, H, D] with each head a
    power-of-two number of 16-byte vectors."""
    per = 16 // Z.element_size()
    D = Z.shape[2]
    return D % per == 0 and ((D // per) & (D // per - 1)) == 0 and Z.data_ptr() % 16 == 0


def gat_forward(rowptr, col, X, params, negative_slope: float = 0.2, plan: Plan | None = None):
    """2-layer GAT inference: layer 1 with H heads of D (concatenated, ELU), layer 2 with one
    head of C outputs.  params: W1 [H*D, in], a_src1 / a_dst1 [H, D], b1 [H*D], W2 [C, H*D],
    a_src2 / a_dst2 [1, C], b2 [C].  Returns Y [n, C] (a view of the padded output when C is
    not a multiple of 8)."""
    H, D = params["a_src1"].shape
    C, C8, pad = _padded_output_layer(params, ("W2", "b2"), ("a_src2", "a_dst2"))
    n = X.shape[0]
    Z1 = linear(X, params["W1"]).view(n, H, D)
    if _proj_ok(Z1):
        # source scores formed from the rows the aggregation gathers: only s_dst is precomputed
        _, s_dst = head_scores(Z1, None, params["a_dst1"])
        H1 = gat_aggregate_proj(rowptr, col, s_dst, params["a_src1"], Z1, negative_slope, plan=plan,
                                bias=params["b1"], act="elu")
    else:
        s_src, s_dst = head_scores(Z1, params["a_src1"], params["a_dst1"])
        H1 = gat_aggregate(rowptr, col, s_dst, s_src, Z1, negative_slope, plan=plan, bias=params["b1"],
                           act="elu")
    Z2 = linear(H1.view(n, H * D), pad["W2"]).view(n, 1, C8)
    s_src2, s_dst2 = head_scores(Z2, pad["a_src2"], pad["a_dst2"])
    Y = gat_aggregate(rowptr, col, s_dst2, s_src2, Z2, negative_slope, plan=plan,
                      bias=pad["b2"]).view(n, C8)
    return Y if C8 == C else Y[:, :C]


def act_codec_size(n: int, F: int, bits: int, group: int):
    """(uint64 code words, fp32 stats) of a compressed n x F activation array."""
    w, st = ctypes.c_int64(), ctypes.c_int64()
    _check(lib().cogdl_act_codec_size(n, F, bits, group, ctypes.byref(w), ctypes.byref(st)),
           "cogdl_act_codec_size")
    return w.value, st.value


def act_compress(A, bits: int, group: int, seed: int, codes=None, stats=None):
    """Per-group `bits`-bit stochastic quantization of A [n, F]: returns (codes int64 view of
    the uint64 bit planes, stats fp32 [groups, 2] = (min, step))."""
    import torch
    n, F = _dims(A, "A", 2)
    words, nst = act_codec_size(n, F, bits, group)
    _at_least(codes, "codes", words)
    _at_least(stats, "stats", nst)
    _dev(A, "A")
    if codes is None:
        codes = torch.empty(max(words, 1), dtype=torch.int64, device=A.device)
    if stats is None:
        stats = torch.empty(max(nst, 1), dtype=torch.float32, device=A.device)
    _dev(codes, "codes", torch.int64), _dev(stats, "stats", torch.float32)
    _check(lib().cogdl_act_compress(n, F, _ptr(A), _dtype_code(A), bits, group,
                                    ctypes.c_uint64(seed & 0xFFFFFFFFFFFFFFFF), _ptr(codes),
                                    _ptr(stats), _stream()), "cogdl_act_compress")
    return codes[:words], stats[:nst]


def act_decompress(codes, stats, n: int, F: int, bits: int, group: int, out_dtype=None, out=None):
    import torch
    words, nst = act_codec_size(n, F, bits, group)
    _at_least(codes, "codes", words)
    _at_least(stats, "stats", nst)
    _numel(out, "out", n * F)
    _dev(codes, "codes", torch.int64), _dev(stats, "stats", torch.float32)
    if out is None:
        out = torch.empty((n, F), dtype=out_dtype or torch.float32, device=codes.device)
    _dev(out, "out")
    _check(lib().cogdl_act_decompress(n, F, bits, group, _ptr(codes), _ptr(stats), _ptr(out),
                                      _dtype_code(out), _stream()), "cogdl_act_decompress")
    return out


CKPT_BLOCK = 32        # COGDL_CKPT_BLOCK: features that share an exponent byte
MAX_GROUPS = 4096      # COGDL_MAX_GROUPS


_HERE = contextlib.nullcontext()


def _on_device(*tensors):
    """A context with the tensors' device current (they must share one)."""
    import torch
    devices = {t.get_device() for t in tensors if t is not None}
    if len(devices) != 1:
        raise CogdlError(f"the tensors lie on several devices: {sorted(devices)}")
    device = devices.pop()
    return _HERE if device == torch.cuda.current_device() else torch.cuda.device(device)


def _addr(t):
    return None if t is None else t.data_ptr()


def _ckpt_blocks(F):
    return (F + CKPT_BLOCK - 1) // CKPT_BLOCK


def act_checkpoint(A, codes=None, exps=None):
    """The 8-bit checkpoint of activations A [n, F] (cogdl_act_checkpoint): returns (codes int8
    [n, F], exps uint8 [n, ceil(F / 32)]).  Feature x of a block of 32 is kept as q * 2^(b - 127),
    b its exponent byte, within half a step (at most 1/127.5 of the block's largest magnitude)."""
    import torch
    n, F = _dims(A, "A", 2)
    if F < 1:
        raise CogdlError("A needs at least one feature")
    nb = _ckpt_blocks(F)
    _numel(codes, "codes", n * F)
    _numel(exps, "exps", n * nb)
    _dev(A, "A")
    dt = _dtype_code(A)
    if codes is None:
        codes = A.new_empty((n, F), dtype=torch.int8)
    if exps is None:
        exps = A.new_empty((n, nb), dtype=torch.uint8)
    _dev(codes, "codes", torch.int8), _dev(exps, "exps", torch.uint8)
    with _on_device(A, codes, exps):
        _check(lib().cogdl_act_checkpoint(n, F, _addr(A), dt, _addr(codes), _addr(exps), _stream()),
               "cogdl_act_checkpoint")
    return codes, exps


def act_restore(codes, exps, out_dtype=None, out=None):
    """The activations [n, F] that a checkpoint (act_checkpoint) stands for, in out_dtype (fp32 by
    default; bf16 holds every value exactly, fp16 those of fp16 activations)."""
    import torch
    n, F = _dims(codes, "codes", 2)
    if F < 1:
        raise CogdlError("codes need at least one feature")
    _numel(exps, "exps", n * _ckpt_blocks(F))
    _numel(out, "out", n * F)
    _dev(codes, "codes", torch.int8), _dev(exps, "exps", torch.uint8)
    if out is None:
        out = codes.new_empty((n, F), dtype=out_dtype or torch.float32)
    _dev(out, "out")
    with _on_device(codes, exps, out):
        _check(lib().cogdl_act_restore(n, F, _addr(codes), _addr(exps), _addr(out), _dtype_code(out), _stream()),
               "cogdl_act_restore")
    return out


def _groups(W, offsets):
    """(E, m, k) of grouped weights, with the offsets' size checked."""
    E, m, k = _dims(W, "W", 3)
    if E < 1 or E > MAX_GROUPS:
        raise CogdlError(f"W has {E} groups, 1 to {MAX_GROUPS} are supported")
    _dims(offsets, "offsets", 1)
    _numel(offsets, "offsets", E + 1)
    return E, m, k


def grouped_linear(X, W, offsets, bias=None, act: str = "none", out_dtype=None, out=None, save: bool = False,
                   codes=None, exps=None):
    """linear() with a weight matrix per group of rows: Y[i] = act(X[i] W[g]^T + bias[g]) for the rows i
    in [offsets[g], offsets[g + 1]) of group g (sorted node types, relations, experts; a group may have
    none).  X [n, k] and W [E, m, k] both bf16 or both fp16; offsets int32 [E + 1] on the device; bias
    fp32 [E, m] or None.  Rows before offsets[0] and from offsets[E] on belong to no group: ``out`` keeps
    what it held there, a fresh output holds anything.  With ``save`` (or codes and exps given) returns
    (Y, codes, exps), the 8-bit checkpoint of X for grouped_linear_backward.  A given ``out`` has the type
    it has (out_dtype is for a fresh one).  Not recorded by autograd: the gradients are
    grouped_linear_backward's."""
    import torch
    if act not in ACT:
        raise ValueError(f"act must be one of {sorted(ACT)}")
    n, k = _dims(X, "X", 2)
    E, m, kw = _groups(W, offsets)
    if kw != k or X.dtype != W.dtype:
        raise CogdlError("X must be [n, k] and W [E, m, k] of the same dtype")
    if (codes is None) != (exps is None):
        raise CogdlError("give codes and exps together")
    save = save or codes is not None
    if save and k < 1:
        raise CogdlError("X needs at least one feature to be saved")
    _numel(bias, "bias", E * m)
    _numel(out, "out", n * m)
    _numel(codes, "codes", n * k)
    _numel(exps, "exps", n * _ckpt_blocks(k))
    _dev(X, "X"), _dev(W, "W"), _dev(offsets, "offsets", torch.int32), _dev(bias, "bias", torch.float32)
    if out is None:
        out = X.new_empty((n, m), dtype=out_dtype or X.dtype)
    if save and codes is None:
        codes = X.new_empty((n, k), dtype=torch.int8)
        exps = X.new_empty((n, _ckpt_blocks(k)), dtype=torch.uint8)
    _dev(out, "out"), _dev(codes, "codes", torch.int8), _dev(exps, "exps", torch.uint8)
    with _on_device(X, W, offsets, bias, out, codes, exps):
        _check(lib().cogdl_grouped_linear(n, E, k, m, _addr(offsets), _addr(X), _addr(W), _dtype_code(X), _addr(bias),
                                          ACT[act], _addr(out), _dtype_code(out), _addr(codes), _addr(exps),
                                          _stream()), "cogdl_grouped_linear")
    return (out, codes, exps) if save else out


@functools.lru_cache(maxsize=256)
def grouped_linear_backward_workspace(n: int, E: int, k: int, m: int) -> int:
    """Bytes of scratch that grouped_linear_backward takes for n rows and E groups of k features to m outputs."""
    b = ctypes.c_size_t()
    _check(lib().cogdl_grouped_linear_backward_workspace(n, E, k, m, ctypes.byref(b)),
           "cogdl_grouped_linear_backward_workspace")
    return b.value


def grouped_linear_backward(dY, W, offsets, X=None, codes=None, exps=None, Y=None, act: str = "none",
                            dw_dtype=None, out=None, workspace=None):
    """Gradients of grouped_linear for dY = dL/dY [n, m]: returns dict(dX [n, k], dW [E, m, k], db fp32
    [E, m]).  The input comes as X [n, k] or as its 8-bit checkpoint (codes, exps), which the products read
    as it is.  With an activation, Y is the forward's output in dY's dtype (ELU's dZ is rounded to that
    dtype for dX and dW, an fp32 dW too).  dw_dtype, of a fresh dW: dY's dtype (default) or fp32.  ``out``
    may supply the tensors, of either type for dW; a None among them leaves that gradient out.  Groups without
    rows get zeros; rows of no group keep what dX held there (anything in a fresh one).  ``workspace``: at
    least grouped_linear_backward_workspace bytes."""
    import torch
    if act not in ACT:
        raise ValueError(f"act must be one of {sorted(ACT)}")
    n, m = _dims(dY, "dY", 2)
    E, mw, k = _groups(W, offsets)
    if mw != m or dY.dtype != W.dtype:
        raise CogdlError("dY must be [n, m] and W [E, m, k] of the same dtype")
    o = dict(out or {})
    sizes = {"dX": n * k, "dW": E * m * k, "db": E * m}
    for name, t in o.items():
        if name not in sizes:
            raise CogdlError(f"unknown output {name!r}")
        _numel(t, name, sizes[name])
    if (codes is None) != (exps is None):
        raise CogdlError("give codes and exps together")
    if X is not None and codes is not None:
        raise CogdlError("give X or its checkpoint (codes and exps), not both")
    if o.get("dW", 0) is not None and X is None and codes is None:
        raise CogdlError("dW needs X or its checkpoint (codes and exps)")
    if X is not None and (_dims(X, "X", 2) != (n, k) or X.dtype != dY.dtype):
        raise CogdlError(f"X must be [{n}, {k}] of dY's dtype")
    if codes is not None and _dims(codes, "codes", 2) != (n, k):
        raise CogdlError(f"codes must be [{n}, {k}], got {tuple(codes.shape)}")
    _numel(exps, "exps", n * _ckpt_blocks(k))
    if act == "none":
        Y = None
    elif Y is None:
        raise CogdlError("the activation's gradient needs Y, the forward's output")
    elif _dims(Y, "Y", 2) != (n, m) or Y.dtype != dY.dtype:
        raise CogdlError(f"Y must be [{n}, {m}] of dY's dtype")
    need = grouped_linear_backward_workspace(n, E, k, m)
    if workspace is not None:
        _at_least(workspace, "workspace", (need + workspace.element_size() - 1) // workspace.element_size())
    _dev(dY, "dY"), _dev(W, "W"), _dev(offsets, "offsets", torch.int32), _dev(X, "X"), _dev(Y, "Y")
    _dev(codes, "codes", torch.int8), _dev(exps, "exps", torch.uint8)
    if "dX" not in o:
        o["dX"] = dY.new_empty((n, k), dtype=dY.dtype)
    if "dW" not in o:
        o["dW"] = dY.new_empty((E, m, k), dtype=dw_dtype or dY.dtype)
    if "db" not in o:
        o["db"] = dY.new_empty((E, m), dtype=torch.float32)
    dX, dW, db = o["dX"], o["dW"], o["db"]
    _dev(dX, "dX", dY.dtype), _dev(dW, "dW"), _dev(db, "db", torch.float32)
    if workspace is None and need > 0 and (dW is not None or db is not None):
        workspace = dY.new_empty(need, dtype=torch.uint8)
    _dev(workspace, "workspace")
    with _on_device(dY, W, offsets, X, codes, exps, Y, dX, dW, db, workspace):
        _check(lib().cogdl_grouped_linear_backward(
            n, E, k, m, _addr(offsets), _addr(dY), _addr(W), _addr(X), _addr(codes), _addr(exps), _dtype_code(dY),
            _addr(Y), ACT[act], _addr(dX), _addr(dW), _dtype_code(dY if dW is None else dW), _addr(db),
            _addr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(),
            _stream()), "cogdl_grouped_linear_backward")
    return o


def _take(t, name, dtype, device):
    """The address of a contiguous tensor of this dtype (None: of any) on this device; None for None."""
    if t is None:
        return None
    if (dtype is not None and t.dtype is not dtype) or t.get_device() != device or not t.is_contiguous():
        _dev(t, name, dtype)
        raise CogdlError(f"the tensors lie on several devices: {name} on {t.get_device()}, others on {device}")
    return t.data_ptr()


def _home(t, name):
    """The device of the tensor that the others have to share, and a context with it current."""
    import torch
    if not t.is_cuda:
        raise CogdlError(f"{name} must be a CUDA (HIP) tensor")
    device = t.get_device()
    return device, _HERE if device == torch._C._cuda_getDevice() else torch.cuda.device(device)


def _stream_of(device):
    import torch
    return torch._C._cuda_getCurrentRawStream(device)


def _scratch(workspace, need, like, device):
    """(address, bytes, tensor) of a workspace of at least `need` bytes: the one given, or a fresh one."""
    import torch
    if workspace is None:
        if need == 0:
            return None, 0, None
        workspace = like.new_empty(need, dtype=torch.uint8)
        return workspace.data_ptr(), need, workspace
    _at_least(workspace, "workspace", (need + workspace.element_size() - 1) // workspace.element_size())
    return _take(workspace, "workspace", None, device), workspace.numel() * workspace.element_size(), workspace


_I32_MAX = 2 ** 31 - 1


def _in_32_bits(V, k):
    """Refuses a table whose sizes the C ABI does not take."""
    if V > _I32_MAX or k > _I32_MAX:
        raise CogdlError(f"a table of {V} rows of {k} has a size past 32 bits")


def embedding(table, index, scale: float = 1.0, out_dtype=None, out=None):
    """Rows of a table [V, k] (fp32, bf16 or fp16) by an int32 index [n], times ``scale``: Y [n, k] in out_dtype (the
    table's by default).  An index outside [0, V) stands for a padded place: a row of zeros.  A given ``out``
    has the type it has.  Not recorded by autograd: the gradient is embedding_backward's."""
    import torch
    V, k = _dims(table, "table", 2)
    if V < 1:
        raise CogdlError("table needs at least one row")
    _in_32_bits(V, k)
    n = _index_array(index, "index")
    _numel(out, "out", n * k)
    device, here = _home(table, "table")
    pt, pi = _take(table, "table", None, device), _take(index, "index", torch.int32, device)
    if out is None:
        out = table.new_empty((n, k), dtype=out_dtype or table.dtype)
    po = _take(out, "out", None, device)
    with here:
        _check(lib().cogdl_embedding(n, V, k, pt, _dtype_code(table), pi, float(scale), po, _dtype_code(out),
                                     _stream_of(device)), "cogdl_embedding")
    return out


@functools.lru_cache(maxsize=256)
def embedding_backward_workspace(n: int, V: int, k: int) -> int:
    """Bytes of scratch that embedding_backward takes for n places and a table of V rows of k features."""
    b = ctypes.c_size_t()
    _check(lib().cogdl_embedding_backward_workspace(n, V, k, ctypes.byref(b)), "cogdl_embedding_backward_workspace")
    return b.value


def embedding_backward(dY, index, V: int, scale: float = 1.0, out_dtype=None, out=None, accumulate: bool = False,
                       workspace=None):
    """Gradient of embedding for dY = dL/dY [n, k]: dtable [V, k] in out_dtype (dY's by default), with
    dtable[v] = scale * the sum of dY over the places of v, in fp32 and in a fixed order (the same bits every run).
    With ``accumulate``, ``out`` must be given: the sums are added to it, and its other rows are left alone (the
    other gradient of a tied table, such as linear_cross_entropy_backward's dW); else they become zeros.  Padded
    places (an index outside [0, V)) count for nothing.  ``workspace``: at least embedding_backward_workspace
    bytes."""
    import torch
    n, k = _dims(dY, "dY", 2)
    V = operator.index(V)
    if V < 1:
        raise CogdlError("the table needs at least one row")
    _in_32_bits(V, k)
    _index_array(index, "index")
    _numel(index, "index", n)
    _numel(out, "out", V * k)
    if accumulate and out is None:
        raise CogdlError("accumulate needs out, the gradient to add to")
    need = embedding_backward_workspace(n, V, k)
    device, here = _home(dY, "dY")
    pd, pi = _take(dY, "dY", None, device), _take(index, "index", torch.int32, device)
    if out is None:
        out = dY.new_empty((V, k), dtype=out_dtype or dY.dtype)
    po = _take(out, "out", None, device)
    pw, bytes_, workspace = _scratch(workspace, need, dY, device)
    with here:
        _check(lib().cogdl_embedding_backward(n, V, k, pd, _dtype_code(dY), pi, float(scale), po, _dtype_code(out),
                                              1 if accumulate else 0, pw, bytes_, _stream_of(device)),
               "cogdl_embedding_backward")
    return out


MAX_TEACHER = 1024     # COGDL_MAX_TEACHER: entries of a teacher's row


@functools.lru_cache(maxsize=256)
def linear_loss_workspace(n: int, V: int, k: int, K: int = 0) -> int:
    """Bytes of scratch that linear_cross_entropy (K = 0) or linear_distill of K entries takes."""
    b = ctypes.c_size_t()
    _check(lib().cogdl_linear_loss_workspace(n, V, k, K, ctypes.byref(b)), "cogdl_linear_loss_workspace")
    return b.value


@functools.lru_cache(maxsize=256)
def linear_loss_backward_workspace(n: int, V: int, k: int, K: int = 0) -> int:
    """Bytes of scratch that the backward of linear_cross_entropy (K = 0) or linear_distill takes."""
    b = ctypes.c_size_t()
    _check(lib().cogdl_linear_loss_backward_workspace(n, V, k, K, ctypes.byref(b)),
           "cogdl_linear_loss_backward_workspace")
    return b.value


def _head(X, W, bias):
    """(n, V, k, dtype code) of a linear layer over a vocabulary, with its sizes checked."""
    n, k = _dims(X, "X", 2)
    V, kw = _dims(W, "W", 2)
    if kw != k or X.dtype != W.dtype:
        raise CogdlError("X must be [n, k] and W [V, k] of the same dtype")
    if V < 1:
        raise CogdlError("W needs at least one row")
    _in_32_bits(V, k)
    if bias is not None:
        _numel(bias, "bias", V)
    return n, V, k, _dtype_code(X)


def _teacher(index, teacher, n, temperature):
    """The entries of a teacher's row, with sizes and temperature checked."""
    if _dims(index, "index", 2)[0] != n or _dims(teacher, "teacher", 2) != tuple(index.shape):
        raise CogdlError(f"index and teacher must both be [{n}, K]")
    K = index.shape[1]
    if K < 1 or K > MAX_TEACHER:
        raise CogdlError(f"index has {K} entries a row, 1 to {MAX_TEACHER} are supported")
    if not 2.0 ** -20 <= float(temperature) <= 2.0 ** 20:
        raise CogdlError(f"temperature must be positive, from 2^-20 to 2^20, got {temperature}")
    return K


def linear_cross_entropy(X, W, target, bias=None, loss=None, lse=None, workspace=None):
    """Softmax cross entropy of the logits z = X W^T + bias over a large vocabulary, which are never kept: returns
    (loss, lse), fp32 [n] each, with lse = logsumexp(z) and loss = lse - z[target].  X [n, k] and W [V, k] both
    bf16 or both fp16; target int32 [n], a row whose target lies outside [0, V) is left out (loss and lse 0);
    bias fp32 [V] or None (-inf takes an answer out).  ``workspace``: at least linear_loss_workspace bytes.  Not
    recorded by autograd: the gradients are linear_cross_entropy_backward's."""
    import torch
    n, V, k, dt = _head(X, W, bias)
    _index_array(target, "target")
    _numel(target, "target", n)
    _numel(loss, "loss", n), _numel(lse, "lse", n)
    need = linear_loss_workspace(n, V, k)
    device, here = _home(X, "X")
    f32, i32 = torch.float32, torch.int32
    px, pw, pt = _take(X, "X", None, device), _take(W, "W", None, device), _take(target, "target", i32, device)
    pb = _take(bias, "bias", f32, device)
    if loss is None:
        loss = X.new_empty(n, dtype=f32)
    if lse is None:
        lse = X.new_empty(n, dtype=f32)
    pl, ps = _take(loss, "loss", f32, device), _take(lse, "lse", f32, device)
    ws, bytes_, workspace = _scratch(workspace, need, X, device)
    with here:
        _check(lib().cogdl_linear_cross_entropy(n, V, k, px, pw, dt, pb, pt, pl, ps, ws, bytes_, _stream_of(device)),
               "cogdl_linear_cross_entropy")
    return loss, lse


def linear_distill(X, W, index, teacher, bias=None, temperature: float = 1.0, loss=None, lse=None, logp=None,
                   workspace=None):
    """Distillation from a teacher's top K logits: the loss of the logits z = X W^T + bias, over the whole
    vocabulary and never kept, against q = softmax(teacher / T) over the K entries of a row.  Returns (loss, lse,
    logp): loss = T^2 sum q (log q - logp) [n], lse = logsumexp(z / T) [n], logp = z[index] / T - lse [n, K], all
    fp32.  index int32 [n, K] (outside [0, V): no entry), teacher fp32 [n, K]; a row without entries is left out
    (zeros).  A loss may lie below 0: by rounding, or where entries share an answer.  Everything else as
    linear_cross_entropy; the gradients are linear_distill_backward's."""
    import torch
    n, V, k, dt = _head(X, W, bias)
    K = _teacher(index, teacher, n, temperature)
    _numel(loss, "loss", n), _numel(lse, "lse", n), _numel(logp, "logp", n * K)
    need = linear_loss_workspace(n, V, k, K)
    device, here = _home(X, "X")
    f32, i32 = torch.float32, torch.int32
    px, pw, pi = _take(X, "X", None, device), _take(W, "W", None, device), _take(index, "index", i32, device)
    pt, pb = _take(teacher, "teacher", f32, device), _take(bias, "bias", f32, device)
    if loss is None:
        loss = X.new_empty(n, dtype=f32)
    if lse is None:
        lse = X.new_empty(n, dtype=f32)
    if logp is None:
        logp = X.new_empty((n, K), dtype=f32)
    pl, ps, pp = _take(loss, "loss", f32, device), _take(lse, "lse", f32, device), _take(logp, "logp", f32, device)
    ws, bytes_, workspace = _scratch(workspace, need, X, device)
    with here:
        _check(lib().cogdl_linear_distill(n, V, k, K, px, pw, dt, pb, pi, pt, float(temperature), pl, ps, pp, ws, bytes_,
                                          _stream_of(device)), "cogdl_linear_distill")
    return loss, lse, logp


def _head_gradients(X, W, bias, out, device):
    """The gradients' outputs, those given, checked, or fresh ones (db where there is a bias), and their addresses."""
    import torch
    if out is None:
        dX, dW = torch.empty_like(X), torch.empty_like(W)
        db = None if bias is None else torch.empty_like(bias)
        return {"dX": dX, "dW": dW, "db": db}, dX.data_ptr(), dW.data_ptr(), None if db is None else db.data_ptr()
    o = dict(out)
    sizes = {"dX": X.numel(), "dW": W.numel(), "db": W.shape[0]}
    for name, t in o.items():
        if name not in sizes:
            raise CogdlError(f"unknown output {name!r}")
        _numel(t, name, sizes[name])
    for name, like in (("dX", X), ("dW", W), ("db", bias)):
        if name not in o:
            o[name] = None if like is None else torch.empty_like(like)
    return (o, _take(o["dX"], "dX", X.dtype, device), _take(o["dW"], "dW", X.dtype, device),
            _take(o["db"], "db", torch.float32, device))


def linear_cross_entropy_backward(dloss, X, W, target, loss, lse, bias=None, out=None, workspace=None):
    """Gradients of linear_cross_entropy for dloss = dL/dloss fp32 [n], from the forward's loss and lse: returns
    dict(dX [n, k], dW [V, k], db fp32 [V]; db None without a bias).  The logits are computed again by pieces of the
    vocabulary; the products take dz = dloss (softmax(z) - onehot) rounded to X's dtype, db sums it unrounded.
    Rows left out get zeros in dX and enter no sum.  ``out`` may supply the tensors; a None among them leaves that
    gradient out.  ``workspace``: at least linear_loss_backward_workspace bytes."""
    import torch
    n, V, k, dt = _head(X, W, bias)
    _index_array(target, "target")
    _numel(target, "target", n)
    for name, t in (("dloss", dloss), ("loss", loss), ("lse", lse)):
        if _tensor(t, name).numel() != n:
            _numel(t, name, n)
    need = linear_loss_backward_workspace(n, V, k)
    device, here = _home(X, "X")
    f32, i32 = torch.float32, torch.int32
    px, pw, pt = _take(X, "X", None, device), _take(W, "W", None, device), _take(target, "target", i32, device)
    pb, pd = _take(bias, "bias", f32, device), _take(dloss, "dloss", f32, device)
    pl, ps = _take(loss, "loss", f32, device), _take(lse, "lse", f32, device)
    o, dx, dw, db = _head_gradients(X, W, bias, out, device)
    ws, bytes_, workspace = _scratch(workspace, need, X, device)
    with here:
        _check(lib().cogdl_linear_cross_entropy_backward(n, V, k, pd, px, pw, dt, pb, pt, pl, ps, dx, dw, db, ws, bytes_,
                                                         _stream_of(device)), "cogdl_linear_cross_entropy_backward")
    return o


def linear_distill_backward(dloss, X, W, index, teacher, lse, logp, bias=None, temperature: float = 1.0, out=None,
                            workspace=None):
    """Gradients of linear_distill for dloss = dL/dloss fp32 [n], from the forward's lse and logp: returns
    dict(dX, dW, db) as linear_cross_entropy_backward does (none of the teacher's logits)."""
    import torch
    n, V, k, dt = _head(X, W, bias)
    K = _teacher(index, teacher, n, temperature)
    for name, t, size in (("dloss", dloss, n), ("lse", lse, n), ("logp", logp, n * K)):
        if _tensor(t, name).numel() != size:
            _numel(t, name, size)
    need = linear_loss_backward_workspace(n, V, k, K)
    device, here = _home(X, "X")
    f32, i32 = torch.float32, torch.int32
    px, pw, pi = _take(X, "X", None, device), _take(W, "W", None, device), _take(index, "index", i32, device)
    pt, pb = _take(teacher, "teacher", f32, device), _take(bias, "bias", f32, device)
    pd, ps, pp = _take(dloss, "dloss", f32, device), _take(lse, "lse", f32, device), _take(logp, "logp", f32, device)
    o, dx, dw, db = _head_gradients(X, W, bias, out, device)
    ws, bytes_, workspace = _scratch(workspace, need, X, device)
    with here:
        _check(lib().cogdl_linear_distill_backward(n, V, k, K, pd, px, pw, dt, pb, pi, pt, float(temperature), ps, pp, dx, dw,
                                                   db, ws, bytes_, _stream_of(device)), "cogdl_linear_distill_backward")
    return o
