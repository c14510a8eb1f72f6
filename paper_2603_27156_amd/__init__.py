"""Python binding of libgsr.so, the MI355X (gfx950) GSR-GNN training-step library.

Argument marshalling only: every function has the name of the C entry point it calls
(include/gsr.h) and does no arithmetic of its own.  PyTorch provides device memory and the
current HIP stream, nothing else.  If the compiled library is missing the import of the
package still works (so the input generators in `synth` stay usable on a CPU-only box) but
every call raises: there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import os
from array import array
from dataclasses import dataclass
from typing import Optional, Tuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
# GSR_LIB names another build of the library (kernel variants under measurement); default: the one built in-tree
LIB_PATH = os.environ.get("GSR_LIB") or os.path.join(_HERE, "libgsr.so")
MARSHAL_PATH = os.path.join(_HERE, "libgsr_marshal.so")     # reads lists of torch tensors for the entry points that take lists

GSR_OK, GSR_ERR_INVALID_ARG, GSR_ERR_BAD_CSR, GSR_ERR_UNSUPPORTED, GSR_ERR_WORKSPACE_TOO_SMALL, GSR_ERR_HIP = range(6)
GSR_F32, GSR_BF16 = 0, 1
GSR_NORM_NONE, GSR_NORM_RMS = 0, 1
GSR_LAYOUT_ROW_MAJOR, GSR_LAYOUT_GROUP_PLANAR = 0, 1
GSR_GRAPH_SYMMETRISE, GSR_GRAPH_ADD_SELF_LOOPS, GSR_GRAPH_GCN_NORM, GSR_GRAPH_ROWPTR_I64 = 1, 2, 4, 8
GSR_ADJ_UNIT, GSR_ADJ_GCN_SYM = 0, 1
GSR_ACT_NONE, GSR_ACT_RELU, GSR_ACT_SILU = 0, 1, 2
GSR_CHECKPOINT_BLOCK = 64

EXPORTED = [
    "gsr_last_error", "gsr_version", "gsr_set_option", "gsr_profile_read", "gsr_profile_reset",
    "gsr_profile_class_name", "gsr_graph_create", "gsr_graph_normalize", "gsr_graph_info",
    "gsr_graph_export", "gsr_graph_destroy", "gsr_group_sparse", "gsr_spmm", "gsr_spmm_noalloc",
    "gsr_spmm_compressed_workspace",
    "gsr_spmm_compressed", "gsr_workspace_size", "gsr_layer_forward", "gsr_layer_inverse", "gsr_layer_backward",
    "gsr_step", "gsr_step_tie_stats", "gsr_step_tie_export", "gsr_walkthrough_workspace", "gsr_slot_block", "gsr_alg1_layer_forward", "gsr_alg2_layer_backward",
    "gsr_sgd_update", "gsr_adam_update",
    "gsr_embed_lookup", "gsr_embed_grad_workspace", "gsr_embed_grad",
    "gsr_grad_norm_workspace", "gsr_grad_norm", "gsr_grad_clip", "gsr_adam_update_list",
    "gsr_group_norm_workspace", "gsr_group_norm", "gsr_group_norm_grad", "gsr_checkpoint_save", "gsr_checkpoint_load",
    "gsr_class_loss_workspace", "gsr_class_grad_workspace", "gsr_class_loss", "gsr_class_grad",
]


class GsrError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"gsr status {status}: {message}")
        self.status = status


def gsr_last_error() -> str:
    """Message of the last call that returned a status other than GSR_OK."""
    return lib().gsr_last_error().decode()


class gsr_config_t(C.Structure):
    _fields_ = [("n", C.c_int64), ("d", C.c_int32), ("c", C.c_int32), ("l", C.c_int32), ("k", C.c_int32),
                ("dtype", C.c_int32), ("norm", C.c_int32), ("eps", C.c_float), ("layout", C.c_int32),
                ("save_indices", C.c_int32), ("tie_tol", C.c_float), ("tie_capacity", C.c_int32)]


_lib = None


def lib():
    """The loaded libgsr.so.  Raises if it has not been built (python -m paper_2603_27156_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise GsrError(-1, f"{LIB_PATH} is missing: build it with `python -m paper_2603_27156_amd.build`; "
                               "there is no CPU fallback")
        l = C.CDLL(LIB_PATH)
        l.gsr_last_error.restype = C.c_char_p
        l.gsr_version.restype = C.c_char_p
        l.gsr_profile_class_name.restype = C.c_char_p
        l.gsr_spmm_compressed_workspace.restype = C.c_size_t
        l.gsr_spmm_compressed_workspace.argtypes = [C.c_void_p, C.c_int32, C.c_int32]
        l.gsr_walkthrough_workspace.restype = C.c_size_t
        l.gsr_walkthrough_workspace.argtypes = [C.c_void_p, C.c_int32]
        p, i32, i64, f32, size = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_size_t
        l.gsr_embed_lookup.argtypes = [p, i64, i64, i32, p, i32, i64, i32, i32, i32, i32, f32, p, i64, p]
        l.gsr_embed_grad_workspace.restype = size
        l.gsr_embed_grad_workspace.argtypes = [i64, i64, i32]
        l.gsr_embed_grad.argtypes = [p, i32, i64, p, i64, i32, i32, i32, i32, f32, i64, p, i64, p, size, p]
        l.gsr_grad_norm_workspace.restype = size
        l.gsr_grad_norm_workspace.argtypes = [p, i32]
        l.gsr_grad_norm.argtypes = [p, p, i32, i32, p, p, size, p]
        l.gsr_grad_clip.argtypes = [p, p, i32, i32, f32, p, p, i32, p, size, p]
        l.gsr_adam_update_list.argtypes = [p, p, p, p, p, i32, i32, p, f32, i64, *[C.c_double] * 5, p]
        l.gsr_group_norm_workspace.restype = size
        l.gsr_group_norm_workspace.argtypes = [i64, i64, i32, i32, i32, i32, i32]
        l.gsr_group_norm.argtypes = [p, i64, i64, i32, i32, i32, i32, p, i32, i64, i32, p, p, f32, i32, p, i64, p, p, p, p, p, size, p]
        l.gsr_group_norm_grad.argtypes = [p, i64, p, i64, p, p, i64, i32, i32, i32, i32, p, i32, i64, i32, p, p, p, p, i32, p, i64, p, p, p, size, p]
        l.gsr_checkpoint_save.argtypes = [p, i64, i64, i32, i32, i32, i32, p, p, p]
        l.gsr_checkpoint_load.argtypes = [p, p, i64, i32, i32, i32, i32, p, i64, p]
        for f in (l.gsr_class_loss_workspace, l.gsr_class_grad_workspace):
            f.restype = size
            f.argtypes = [i64, i64, i32, i32]
        l.gsr_class_loss.argtypes = [p, i64, i64, i32, i32, i32, i32, p, i64, i64, p, p, i32, p, p, p, size, p]
        l.gsr_class_grad.argtypes = [p, i64, i64, i32, i32, i32, i32, p, i64, i64, p, p, i32, p, f32, p, i64, p, i64, p, p, size, p]
        _lib = l
    return _lib


def _check(st: int):
    if st != GSR_OK:
        raise GsrError(st, lib().gsr_last_error().decode())


def _stream() -> C.c_void_p:
    # The handle of torch.cuda.current_stream(), without the 3 us that making a Stream object of it takes, where torch has a function for it: that
    # one is not part of its documented interface.
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return C.c_void_p(torch.cuda.current_stream().cuda_stream if raw is None else raw(torch.cuda.current_device()))


def _dp(t) -> C.c_void_p:
    return C.c_void_p(0 if t is None else t.data_ptr())


def _np(a) -> C.c_void_p:
    return None if a is None else a.ctypes.data_as(C.c_void_p)


def gsr_version() -> str:
    return lib().gsr_version().decode()


def gsr_set_option(key: str, value: int) -> None:
    _check(lib().gsr_set_option(key.encode(), C.c_int64(value)))


KERNEL_CLASSES = 11


def gsr_profile_reset() -> None:
    _check(lib().gsr_profile_reset())


def gsr_profile_read(kernel_class: int) -> Tuple[float, int]:
    """(summed milliseconds, launches) of one kernel class since the last reset."""
    ms, cnt = C.c_double(), C.c_int64()
    _check(lib().gsr_profile_read(C.c_int32(kernel_class), C.byref(ms), C.byref(cnt)))
    return ms.value, cnt.value


def gsr_profile_class_name(kernel_class: int) -> str:
    return lib().gsr_profile_class_name(C.c_int32(kernel_class)).decode()


@dataclass
class Config:
    n: int
    d: int
    c: int
    k: int
    l: int = 1
    dtype: int = GSR_F32
    norm: int = GSR_NORM_NONE
    eps: float = 1e-5
    layout: int = GSR_LAYOUT_ROW_MAJOR
    save_indices: int = 0
    tie_tol: float = 2.0 ** -12
    tie_capacity: int = 0

    @property
    def dg(self) -> int:
        return self.d // self.c

    def c_struct(self) -> gsr_config_t:
        return gsr_config_t(self.n, self.d, self.c, self.l, self.k, self.dtype, self.norm, self.eps, self.layout,
                            self.save_indices, self.tie_tol, self.tie_capacity)


class Graph:
    """Owner of a gsr_graph_t*."""

    def __init__(self, ptr: int):
        self.ptr = C.c_void_p(ptr)

    def destroy(self):
        if self.ptr:
            lib().gsr_graph_destroy(self.ptr)
            self.ptr = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def gsr_graph_create(rowptr: np.ndarray, colidx: np.ndarray, vals: Optional[np.ndarray] = None,
                     flags: int = GSR_GRAPH_SYMMETRISE | GSR_GRAPH_ADD_SELF_LOOPS | GSR_GRAPH_GCN_NORM,
                     n: Optional[int] = None, nnz: Optional[int] = None) -> Graph:
    """Host CSR (numpy) -> device graph.  rowptr int32 or int64 (flag set automatically)."""
    rowptr = np.ascontiguousarray(rowptr)
    if rowptr.dtype == np.int64:
        flags |= GSR_GRAPH_ROWPTR_I64
    elif rowptr.dtype == np.int32:
        flags &= ~GSR_GRAPH_ROWPTR_I64
    else:
        raise TypeError("rowptr must be int32 or int64")
    colidx = np.ascontiguousarray(colidx, dtype=np.int32)
    if vals is not None:
        vals = np.ascontiguousarray(vals, dtype=np.float32)
    n = len(rowptr) - 1 if n is None else n
    nnz = len(colidx) if nnz is None else nnz
    out = C.c_void_p()
    _check(lib().gsr_graph_create(C.byref(out), C.c_int64(n), C.c_int64(nnz), _np(rowptr), _np(colidx), _np(vals),
                                  C.c_uint32(flags), _stream() if _has_cuda() else None))
    return Graph(out.value)


def _has_cuda() -> bool:
    try:
        import torch
        return torch.cuda.is_available()
    except Exception:
        return False


def gsr_graph_normalize(g: Graph, mode: int) -> None:
    _check(lib().gsr_graph_normalize(g.ptr, C.c_int32(mode), _stream()))


def gsr_graph_info(g: Graph) -> dict:
    n, nnz, md, nh = C.c_int64(), C.c_int64(), C.c_int64(), C.c_int64()
    _check(lib().gsr_graph_info(g.ptr, C.byref(n), C.byref(nnz), C.byref(md), C.byref(nh)))
    return dict(n=n.value, nnz=nnz.value, max_degree=md.value, n_hub_rows=nh.value)


def gsr_graph_export(g: Graph) -> Tuple[np.ndarray, np.ndarray, np.ndarray]:
    info = gsr_graph_info(g)
    rp = np.zeros(info["n"] + 1, dtype=np.int64)
    ci = np.zeros(max(1, info["nnz"]), dtype=np.int32)
    av = np.zeros(max(1, info["nnz"]), dtype=np.float32)
    _check(lib().gsr_graph_export(g.ptr, _np(rp), _np(ci), _np(av)))
    return rp, ci[:info["nnz"]], av[:info["nnz"]]


def _dtype_of(t) -> int:
    import torch
    if t.dtype == torch.float32:
        return GSR_F32
    if t.dtype == torch.bfloat16:
        return GSR_BF16
    raise TypeError(f"unsupported tensor dtype {t.dtype}")


def gsr_group_sparse(x, k: int, norm: int = GSR_NORM_NONE, eps: float = 1e-5):
    """GS(X, k) -> (V [n,k] of x.dtype, I [n,k] int32).  x: device tensor [n, dg], last dim contiguous."""
    import torch
    assert x.is_cuda and x.dim() == 2 and x.stride(1) == 1
    n, dg = x.shape
    vals = torch.empty((n, k), dtype=x.dtype, device=x.device)
    idx = torch.empty((n, k), dtype=torch.int32, device=x.device)
    _check(lib().gsr_group_sparse(_dp(x), C.c_int64(n), C.c_int32(dg), C.c_int64(x.stride(0) if n > 1 else dg),
                                  C.c_int32(k), C.c_int32(_dtype_of(x)), C.c_int32(norm), C.c_float(eps), _dp(vals),
                                  _dp(idx), _stream()))
    return vals, idx


def gsr_spmm(g: Graph, x, transpose: bool = False):
    import torch
    assert x.is_cuda and x.dtype == torch.float32 and x.dim() == 2 and x.stride(1) == 1
    n, width = x.shape
    y = torch.empty((n, width), dtype=torch.float32, device=x.device)
    _check(lib().gsr_spmm(g.ptr, _dp(x), C.c_int64(x.stride(0) if n > 1 else width), C.c_int32(width), _dp(y),
                          C.c_int64(width), C.c_int32(1 if transpose else 0), _stream()))
    return y


def gsr_spmm_noalloc(g: Graph, x, y, transpose: bool = False) -> None:
    """gsr_spmm into the caller's y, with the library's scratch in a fixed device array: nothing is allocated."""
    import torch
    for t in (x, y):
        assert t.is_cuda and t.dtype == torch.float32 and t.dim() == 2 and t.stride(1) == 1
    assert x.shape == y.shape
    n, width = x.shape
    _check(lib().gsr_spmm_noalloc(g.ptr, _dp(x), C.c_int64(x.stride(0) if n > 1 else width), C.c_int32(width), _dp(y),
                                  C.c_int64(y.stride(0) if n > 1 else width), C.c_int32(1 if transpose else 0), _stream()))


def _walkthrough_ws(g: Graph, k: int, device):
    import torch
    nbytes = lib().gsr_walkthrough_workspace(g.ptr, C.c_int32(k))
    return torch.empty(max(1, nbytes), dtype=torch.uint8, device=device), nbytes


def gsr_slot_block(g: Graph, vals, idx, dg: int, transpose: bool = False):
    """The block of the Section 4.3 / 4.4 walk-throughs: out[i, idx[i,t]] = sum_j a_ij vals[j,t] -> float32 [n, dg]."""
    import torch
    assert vals.is_cuda and idx.is_cuda and vals.dtype == torch.float32 and idx.dtype == torch.int32
    assert vals.is_contiguous() and idx.is_contiguous()
    n, k = vals.shape
    out = torch.empty((n, dg), dtype=torch.float32, device=vals.device)
    ws, nbytes = _walkthrough_ws(g, k, vals.device)
    _check(lib().gsr_slot_block(g.ptr, _dp(vals), _dp(idx), C.c_int32(k), C.c_int32(dg), C.c_int32(1 if transpose else 0),
                                _dp(out), C.c_int64(dg), _dp(ws), C.c_size_t(nbytes), _stream()))
    return out


def gsr_alg1_layer_forward(g: Graph, x1, x2, k: int):
    """One pass of the loop body of Algorithm 1 on the planes x1, x2 (float32 [n, dg], updated in place)."""
    import torch
    for x in (x1, x2):
        assert x.is_cuda and x.dtype == torch.float32 and x.dim() == 2 and x.stride(1) == 1
    assert x1.shape == x2.shape and x1.stride(0) == x2.stride(0)
    n, dg = x1.shape
    ws, nbytes = _walkthrough_ws(g, k, x1.device)
    _check(lib().gsr_alg1_layer_forward(g.ptr, C.c_int32(dg), C.c_int32(k), _dp(x1), _dp(x2),
                                        C.c_int64(x1.stride(0) if n > 1 else dg), _dp(ws), C.c_size_t(nbytes), _stream()))


def gsr_alg2_layer_backward(g: Graph, g1, g2, k: int):
    """One pass of the loop body of Algorithm 2 on the gradient planes g1, g2 (float32 [n, dg], in place)."""
    import torch
    for x in (g1, g2):
        assert x.is_cuda and x.dtype == torch.float32 and x.dim() == 2 and x.stride(1) == 1
    assert g1.shape == g2.shape and g1.stride(0) == g2.stride(0)
    n, dg = g1.shape
    ws, nbytes = _walkthrough_ws(g, k, g1.device)
    _check(lib().gsr_alg2_layer_backward(g.ptr, C.c_int32(dg), C.c_int32(k), _dp(g1), _dp(g2),
                                         C.c_int64(g1.stride(0) if n > 1 else dg), _dp(ws), C.c_size_t(nbytes), _stream()))


def gsr_sgd_update(w, dw, lr: float, weight_decay: float = 0.0):
    """w <- w - lr * (dw + weight_decay * w), in place (float32 device tensors of one shape)."""
    import torch
    assert w.is_cuda and dw.is_cuda and w.dtype == dw.dtype == torch.float32 and w.is_contiguous() and dw.is_contiguous()
    assert w.numel() == dw.numel()
    _check(lib().gsr_sgd_update(_dp(w), _dp(dw), C.c_int64(w.numel()), C.c_float(lr), C.c_float(weight_decay), _stream()))


def gsr_adam_update(w, dw, m, v, t: int, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                    weight_decay: float = 0.0):
    """One Adam step with bias correction, in place; m, v: state tensors (zero before t = 1)."""
    import torch
    for x in (w, dw, m, v):
        assert x.is_cuda and x.dtype == torch.float32 and x.is_contiguous() and x.numel() == w.numel()
    _check(lib().gsr_adam_update(_dp(w), _dp(dw), _dp(m), _dp(v), C.c_int64(w.numel()), C.c_int64(t), C.c_float(lr),
                                 C.c_float(beta1), C.c_float(beta2), C.c_float(eps), C.c_float(weight_decay), _stream()))


def _plane(x, dev: int):
    """(rows, D, groups, layout, row stride) of a plane [n, D] (rows may be strided) or [C, n, D/C] on GPU `dev`."""
    shape, strides = x.shape, x.stride()
    assert x.get_device() == dev and (strides[-1] == 1 or shape[-1] == 1)
    if len(shape) == 2:
        n, d = shape
        return n, d, 1, GSR_LAYOUT_ROW_MAJOR, strides[0] if n > 1 else d
    c, n, dg = shape
    ld = strides[1] if n > 1 else strides[0] if n and c > 1 else dg
    assert c == 1 or n == 0 or strides[0] == n * ld, "the groups of a plane follow each other"
    return n, c * dg, c, GSR_LAYOUT_GROUP_PLANAR, ld


def _current_device() -> int:
    import torch
    return torch.cuda.current_device()


def _tokens(ids, n: int, dev: int) -> int:
    import torch
    assert ids.get_device() == dev and ids.shape == (n,) and ids.is_contiguous()
    dtype = ids.dtype
    assert dtype == torch.int32 or dtype == torch.int64
    return 1 if dtype == torch.int64 else 0


def gsr_embed_lookup(table, ids, x_out, scale: float = 1.0) -> None:
    """x_out[i] = scale * table[ids[i]], zeros where a token lies outside the table.  table: [vocab, D], rows may be strided; x_out: a
    plane [n, D] or [C, n, D/C]; either of both float32 or bfloat16.  ids: [n] int32 or int64."""
    dev = _current_device()
    n, d, c, layout, ldx = _plane(x_out, dev)
    vocab, dt, _, rows, ldt = _plane(table, dev)
    assert dt == d and rows == GSR_LAYOUT_ROW_MAJOR
    _check(lib().gsr_embed_lookup(table.data_ptr(), vocab, ldt, _dtype_of(table), ids.data_ptr(), _tokens(ids, n, dev), n, d, c, layout,
                                  _dtype_of(x_out), scale, x_out.data_ptr(), ldx, _stream()))


def gsr_embed_grad_workspace(n: int, vocab: int, d: int) -> int:
    """Bytes of workspace that gsr_embed_grad needs for n rows of d columns."""
    return lib().gsr_embed_grad_workspace(n, vocab, d)


def gsr_embed_grad(ids, dx, dtable_out, scale: float = 1.0, workspace=None) -> None:
    """dtable_out[t] = scale * sum of dx[i] over ids[i] == t (float32 [vocab, D], rows may be strided; written whole).  dx: a plane as
    gsr_embed_lookup's x_out; workspace: device tensor of gsr_embed_grad_workspace(n, vocab, D) bytes, or None."""
    import torch
    dev = _current_device()
    n, d, c, layout, ldx = _plane(dx, dev)
    vocab, dt, _, rows, ldt = _plane(dtable_out, dev)
    assert dt == d and rows == GSR_LAYOUT_ROW_MAJOR and dtable_out.dtype == torch.float32
    if workspace is None:
        workspace = torch.empty(gsr_embed_grad_workspace(n, vocab, d), dtype=torch.uint8, device=dx.device)
    assert workspace.get_device() == dev and workspace.is_contiguous()
    _check(lib().gsr_embed_grad(ids.data_ptr(), _tokens(ids, n, dev), n, dx.data_ptr(), ldx, d, c, layout, _dtype_of(dx), scale, vocab,
                                dtable_out.data_ptr(), ldt, workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream()))


_marshal = None
_REFUSED = ("", "a list or tuple of tensors", "a tensor", "a tensor on the current device", "a tensor of the list's type (float32, or bfloat16)",
            "contiguous", "of the size that the other lists have there")


def _marshal_list():
    """The helper that reads lists of tensors.  Raises if it has not been built."""
    global _marshal
    if _marshal is None:
        import torch  # noqa: F401  (the helper uses its libraries)
        if not os.path.exists(MARSHAL_PATH):
            raise GsrError(-1, f"{MARSHAL_PATH} is missing: build it with `python -m paper_2603_27156_amd.build`")
        f = C.PyDLL(MARSHAL_PATH).gsr_marshal_list
        f.restype = C.c_int
        f.argtypes = [C.py_object, C.c_int64, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]
        _marshal = f
    return _marshal


def _addresses(tensors, dtype: int, dev: int, counts=None):
    """(addresses, sizes) of a list of contiguous tensors of one type on GPU `dev`; `counts`: the sizes that they must have."""
    n = len(tensors)
    if counts is not None and len(counts) != n:
        raise TypeError("lists of different lengths")
    at, which = array("Q", bytes(8 * n)), array("q", (0,))
    sizes = array("q", bytes(8 * n)) if counts is None else counts
    why = _marshal_list()(tensors, n, dev, dtype, counts is not None, _at(at), _at(sizes), _at(which))
    if why:
        raise TypeError(f"tensor {which[0]} of the list is not {_REFUSED[why]}")
    return at, sizes


def _at(a: array) -> int:
    return a.buffer_info()[0]


def _list_type(tensors) -> int:
    return _dtype_of(tensors[0]) if len(tensors) else GSR_F32


def _norm_workspace(counts, workspace, dev: int):
    if workspace is None:
        import torch
        nbytes = lib().gsr_grad_norm_workspace(_at(counts), len(counts))
        return torch.empty(nbytes, dtype=torch.uint8, device="cuda"), nbytes
    assert workspace.get_device() == dev and workspace.is_contiguous()
    return workspace, workspace.numel() * workspace.element_size()


def gsr_grad_norm_workspace(grads) -> int:
    """Bytes of workspace that gsr_grad_norm and gsr_grad_clip need for this list."""
    counts = array("q", [t.numel() for t in grads])
    return lib().gsr_grad_norm_workspace(_at(counts), len(counts))


def _scalar(t, dev: int) -> int:
    import torch
    if t is None:
        return 0
    assert t.get_device() == dev and t.dtype == torch.float32 and t.numel() == 1
    return t.data_ptr()


def gsr_grad_norm(grads, norm_out, workspace=None) -> None:
    """norm_out (float32, one element) = the 2-norm over all elements of a list of tensors (float32, or all bfloat16)."""
    dev, dtype = _current_device(), _list_type(grads)
    at, counts = _addresses(grads, dtype, dev)
    ws, nb = _norm_workspace(counts, workspace, dev)
    _check(lib().gsr_grad_norm(_at(at), _at(counts), len(counts), dtype, _scalar(norm_out, dev), ws.data_ptr(), nb, _stream()))


def gsr_grad_clip(grads, max_norm: float, norm_out=None, out=None, workspace=None) -> None:
    """Multiplies the tensors of a list by min(1, max_norm / (norm + 1e-6)), in place or into the tensors of `out` (of the same sizes, of
    one type); norm_out (float32, one element): the norm before clipping."""
    dev, dtype = _current_device(), _list_type(grads)
    at, counts = _addresses(grads, dtype, dev)
    to, out_dtype = None, dtype
    if out is not None:
        out_dtype = _list_type(out)
        to, _ = _addresses(out, out_dtype, dev, counts)
    ws, nb = _norm_workspace(counts, workspace, dev)
    _check(lib().gsr_grad_clip(_at(at), _at(counts), len(counts), dtype, max_norm, _scalar(norm_out, dev), None if to is None else _at(to),
                               out_dtype, ws.data_ptr(), nb, _stream()))


def gsr_adam_update_list(w, dw, m, v, t: int, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                         weight_decay: float = 0.0, norm=None, max_norm: Optional[float] = None) -> None:
    """gsr_adam_update on every tensor of four lists, dw (float32, or all bfloat16) multiplied by min(1, max_norm / (norm + 1e-6)) where
    norm, as gsr_grad_norm leaves it on the device, is given; max_norm has to be given with it."""
    if norm is not None and max_norm is None:
        raise TypeError("a norm without max_norm")
    dev, dtype = _current_device(), _list_type(dw)
    aw, counts = _addresses(w, GSR_F32, dev)
    ag, am, av = (_addresses(x, k, dev, counts)[0] for x, k in ((dw, dtype), (m, GSR_F32), (v, GSR_F32)))
    _check(lib().gsr_adam_update_list(_at(aw), _at(ag), _at(am), _at(av), _at(counts), len(counts), dtype, _scalar(norm, dev), max_norm or 0.0, t, lr,
                                      beta1, beta2, eps, weight_decay, _stream()))


def _like_plane(x, dev: int, n: int, d: int, c: int, layout: int, dtype) -> int:
    """Row stride of a plane that has to be of the same rows, columns, layout and type as another."""
    assert x.dtype == dtype
    n2, d2, c2, layout2, ld = _plane(x, dev)
    assert (n2, d2, c2, layout2) == (n, d, c, layout)
    return ld


def _floats(t, dev: int, shape) -> int:
    """Address of a contiguous float32 tensor of this shape, or 0 for None."""
    if t is None:
        return 0
    import torch
    assert t.get_device() == dev and t.dtype == torch.float32 and t.shape == shape and t.is_contiguous()
    return t.data_ptr()


def _checkpoint(codes, scales, dev: int, n: int, d: int, c: int):
    """Addresses of a checkpoint of n rows of d columns in c groups, (0, 0) for none."""
    if codes is None and scales is None:
        return 0, 0
    import torch
    assert codes is not None and scales is not None and codes.get_device() == dev and codes.dtype == torch.int8
    assert scales.get_device() == dev and scales.dtype == torch.float32 and codes.is_contiguous() and scales.is_contiguous()
    assert codes.numel() == n * d and scales.numel() == n * gsr_checkpoint_blocks(d, c)
    return codes.data_ptr(), scales.data_ptr()


def _graph_ptr(graph_ptr, dev: int):
    """(address, whether of 64 bits, graphs)."""
    if graph_ptr is None:
        return 0, 0, 1
    assert graph_ptr.dim() == 1 and len(graph_ptr) >= 1
    return graph_ptr.data_ptr(), _tokens(graph_ptr, len(graph_ptr), dev), len(graph_ptr) - 1


def gsr_group_norm_workspace(x, groups: int, graph_ptr=None) -> int:
    """Bytes of workspace that gsr_group_norm and gsr_group_norm_grad need for a plane like x."""
    n, d, c, layout, _ = _plane(x, x.get_device())
    return lib().gsr_group_norm_workspace(n, 1 if graph_ptr is None else len(graph_ptr) - 1, d, c, layout, _dtype_of(x), groups)


def _norm_scratch(workspace, n: int, graphs: int, d: int, c: int, layout: int, dtype: int, groups: int, dev: int):
    if workspace is None:
        import torch
        workspace = torch.empty(lib().gsr_group_norm_workspace(n, graphs, d, c, layout, dtype, groups), dtype=torch.uint8, device="cuda")
    assert workspace.get_device() == dev and workspace.is_contiguous()
    return workspace, workspace.numel() * workspace.element_size()


def gsr_group_norm(x, y_out, mean_out, rstd_out, gamma=None, beta=None, eps: float = 1e-5, act: int = GSR_ACT_NONE, graph_ptr=None,
                   codes_out=None, scales_out=None, workspace=None) -> None:
    """y_out = act(gamma * (x - mean) * rstd + beta), mean and 1 / sqrt(variance + eps) over the rows of a graph and the columns of a group.

    x, y_out: planes [n, D] (rows may be strided) or [C, n, D/C], both float32 or both bfloat16; y_out may be x.  mean_out, rstd_out: float32
    [graphs, groups].  gamma, beta: float32 [D].  graph_ptr: [graphs + 1] int32 or int64, first rows of the graphs; None: one graph of all rows.
    Rows of no graph are left as they are.  codes_out, scales_out: also the checkpoint of x, as gsr_checkpoint_save leaves it."""
    dev = _current_device()
    n, d, c, layout, ldx = _plane(x, dev)
    dtype = _dtype_of(x)
    ldy = _like_plane(y_out, dev, n, d, c, layout, x.dtype)
    at, i64, graphs = _graph_ptr(graph_ptr, dev)
    groups = mean_out.shape[-1]
    codes, scales = _checkpoint(codes_out, scales_out, dev, n, d, c)
    ws, nb = _norm_scratch(workspace, n, graphs, d, c, layout, dtype, groups, dev)
    _check(lib().gsr_group_norm(x.data_ptr(), ldx, n, d, c, layout, dtype, at, i64, graphs, groups, _floats(gamma, dev, (d,)), _floats(beta, dev, (d,)),
                                eps, act, y_out.data_ptr(), ldy, _floats(mean_out, dev, (graphs, groups)), _floats(rstd_out, dev, (graphs, groups)),
                                codes, scales, ws.data_ptr(), nb, _stream()))


def gsr_group_norm_grad(dy, mean, rstd, dx_out, x=None, codes=None, scales=None, gamma=None, beta=None, act: int = GSR_ACT_NONE, graph_ptr=None,
                        dgamma_out=None, dbeta_out=None, workspace=None) -> None:
    """The gradients of gsr_group_norm: dx_out (a plane as dy, may be dy), dgamma_out and dbeta_out (float32 [D], or None), from mean and rstd as
    it left them and x, or x's checkpoint (codes, scales) in its place."""
    dev = _current_device()
    n, d, c, layout, lddy = _plane(dy, dev)
    dtype = _dtype_of(dy)
    lddx = _like_plane(dx_out, dev, n, d, c, layout, dy.dtype)
    assert (x is None) != (codes is None), "x or its checkpoint"
    ldx = 0 if x is None else _like_plane(x, dev, n, d, c, layout, dy.dtype)
    at, i64, graphs = _graph_ptr(graph_ptr, dev)
    groups = mean.shape[-1]
    k, s = _checkpoint(codes, scales, dev, n, d, c)
    ws, nb = _norm_scratch(workspace, n, graphs, d, c, layout, dtype, groups, dev)
    _check(lib().gsr_group_norm_grad(dy.data_ptr(), lddy, 0 if x is None else x.data_ptr(), ldx, k, s, n, d, c, layout, dtype, at, i64, graphs, groups,
                                     _floats(mean, dev, (graphs, groups)), _floats(rstd, dev, (graphs, groups)), _floats(gamma, dev, (d,)),
                                     _floats(beta, dev, (d,)), act, dx_out.data_ptr(), lddx, _floats(dgamma_out, dev, (d,)), _floats(dbeta_out, dev, (d,)),
                                     ws.data_ptr(), nb, _stream()))


def gsr_checkpoint_blocks(d: int, c: int = 1) -> int:
    """Scales of a row in a checkpoint of planes [n, d] (c = 1) or [c, n, d / c]."""
    return c * -(-(d // c) // GSR_CHECKPOINT_BLOCK)


def gsr_checkpoint_save(x, codes_out, scales_out) -> None:
    """A plane ([n, D], rows may be strided, or [C, n, D/C]; float32 or bfloat16) in 8 bits: codes_out int8, n * D of them, and scales_out float32,
    n * gsr_checkpoint_blocks(D, C), contiguous and of any shape: they hold [n, D] and [n, blocks], or [C, n, D/C] and [C, n, blocks of a group]."""
    dev = _current_device()
    n, d, c, layout, ldx = _plane(x, dev)
    codes, scales = _checkpoint(codes_out, scales_out, dev, n, d, c)
    _check(lib().gsr_checkpoint_save(x.data_ptr(), ldx, n, d, c, layout, _dtype_of(x), codes, scales, _stream()))


def gsr_checkpoint_load(codes, scales, x_out) -> None:
    """The plane that gsr_checkpoint_save put away, every value as code * scale."""
    dev = _current_device()
    n, d, c, layout, ldx = _plane(x_out, dev)
    k, s = _checkpoint(codes, scales, dev, n, d, c)
    _check(lib().gsr_checkpoint_load(k, s, n, d, c, layout, _dtype_of(x_out), x_out.data_ptr(), ldx, _stream()))


def gsr_class_loss_workspace(x, classes: int) -> int:
    """Bytes of workspace that gsr_class_loss needs for a plane like x."""
    n, d, *_ = _plane(x, x.get_device())
    return lib().gsr_class_loss_workspace(n, classes, d, _dtype_of(x))


def gsr_class_grad_workspace(x, classes: int) -> int:
    """Bytes of workspace that gsr_class_grad needs for a plane like x."""
    n, d, *_ = _plane(x, x.get_device())
    return lib().gsr_class_grad_workspace(n, classes, d, _dtype_of(x))


def _class_table(t, d: int, dtype, dev: int):
    """(address, rows, row stride) of a table [classes, d] of a type; rows may be strided."""
    assert t.dtype == dtype
    classes, dt, _, layout, ld = _plane(t, dev)
    assert dt == d and layout == GSR_LAYOUT_ROW_MAJOR
    return t.data_ptr(), classes, ld


def _class_scratch(workspace, size, n: int, classes: int, d: int, dtype: int, dev: int):
    if workspace is None:
        import torch
        workspace = torch.empty(size(n, classes, d, dtype), dtype=torch.uint8, device="cuda")
    assert workspace.get_device() == dev and workspace.is_contiguous()
    return workspace, workspace.numel() * workspace.element_size()


def gsr_class_loss(x, table, targets, loss_out, lse_out, bias=None, workspace=None) -> None:
    """loss_out (float32, one element) = mean over the rows with a class of lse - logit of the class, where the logits x @ table.T + bias are
    never stored; lse_out (float32 [n]): log sum exp of every row's.  x: a plane [n, D] (rows may be strided) or [C, n, D/C]; table: [classes, D]
    of x's type, rows may be strided; targets: [n] int32 or int64, no class where outside [0, classes); bias: float32 [classes] or None."""
    dev = _current_device()
    n, d, c, layout, ldx = _plane(x, dev)
    dtype = _dtype_of(x)
    at, classes, ldt = _class_table(table, d, x.dtype, dev)
    ws, nb = _class_scratch(workspace, lib().gsr_class_loss_workspace, n, classes, d, dtype, dev)
    _check(lib().gsr_class_loss(x.data_ptr(), ldx, n, d, c, layout, dtype, at, classes, ldt, _floats(bias, dev, (classes,)), targets.data_ptr(),
                                _tokens(targets, n, dev), _scalar(loss_out, dev), _floats(lse_out, dev, (n,)), ws.data_ptr(), nb, _stream()))


def gsr_class_grad(x, table, targets, lse, dx_out=None, dtable_out=None, bias=None, dbias_out=None, scale: float = 1.0, workspace=None) -> None:
    """The gradients of scale * gsr_class_loss, lse as it left it: dx_out (a plane as x), dtable_out (as table), dbias_out (float32
    [classes]); at least one of them."""
    dev = _current_device()
    n, d, c, layout, ldx = _plane(x, dev)
    dtype = _dtype_of(x)
    at, classes, ldt = _class_table(table, d, x.dtype, dev)
    lddx = 0 if dx_out is None else _like_plane(dx_out, dev, n, d, c, layout, x.dtype)
    dt, rows, lddt = (0, classes, 0) if dtable_out is None else _class_table(dtable_out, d, x.dtype, dev)
    assert rows == classes
    ws, nb = _class_scratch(workspace, lib().gsr_class_grad_workspace, n, classes, d, dtype, dev)
    _check(lib().gsr_class_grad(x.data_ptr(), ldx, n, d, c, layout, dtype, at, classes, ldt, _floats(bias, dev, (classes,)), targets.data_ptr(),
                                _tokens(targets, n, dev), _floats(lse, dev, (n,)), scale, 0 if dx_out is None else dx_out.data_ptr(), lddx, dt, lddt,
                                _floats(dbias_out, dev, (classes,)), ws.data_ptr(), nb, _stream()))


def gsr_spmm_compressed(g: Graph, vals, idx, dg: int):
    """A * scatter(V, I) -> dense float32 [n, dg]."""
    import torch
    assert vals.is_cuda and idx.is_cuda and idx.dtype == torch.int32 and vals.is_contiguous() and idx.is_contiguous()
    n, k = vals.shape
    h = torch.empty((n, dg), dtype=torch.float32, device=vals.device)
    nbytes = lib().gsr_spmm_compressed_workspace(g.ptr, C.c_int32(k), C.c_int32(dg))
    ws = torch.empty(max(1, nbytes), dtype=torch.uint8, device=vals.device)
    _check(lib().gsr_spmm_compressed(g.ptr, _dp(vals), _dp(idx), C.c_int32(k), C.c_int32(dg),
                                     C.c_int32(_dtype_of(vals)), _dp(h), _dp(ws), C.c_size_t(nbytes), _stream()))
    return h


def gsr_workspace_size(g: Graph, cfg: Config) -> Tuple[int, int]:
    """(bytes for the layer calls, bytes for gsr_step)."""
    lb, sb = C.c_size_t(), C.c_size_t()
    cs = cfg.c_struct()
    _check(lib().gsr_workspace_size(C.byref(cs), g.ptr, C.byref(lb), C.byref(sb)))
    return lb.value, sb.value


def _workspace(g: Graph, cfg: Config, workspace, step: bool, device):
    import torch
    need = gsr_workspace_size(g, cfg)[1 if step else 0]
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    return workspace, workspace.numel() * workspace.element_size()


def gsr_layer_forward(g: Graph, cfg: Config, w, x_inout, workspace=None) -> None:
    ws, nb = _workspace(g, cfg, workspace, False, x_inout.device)
    cs = cfg.c_struct()
    _check(lib().gsr_layer_forward(g.ptr, C.byref(cs), _dp(w), _dp(x_inout), _dp(ws), C.c_size_t(nb), _stream()))


def gsr_layer_inverse(g: Graph, cfg: Config, w, y_inout, workspace=None) -> None:
    ws, nb = _workspace(g, cfg, workspace, False, y_inout.device)
    cs = cfg.c_struct()
    _check(lib().gsr_layer_inverse(g.ptr, C.byref(cs), _dp(w), _dp(y_inout), _dp(ws), C.c_size_t(nb), _stream()))


def gsr_layer_backward(g: Graph, cfg: Config, w, y_inout, dy_inout, dw_out, workspace=None) -> None:
    ws, nb = _workspace(g, cfg, workspace, False, y_inout.device)
    cs = cfg.c_struct()
    _check(lib().gsr_layer_backward(g.ptr, C.byref(cs), _dp(w), _dp(y_inout), _dp(dy_inout), _dp(dw_out), _dp(ws),
                                    C.c_size_t(nb), _stream()))


def gsr_step(g: Graph, cfg: Config, x0, w_all, w_out, b_out, target, loss_out, dw_all, dw_out, db_out,
             yhat_out=None, dx0_out=None, x0_rebuilt_out=None, xl_out=None, workspace=None) -> None:
    """All tensors are caller-allocated device tensors (see include/gsr.h for shapes)."""
    ws, nb = _workspace(g, cfg, workspace, True, x0.device)
    cs = cfg.c_struct()
    _check(lib().gsr_step(g.ptr, C.byref(cs), _dp(x0), _dp(w_all), _dp(w_out), _dp(b_out), _dp(target), _dp(loss_out),
                          _dp(yhat_out), _dp(dw_all), _dp(dw_out), _dp(db_out), _dp(dx0_out), _dp(x0_rebuilt_out),
                          _dp(xl_out), _dp(ws), C.c_size_t(nb), _stream()))


def gsr_step_tie_stats(g: Graph, cfg: Config, workspace) -> dict:
    """Counts of the last gsr_step with save_indices == 2 in `workspace`: rows kept, most per block, rows dropped."""
    a, b, c = C.c_int64(), C.c_int64(), C.c_int64()
    cs = cfg.c_struct()
    _check(lib().gsr_step_tie_stats(g.ptr, C.byref(cs), _dp(workspace), C.byref(a), C.byref(b), C.byref(c), _stream()))
    return dict(listed=a.value, max_per_block=b.value, dropped=c.value)


def gsr_step_tie_export(g: Graph, cfg: Config, workspace, layer: int, block: int):
    """(rows int32 [m], masks uint64 [m]) kept by the last save_indices == 2 step for the input of `block` of `layer`."""
    cap = cfg.tie_capacity if cfg.tie_capacity > 0 else cfg.n // 32 + 1024
    cap = (cap + 15) // 16 * 16                    # the library keeps sixteen sub-lists of cap / 16 places, rounded up
    rows = np.zeros(cap, dtype=np.int32)
    masks = np.zeros(cap, dtype=np.uint64)
    cnt = C.c_int64()
    cs = cfg.c_struct()
    _check(lib().gsr_step_tie_export(g.ptr, C.byref(cs), _dp(workspace), C.c_int32(layer), C.c_int32(block), _np(rows),
                                     _np(masks), C.byref(cnt), _stream()))
    return rows[:cnt.value].copy(), masks[:cnt.value].copy()
