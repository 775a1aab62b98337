"""ctypes binding of libgmeta.so: argument marshalling only.

Every step of the MAML-DLRM path runs inside the library's HIP kernels; PyTorch
is used here for device memory (torch.empty on the GPU) and nothing else.
There is no CPU fallback: if the shared library is missing, loading fails.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, List, Optional, Sequence

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgmeta.so")

GM_OK, GM_ERR_ARG, GM_ERR_INDEX, GM_ERR_CAPACITY, GM_ERR_WORKSPACE, GM_ERR_HIP = 0, -1, -2, -3, -4, -5

EXPORTS = ["gm_create", "gm_destroy", "gm_last_error", "gm_workspace_bytes", "gm_meta_step", "gm_meta_step_static",
           "gm_meta_train_step", "gm_meta_train_step_table", "gm_meta_train", "gm_group_batch", "gm_scatter_add", "gm_gather_pool", "gm_index_prep", "gm_configure", "gm_profile", "gm_profile_report", "gm_ceilings",
           "gm_wait", "gm_seq_embed", "gm_seq_embed_grad", "gm_seq_embed_grad_bytes", "gm_seq_scan", "gm_seq_scan_grad", "gm_seq_scan_bytes",
           "gm_seq_scan_step", "gm_seq_attend", "gm_seq_attend_grad", "gm_seq_attend_bytes"]


class gm_model_desc(C.Structure):
    _fields_ = [("n_fields", C.c_int32), ("rows_per_field", C.POINTER(C.c_int64)),
                ("emb_dim", C.c_int32), ("n_dense", C.c_int32), ("n_layers", C.c_int32),
                ("layer_dims", C.POINTER(C.c_int32)), ("mlp_dtype", C.c_int32)]


class gm_set(C.Structure):
    _fields_ = [("n_samples", C.c_int64), ("nnz", C.c_int64), ("task_offsets", C.POINTER(C.c_int64)),
                ("bag_offsets", C.c_void_p), ("indices", C.c_void_p), ("dense", C.c_void_p),
                ("labels", C.c_void_p)]


class gm_params(C.Structure):
    _fields_ = [("emb", C.c_void_p), ("W", C.POINTER(C.c_void_p)), ("b", C.POINTER(C.c_void_p))]


class gm_grads(C.Structure):
    _fields_ = [("dW", C.POINTER(C.c_void_p)), ("db", C.POINTER(C.c_void_p)), ("emb_rows", C.c_void_p),
                ("emb_grad", C.c_void_p), ("n_emb_rows", C.c_void_p), ("emb_rows_capacity", C.c_int64),
                ("task_loss", C.c_void_p), ("emb_grad_table", C.c_void_p)]


class gm_set_buffers(C.Structure):
    _fields_ = [("n_samples", C.c_int64), ("nnz", C.c_int64), ("task_offsets", C.POINTER(C.c_int64)),
                ("bag_offsets", C.c_void_p), ("indices", C.c_void_p), ("dense", C.c_void_p), ("labels", C.c_void_p)]


class gm_seq(C.Structure):
    _fields_ = [("n_seqs", C.c_int64), ("n_rows", C.c_int64), ("longest", C.c_int64), ("offsets", C.c_void_p), ("lengths", C.c_void_p)]


class gm_seq_heads(C.Structure):
    _fields_ = [("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32), ("scale", C.c_float)]


class GMetaError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"gmeta error {code}: {msg}")
        self.code = code


_lib = None


def load_library() -> C.CDLL:
    """Loads libgmeta.so (built in-tree by paper_2401_04338_amd.build); raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} is not built; run `python -m paper_2401_04338_amd.build` (there is no fallback path)")
    lib = C.CDLL(LIB_PATH)
    lib.gm_create.restype = C.c_int
    lib.gm_create.argtypes = [C.POINTER(C.c_void_p), C.POINTER(gm_model_desc), C.c_int, C.c_void_p, C.c_size_t]
    lib.gm_destroy.restype = None
    lib.gm_destroy.argtypes = [C.c_void_p]
    lib.gm_last_error.restype = C.c_char_p
    lib.gm_last_error.argtypes = [C.c_void_p]
    lib.gm_workspace_bytes.restype = C.c_size_t
    lib.gm_workspace_bytes.argtypes = [C.POINTER(gm_model_desc), C.c_int32, C.c_int64, C.c_int64, C.c_int64,
                                       C.c_int64, C.c_int32, C.c_int32]
    lib.gm_group_batch.restype = C.c_int
    lib.gm_group_batch.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.POINTER(C.c_int64), C.POINTER(C.c_int64), C.c_void_p,
                                   C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.POINTER(gm_set_buffers),
                                   C.POINTER(gm_set_buffers), C.POINTER(C.c_int32)]
    lib.gm_meta_train_step.restype = C.c_int
    lib.gm_meta_train_step.argtypes = [C.c_void_p, C.c_int32, C.POINTER(gm_set), C.POINTER(gm_set), C.POINTER(gm_params),
                                       C.c_float, C.c_int32, C.c_int32, C.c_float, C.c_void_p, C.c_void_p]
    lib.gm_meta_train_step_table.restype = C.c_int
    lib.gm_meta_train_step_table.argtypes = [C.c_void_p, C.c_int32, C.POINTER(gm_set), C.POINTER(gm_set), C.POINTER(gm_params),
                                             C.c_float, C.c_int32, C.c_int32, C.c_float, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.gm_meta_train.restype = C.c_int
    lib.gm_meta_train.argtypes = [C.c_void_p, C.c_int32, C.POINTER(C.c_int32), C.POINTER(gm_set), C.POINTER(gm_set),
                                  C.POINTER(gm_params), C.c_float, C.c_int32, C.c_int32, C.c_float, C.c_void_p,
                                  C.POINTER(C.c_int32)]
    lib.gm_meta_step.restype = C.c_int
    lib.gm_meta_step.argtypes = [C.c_void_p, C.c_int32, C.POINTER(gm_set), C.POINTER(gm_set),
                                 C.POINTER(gm_params), C.c_float, C.c_int32, C.c_int32, C.c_void_p,
                                 C.POINTER(gm_grads)]
    lib.gm_meta_step_static.restype = C.c_int
    lib.gm_meta_step_static.argtypes = lib.gm_meta_step.argtypes
    lib.gm_scatter_add.restype = C.c_int
    lib.gm_scatter_add.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_float]
    lib.gm_gather_pool.restype = C.c_int
    lib.gm_gather_pool.argtypes = [C.c_void_p, C.c_int32, C.POINTER(gm_set), C.c_void_p, C.c_void_p]
    lib.gm_index_prep.restype = C.c_int
    lib.gm_index_prep.argtypes = [C.c_void_p, C.c_int32, C.POINTER(gm_set), C.POINTER(gm_set)] + [C.c_void_p] * 7 + [C.c_int64]
    lib.gm_configure.restype = C.c_int
    lib.gm_configure.argtypes = [C.c_void_p, C.c_char_p, C.c_int64]
    lib.gm_profile.restype = C.c_int
    lib.gm_profile.argtypes = [C.c_void_p, C.c_int]
    lib.gm_profile_report.restype = C.c_char_p
    lib.gm_profile_report.argtypes = [C.c_void_p]
    lib.gm_ceilings.restype = C.c_int
    lib.gm_ceilings.argtypes = [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_double), C.POINTER(C.c_double),
                                C.POINTER(C.c_double), C.POINTER(C.c_int64)]
    p, i32, i64, f32, seq = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.POINTER(gm_seq)
    rows = [p, i64]   # an array and its row stride
    for name, args in (("gm_wait", [p]),
                       ("gm_seq_embed", [p, i64, p, i64, i32, p, f32, i32] + rows),
                       ("gm_seq_embed_grad", [p, i64, p, i64, i32, i32] + rows + [f32, p, p, p, i64, p]),
                       ("gm_seq_scan", [p, seq, i32, i32] + rows * 2 + [p] + rows + [p]),
                       ("gm_seq_scan_grad", [p, seq, i32, i32] + rows * 3 + [p] + rows + [p] + rows * 2 + [p]),
                       ("gm_seq_scan_step", [p, i64, i32, i32] + rows * 2 + [p] + rows),
                       ("gm_seq_attend", [p, seq, seq, C.POINTER(gm_seq_heads)] + rows * 3 + [p] + rows + [p]),
                       ("gm_seq_attend_grad", [p, seq, seq, C.POINTER(gm_seq_heads)] + rows * 5 + [p, p] + rows * 3)):
        getattr(lib, name).restype = C.c_int
        getattr(lib, name).argtypes = args
    for name, args in (("gm_seq_embed_grad_bytes", [i64, i32]), ("gm_seq_scan_bytes", [i64, i64, i32, i32]),
                       ("gm_seq_attend_bytes", [p, seq, seq, C.POINTER(gm_seq_heads), i32])):
        getattr(lib, name).restype = C.c_size_t
        getattr(lib, name).argtypes = args
    _lib = lib
    return lib


def _model_desc(n_fields, rows_per_field, emb_dim, n_dense, layer_dims, mlp_dtype):
    rows = (C.c_int64 * max(n_fields, 1))(*[int(r) for r in rows_per_field])
    dims = (C.c_int32 * len(layer_dims))(*[int(d) for d in layer_dims])
    m = gm_model_desc(n_fields, rows, emb_dim, n_dense, len(layer_dims) - 1, dims, mlp_dtype)
    m._keep = (rows, dims)
    return m


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


def _checked(t: torch.Tensor, dtype, name: str, device=None) -> torch.Tensor:
    """The library reads raw pointers: a tensor of another type, layout or device would be misread silently."""
    if t.dtype != dtype or not t.is_contiguous() or not t.is_cuda or (device is not None and t.device != device):
        raise ValueError(f"{name} must be a contiguous {dtype} tensor on {device or 'the GPU'} "
                         f"(got {t.dtype}, contiguous={t.is_contiguous()}, device={t.device})")
    return t


def _set_struct(s, device=None) -> gm_set:
    """s: an object with task_offsets (host numpy int64), bag_offsets, indices, dense, labels (device tensors)."""
    _checked(s.bag_offsets, torch.int64, "bag_offsets", device)
    _checked(s.indices, torch.int32, "indices", device)
    _checked(s.dense, torch.float32, "dense", device)
    _checked(s.labels, torch.float32, "labels", device)
    toff = np.ascontiguousarray(np.asarray(s.task_offsets, dtype=np.int64))
    st = gm_set(int(toff[-1]), int(s.indices.numel()), toff.ctypes.data_as(C.POINTER(C.c_int64)),
                _ptr(s.bag_offsets), _ptr(s.indices), _ptr(s.dense), _ptr(s.labels))
    st._keep = (toff, s)
    return st


def _current_stream(device: torch.device) -> int:
    """Handle of torch's current stream (without the stream object, which takes longer to make than a small call's kernel runs)."""
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(device.index) if raw else torch.cuda.current_stream(device).cuda_stream


_SEQ_DTYPES = {torch.float32: 0, torch.bfloat16: 1}


def _rows(t: torch.Tensor, name: str, dtype, device, shape) -> tuple:
    """(pointer, row stride) of a tensor whose rows may lie apart but are contiguous themselves."""
    if t.shape != shape or t.dtype is not dtype or t.device != device:
        raise ValueError(f"{name} must be a {dtype} tensor {list(shape)} on {device} (got {t.dtype} {list(t.shape)} on {t.device})")
    if t.is_contiguous():
        return t.data_ptr(), shape[1] if len(shape) == 2 else shape[1] * shape[2]
    inner = 1
    for n, s in zip(reversed(shape[1:]), reversed(t.stride()[1:])):
        if n != 1 and s != inner:
            raise ValueError(f"{name}: a row must be contiguous (strides {t.stride()})")
        inner *= n
    return t.data_ptr(), t.stride(0) if shape[0] > 1 else inner


def _state(t: Optional[torch.Tensor], name: str, device, shape):
    """Pointer of a contiguous fp32 tensor of that shape, or None."""
    if t is None:
        return None
    _checked(t, torch.float32, name, device)
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {list(shape)} (got {list(t.shape)})")
    return t.data_ptr()


class GMeta:
    """One context of the library: model shape + workspace on one GPU."""

    def __init__(self, n_fields: int, rows_per_field: Sequence[int], emb_dim: int, n_dense: int,
                 layer_dims: Sequence[int], mlp_dtype: int = 0, device: int = 0,
                 workspace_bytes: int = 1 << 30, stream: Optional[int] = None):
        self.lib = load_library()
        self.n_fields, self.emb_dim, self.n_dense = n_fields, emb_dim, n_dense
        self.layer_dims = list(layer_dims)
        self.rows_per_field = list(rows_per_field)
        self.device = torch.device("cuda", device)
        self._stream, self._own_stream = int(stream or 0), None
        self._desc = _model_desc(n_fields, rows_per_field, emb_dim, n_dense, layer_dims, mlp_dtype)
        self._ctx = C.c_void_p()
        rc = self.lib.gm_create(C.byref(self._ctx), C.byref(self._desc), device,
                                C.c_void_p(stream) if stream else None, workspace_bytes)
        if rc != GM_OK:
            msg = self.lib.gm_last_error(self._ctx).decode() if self._ctx else "gm_create failed"
            if self._ctx:
                self.lib.gm_destroy(self._ctx)
                self._ctx = C.c_void_p()
            raise GMetaError(rc, msg)

    @classmethod
    def from_config(cls, cfg, device: int = 0, workspace_bytes: int = 1 << 30, stream=None, mlp_dtype=None):
        return cls(cfg.n_fields, [cfg.rows_per_field] * cfg.n_fields, cfg.emb_dim, cfg.n_dense, cfg.layer_dims,
                   cfg.mlp_dtype if mlp_dtype is None else mlp_dtype, device, workspace_bytes, stream)

    def workspace_bytes(self, n_tasks, n_support, n_query, nnz_support, nnz_query, inner_steps, order) -> int:
        return int(self.lib.gm_workspace_bytes(C.byref(self._desc), n_tasks, n_support, n_query, nnz_support,
                                               nnz_query, inner_steps, order))

    def close(self):
        if getattr(self, "_ctx", None):
            self.lib.gm_destroy(self._ctx)
            self._ctx = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc: int):
        if rc != GM_OK:
            raise GMetaError(rc, self.lib.gm_last_error(self._ctx).decode())

    def _check_params(self, params):
        L = len(self.layer_dims) - 1
        if self.n_fields > 0:
            _checked(params.emb, torch.float32, "params.emb", self.device)
            if tuple(params.emb.shape) != (int(sum(self.rows_per_field)), self.emb_dim):
                raise ValueError("params.emb must be [sum rows_per_field, emb_dim]")
        if len(params.W) != L or len(params.b) != L:
            raise ValueError("params.W / params.b must hold one tensor per layer")
        for l in range(L):
            _checked(params.W[l], torch.float32, f"params.W[{l}]", self.device)
            _checked(params.b[l], torch.float32, f"params.b[{l}]", self.device)
            if tuple(params.W[l].shape) != (self.layer_dims[l], self.layer_dims[l + 1]) or params.b[l].numel() != self.layer_dims[l + 1]:
                raise ValueError(f"layer {l}: W must be [{self.layer_dims[l]}, {self.layer_dims[l + 1]}] and b [{self.layer_dims[l + 1]}]")

    # ------------------------------------------------------------------ entry points
    def alloc_outputs(self, n_tasks: int, emb_rows_capacity: int) -> Dict[str, object]:
        dev, L = self.device, len(self.layer_dims) - 1
        return dict(
            loss=torch.empty(1, dtype=torch.float32, device=dev),
            task_loss=torch.empty(max(n_tasks, 1), dtype=torch.float32, device=dev),
            dW=[torch.empty(self.layer_dims[l], self.layer_dims[l + 1], dtype=torch.float32, device=dev) for l in range(L)],
            db=[torch.empty(self.layer_dims[l + 1], dtype=torch.float32, device=dev) for l in range(L)],
            emb_rows=torch.empty(max(emb_rows_capacity, 1), dtype=torch.int64, device=dev),
            emb_grad=torch.empty(max(emb_rows_capacity, 1), self.emb_dim, dtype=torch.float32, device=dev),
            n_emb_rows=torch.zeros(1, dtype=torch.int64, device=dev),
            capacity=emb_rows_capacity)

    def meta_step(self, support, query, params, inner_lr: float, inner_steps: int, order: int,
                  out: Optional[Dict[str, object]] = None, emb_rows_capacity: Optional[int] = None,
                  emb_grad_table: Optional[torch.Tensor] = None, static_scratch: bool = False):
        """gm_meta_step.  support/query: SetData-like; params: object with emb, W[], b[] device tensors.
        emb_grad_table: a float32 device tensor shaped like params.emb that the sparse gradient is added to
        (then no row list is produced).  static_scratch: call gm_meta_step_static instead (the library's static
        scratch array in place of the context's workspace; pass `out` to keep the call itself free of allocations)."""
        n_tasks = len(support.task_offsets) - 1
        if emb_grad_table is not None:
            if (emb_grad_table.dtype != torch.float32 or not emb_grad_table.is_contiguous()
                    or tuple(emb_grad_table.shape) != (int(sum(self.rows_per_field)), self.emb_dim)
                    or emb_grad_table.device != params.emb.device):
                raise ValueError("emb_grad_table must be a contiguous float32 [sum rows_per_field, emb_dim] device tensor")
        if out is None:
            cap = emb_rows_capacity
            if emb_grad_table is not None:
                cap = 0
            elif cap is None:
                cap = min(int(support.indices.numel() + query.indices.numel()), int(sum(self.rows_per_field)))
            out = self.alloc_outputs(n_tasks, cap)
        L = len(self.layer_dims) - 1
        ss, qs = _set_struct(support, self.device), _set_struct(query, self.device)
        self._check_params(params)
        Wp = (C.c_void_p * L)(*[w.data_ptr() for w in params.W])
        bp = (C.c_void_p * L)(*[x.data_ptr() for x in params.b])
        ps = gm_params(_ptr(params.emb), Wp, bp)
        dWp = (C.c_void_p * L)(*[w.data_ptr() for w in out["dW"]])
        dbp = (C.c_void_p * L)(*[x.data_ptr() for x in out["db"]])
        gs = gm_grads(dWp, dbp, _ptr(out["emb_rows"]), _ptr(out["emb_grad"]), _ptr(out["n_emb_rows"]),
                      int(out["capacity"]), _ptr(out["task_loss"]),
                      _ptr(emb_grad_table) if emb_grad_table is not None else None)
        entry = self.lib.gm_meta_step_static if static_scratch else self.lib.gm_meta_step
        rc = entry(self._ctx, n_tasks, C.byref(ss), C.byref(qs), C.byref(ps), float(inner_lr),
                   int(inner_steps), int(order), _ptr(out["loss"]), C.byref(gs))
        self._check(rc)
        return out

    def meta_train_step(self, support, query, params, inner_lr: float, inner_steps: int, order: int, outer_lr: float,
                        loss: Optional[torch.Tensor] = None, task_loss: Optional[torch.Tensor] = None):
        """gm_meta_train_step: the step and the outer update; params.emb / W[] / b[] are updated in place.
        Returns the device scalar holding the step's loss."""
        n_tasks = len(support.task_offsets) - 1
        L = len(self.layer_dims) - 1
        if loss is None:
            loss = torch.empty(1, dtype=torch.float32, device=self.device)
        ss, qs = _set_struct(support, self.device), _set_struct(query, self.device)
        self._check_params(params)
        Wp = (C.c_void_p * L)(*[w.data_ptr() for w in params.W])
        bp = (C.c_void_p * L)(*[x.data_ptr() for x in params.b])
        ps = gm_params(_ptr(params.emb), Wp, bp)
        rc = self.lib.gm_meta_train_step(self._ctx, n_tasks, C.byref(ss), C.byref(qs), C.byref(ps), float(inner_lr),
                                         int(inner_steps), int(order), float(outer_lr), _ptr(loss), _ptr(task_loss))
        self._check(rc)
        return loss

    def meta_train_step_table(self, support, query, params, inner_lr: float, inner_steps: int, order: int, outer_lr: float,
                              emb_grad_table: torch.Tensor, loss: Optional[torch.Tensor] = None,
                              task_loss: Optional[torch.Tensor] = None):
        """gm_meta_train_step_table: the step with the table-shaped sparse meta-gradient (all zero on entry and again on
        return) and the outer update; params.emb / W[] / b[] are updated in place.  Returns the device scalar of the loss."""
        n_tasks = len(support.task_offsets) - 1
        L = len(self.layer_dims) - 1
        if loss is None:
            loss = torch.empty(1, dtype=torch.float32, device=self.device)
        ss, qs = _set_struct(support, self.device), _set_struct(query, self.device)
        self._check_params(params)
        assert emb_grad_table.dtype == torch.float32 and emb_grad_table.is_contiguous() and emb_grad_table.shape == params.emb.shape
        Wp = (C.c_void_p * L)(*[w.data_ptr() for w in params.W])
        bp = (C.c_void_p * L)(*[x.data_ptr() for x in params.b])
        ps = gm_params(_ptr(params.emb), Wp, bp)
        rc = self.lib.gm_meta_train_step_table(self._ctx, n_tasks, C.byref(ss), C.byref(qs), C.byref(ps), float(inner_lr),
                                               int(inner_steps), int(order), float(outer_lr), _ptr(loss), _ptr(task_loss),
                                               _ptr(emb_grad_table))
        self._check(rc)
        return loss

    def meta_train(self, batches, params, inner_lr: float, inner_steps: int, order: int, outer_lr: float,
                   losses: Optional[torch.Tensor] = None):
        """gm_meta_train: one iteration per (support, query) pair of `batches`, parameters updated in place, the index
        side of each batch prepared while the previous one computes.  Returns the device tensor of the steps' losses."""
        n = len(batches)
        L = len(self.layer_dims) - 1
        if losses is None:
            losses = torch.empty(max(n, 1), dtype=torch.float32, device=self.device)
        self._check_params(params)
        sup = (gm_set * max(n, 1))()
        qry = (gm_set * max(n, 1))()
        keep = []
        nt = (C.c_int32 * max(n, 1))()
        for i, (s, q) in enumerate(batches):
            ss, qs = _set_struct(s, self.device), _set_struct(q, self.device)
            keep.append((ss, qs))
            for f, _t in gm_set._fields_:
                setattr(sup[i], f, getattr(ss, f))
                setattr(qry[i], f, getattr(qs, f))
            nt[i] = len(s.task_offsets) - 1
        Wp = (C.c_void_p * L)(*[w.data_ptr() for w in params.W])
        bp = (C.c_void_p * L)(*[x.data_ptr() for x in params.b])
        ps = gm_params(_ptr(params.emb), Wp, bp)
        done = C.c_int32(0)
        rc = self.lib.gm_meta_train(self._ctx, n, nt, sup, qry, C.byref(ps), float(inner_lr), int(inner_steps), int(order),
                                    float(outer_lr), _ptr(losses), C.byref(done))
        self.iterations_done = int(done.value)
        self._check(rc)
        return losses[:n]

    def group_batch(self, task, batch_id, bag_offsets: torch.Tensor, indices: torch.Tensor, dense: torch.Tensor,
                    labels: torch.Tensor, support_num: int, support_den: int):
        """gm_group_batch: task / batch_id host int64 arrays, the other arrays device tensors of the flat stream.
        Returns (support, query) as SetData-like objects (host task_offsets, device tensors)."""
        from types import SimpleNamespace
        task = np.ascontiguousarray(np.asarray(task, dtype=np.int64))
        batch_id = np.ascontiguousarray(np.asarray(batch_id, dtype=np.int64))
        n, nnz, F, nd = int(task.shape[0]), int(indices.numel()), self.n_fields, self.n_dense
        dev = self.device
        outs, structs, toffs = [], [], []
        for _ in range(2):
            o = dict(bag_offsets=torch.empty(n * F + 1, dtype=torch.int64, device=dev),
                     indices=torch.empty(max(nnz, 1), dtype=torch.int32, device=dev),
                     dense=torch.empty(max(n, 1), max(nd, 1), dtype=torch.float32, device=dev),
                     labels=torch.empty(max(n, 1), dtype=torch.float32, device=dev))
            toff = np.zeros(n + 1, dtype=np.int64)
            st = gm_set_buffers(0, 0, toff.ctypes.data_as(C.POINTER(C.c_int64)), _ptr(o["bag_offsets"]), _ptr(o["indices"]),
                                _ptr(o["dense"]), _ptr(o["labels"]))
            outs.append(o); structs.append(st); toffs.append(toff)
        n_tasks = C.c_int32(0)
        rc = self.lib.gm_group_batch(self._ctx, n, nnz, task.ctypes.data_as(C.POINTER(C.c_int64)),
                                     batch_id.ctypes.data_as(C.POINTER(C.c_int64)), _ptr(bag_offsets), _ptr(indices), _ptr(dense),
                                     _ptr(labels), int(support_num), int(support_den), C.byref(structs[0]), C.byref(structs[1]),
                                     C.byref(n_tasks))
        self._check(rc)
        res = []
        for o, st, toff in zip(outs, structs, toffs):
            ns, nz, T = int(st.n_samples), int(st.nnz), int(n_tasks.value)
            sd = SimpleNamespace(task_offsets=toff[: T + 1].copy(), bag_offsets=o["bag_offsets"][: ns * F + 1],
                                 indices=o["indices"][:nz], dense=o["dense"][:ns, :nd], labels=o["labels"][:ns])
            sd.numpy = (lambda d=sd: dict(task_offsets=d.task_offsets, bag_offsets=d.bag_offsets.cpu().numpy(),
                                          indices=d.indices.cpu().numpy(), dense=d.dense.cpu().numpy(),
                                          labels=d.labels.cpu().numpy()))
            res.append(sd)
        return res[0], res[1]

    def gather_pool(self, set_, emb: torch.Tensor) -> torch.Tensor:
        n_tasks = len(set_.task_offsets) - 1
        st = _set_struct(set_, self.device)
        _checked(emb, torch.float32, "emb", self.device)
        x = torch.empty(max(st.n_samples, 1), self.layer_dims[0], dtype=torch.float32, device=self.device)
        self._check(self.lib.gm_gather_pool(self._ctx, n_tasks, C.byref(st), _ptr(emb), _ptr(x)))
        return x[: st.n_samples]

    def index_prep(self, support, query, emb_rows_capacity: Optional[int] = None):
        n_tasks = len(support.task_offsets) - 1
        ss, qs = _set_struct(support, self.device), _set_struct(query, self.device)
        dev, F = self.device, self.n_fields
        cap = emb_rows_capacity
        if cap is None:
            cap = min(ss.nnz + qs.nnz, int(sum(self.rows_per_field)))
        o = dict(slot_counts=torch.zeros(max(n_tasks * F, 1), dtype=torch.int64, device=dev),
                 slot_rows=torch.zeros(max(ss.nnz, 1), dtype=torch.int64, device=dev),
                 sup_slot=torch.zeros(max(ss.nnz, 1), dtype=torch.int32, device=dev),
                 qry_slot=torch.zeros(max(qs.nnz, 1), dtype=torch.int32, device=dev),
                 emb_rows=torch.zeros(max(cap, 1), dtype=torch.int64, device=dev),
                 seg_counts=torch.zeros(max(cap, 1), dtype=torch.int64, device=dev),
                 n_emb_rows=torch.zeros(1, dtype=torch.int64, device=dev))
        rc = self.lib.gm_index_prep(self._ctx, n_tasks, C.byref(ss), C.byref(qs), _ptr(o["slot_counts"]),
                                    _ptr(o["slot_rows"]), _ptr(o["sup_slot"]), _ptr(o["qry_slot"]),
                                    _ptr(o["emb_rows"]), _ptr(o["seg_counts"]), _ptr(o["n_emb_rows"]), cap)
        self._check(rc)
        n = int(o["n_emb_rows"].item())
        ns = int(o["slot_counts"][: n_tasks * F].sum().item())
        return dict(slot_counts=o["slot_counts"][: n_tasks * F], slot_rows=o["slot_rows"][:ns],
                    sup_slot=o["sup_slot"][: ss.nnz], qry_slot=o["qry_slot"][: qs.nnz],
                    emb_rows=o["emb_rows"][:n], seg_counts=o["seg_counts"][:n])

    def configure(self, key: str, value: int):
        self._check(self.lib.gm_configure(self._ctx, key.encode(), int(value)))

    def profile(self, enable: bool):
        self._check(self.lib.gm_profile(self._ctx, 1 if enable else 0))

    def profile_report(self) -> Dict[str, Dict[str, float]]:
        """{family: {launches, ms, bytes, flops}} accumulated since profile(True)."""
        out = {}
        for line in self.lib.gm_profile_report(self._ctx).decode().splitlines():
            name, n, ms, by, fl = line.split()
            out[name] = dict(launches=int(n), ms=float(ms), bytes=float(by), flops=float(fl))
        return out

    def ceilings(self) -> Dict[str, float]:
        """gm_ceilings: streaming copy / read rates and the register-resident bf16 MFMA rate (constant operands, and
        operands that toggle like real data) measured on this GPU with the library's own kernels."""
        a, b, m, r, n = C.c_double(0), C.c_double(0), C.c_double(0), C.c_double(0), C.c_int64(0)
        self._check(self.lib.gm_ceilings(self._ctx, C.byref(a), C.byref(b), C.byref(m), C.byref(r), C.byref(n)))
        return {"copy_GBps": a.value, "read_GBps": b.value, "mfma_bf16_TFLOPs": m.value,
                "mfma_bf16_TFLOPs_toggling_operands": r.value, "copy_buffer_bytes": n.value}

    def scatter_add(self, table: torch.Tensor, rows: torch.Tensor, grad: torch.Tensor, scale: float):
        self._check(self.lib.gm_scatter_add(self._ctx, _ptr(table), _ptr(rows), _ptr(grad), int(rows.numel()),
                                            float(scale)))

    # ------------------------------------------------------------------ histories
    def _seq_call(self, entry, tensors, *args):
        """The call on the context's stream, in order with torch's current one where that is another: the context's stream waits for
        what is enqueued there, the current one for the call, and the allocator learns who uses the tensors."""
        if _current_stream(self.device) == self._stream:
            rc = entry(self._ctx, *args)
            if rc != GM_OK:
                self._check(rc)
            return
        current = torch.cuda.current_stream(self.device)
        if self._own_stream is None:
            self._own_stream = torch.cuda.ExternalStream(self._stream, device=self.device) if self._stream else torch.cuda.default_stream(self.device)
        self._own_stream.wait_stream(current)
        try:
            self._check(entry(self._ctx, *args))
        finally:
            current.wait_stream(self._own_stream)
            for t in tensors:
                if t is not None:
                    t.record_stream(self._own_stream)

    def _seq(self, offsets: torch.Tensor, n_rows: int, longest: int, lengths: Optional[torch.Tensor] = None) -> gm_seq:
        _checked(offsets, torch.int64, "offsets", self.device)
        n = offsets.numel() - 1
        if offsets.dim() != 1 or n < 0:
            raise ValueError("offsets must hold one entry per sequence and one more")
        if lengths is not None:
            _checked(lengths, torch.int64, "lengths", self.device)
            if tuple(lengths.shape) != (n,):
                raise ValueError("lengths must hold one entry per sequence")
        return gm_seq(n, n_rows, int(longest), offsets.data_ptr(), None if lengths is None else lengths.data_ptr())

    def _seq_dtype(self, t: torch.Tensor, name: str) -> int:
        if t.dtype not in _SEQ_DTYPES:
            raise ValueError(f"{name} must be float32 or bfloat16 (got {t.dtype})")
        return _SEQ_DTYPES[t.dtype]

    def wait(self):
        """gm_wait: drains the stream and raises what the seq_* calls since the last wait found wrong ("wait" = 0)."""
        self._check(self.lib.gm_wait(self._ctx))

    def seq_embed(self, table: torch.Tensor, tokens: torch.Tensor, scale: float = 1.0, dtype=torch.float32,
                  out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """gm_seq_embed: scale * table[tokens] as `dtype`, zeros where a token is -1.  tokens int32 of any shape."""
        _checked(tokens, torch.int32, "tokens", self.device)
        _checked(table, torch.float32, "table", self.device)
        if table.dim() != 2:
            raise ValueError("table must be [rows, dim]")
        n, D = tokens.numel(), table.shape[1]
        if out is None:
            out = torch.empty(*tokens.shape, D, dtype=dtype, device=self.device)
        po, ld = _rows(out if out.dim() == 2 else out.view(n, D), "out", dtype, self.device, (n, D))
        self._seq_call(self.lib.gm_seq_embed, (table, tokens, out), n, tokens.data_ptr(), table.shape[0], D, table.data_ptr(), scale,
                       self._seq_dtype(out, "out"), po, ld)
        return out

    def seq_embed_grad(self, grad: torch.Tensor, tokens: torch.Tensor, n_rows: int, scale: float = 1.0, out: Optional[Dict[str, object]] = None,
                       emb_rows_capacity: Optional[int] = None, table: Optional[torch.Tensor] = None):
        """gm_seq_embed_grad.  Returns the coalesced list as a dict (emb_rows, emb_grad, n_emb_rows, capacity; `out` of an earlier call
        is filled again), or with `table` adds the sums to its rows and returns it."""
        _checked(tokens, torch.int32, "tokens", self.device)
        n, D = tokens.numel(), grad.shape[-1]
        pg, ld = _rows(grad if grad.dim() == 2 else grad.view(n, D), "grad", grad.dtype, self.device, (n, D))
        if table is not None:
            pt = _state(table, "table", self.device, (n_rows, D))
            self._seq_call(self.lib.gm_seq_embed_grad, (grad, tokens, table), n, tokens.data_ptr(), n_rows, D, self._seq_dtype(grad, "grad"), pg, ld,
                           scale, None, None, None, 0, pt)
            return table
        if out is None:
            cap = min(n, n_rows) if emb_rows_capacity is None else emb_rows_capacity
            out = dict(emb_rows=torch.empty(cap, dtype=torch.int64, device=self.device), emb_grad=torch.empty(cap, D, device=self.device),
                       n_emb_rows=torch.empty(1, dtype=torch.int64, device=self.device), capacity=cap)
        cap, rows, sums = int(out["capacity"]), out["emb_rows"], out["emb_grad"]
        _checked(rows, torch.int64, "emb_rows", self.device)
        _checked(sums, torch.float32, "emb_grad", self.device)
        _checked(out["n_emb_rows"], torch.int64, "n_emb_rows", self.device)
        if rows.numel() < cap or sums.numel() < cap * D or (sums.dim() > 1 and sums.shape[-1] != D):
            raise ValueError(f"emb_rows / emb_grad hold fewer rows of {D} than the capacity (emb_grad is {list(sums.shape)})")
        self._seq_call(self.lib.gm_seq_embed_grad, (grad, tokens, rows, sums, out["n_emb_rows"]), n, tokens.data_ptr(), n_rows, D,
                       self._seq_dtype(grad, "grad"), pg, ld, scale, rows.data_ptr(), sums.data_ptr(), out["n_emb_rows"].data_ptr(), cap, None)
        return out

    def seq_scan(self, x: torch.Tensor, gate: torch.Tensor, offsets: torch.Tensor, longest: int, h0: Optional[torch.Tensor] = None,
                 out: Optional[torch.Tensor] = None):
        """gm_seq_scan: (h, last) of the recurrence over every sequence; h like x, last [sequences, channels] fp32."""
        N, Ch = x.shape
        s = self._seq(offsets, N, longest)
        px, pg = _rows(x, "x", x.dtype, self.device, (N, Ch)), _rows(gate, "gate", x.dtype, self.device, (N, Ch))
        h = torch.empty(N, Ch, dtype=x.dtype, device=self.device) if out is None else out
        ph = _rows(h, "out", x.dtype, self.device, (N, Ch))
        last = torch.empty(s.n_seqs, Ch, device=self.device)
        self._seq_call(self.lib.gm_seq_scan, (x, gate, offsets, h0, h, last), C.byref(s), Ch, self._seq_dtype(x, "x"), *px, *pg,
                       _state(h0, "h0", self.device, (s.n_seqs, Ch)), *ph, last.data_ptr())
        return h, last

    def seq_scan_grad(self, dh: torch.Tensor, x: torch.Tensor, gate: torch.Tensor, h: torch.Tensor, offsets: torch.Tensor, longest: int,
                      h0: Optional[torch.Tensor] = None, dlast: Optional[torch.Tensor] = None, out=None):
        """gm_seq_scan_grad: (dx, dgate, dh0); dh0 is None without h0.  out: (dx, dgate) to be filled, whose rows may lie apart."""
        N, Ch = x.shape
        s = self._seq(offsets, N, longest)
        ins = [_rows(t, n, x.dtype, self.device, (N, Ch)) for t, n in ((x, "x"), (gate, "gate"), (h, "h"), (dh, "dh"))]
        dx, dg = out if out is not None else (torch.empty(N, Ch, dtype=x.dtype, device=self.device) for _ in range(2))
        pdx, pdg = (_rows(t, n, x.dtype, self.device, (N, Ch)) for t, n in ((dx, "dx"), (dg, "dgate")))
        dh0 = None if h0 is None else torch.empty(s.n_seqs, Ch, device=self.device)
        self._seq_call(self.lib.gm_seq_scan_grad, (dh, x, gate, h, offsets, h0, dlast, dx, dg, dh0), C.byref(s), Ch, self._seq_dtype(x, "x"),
                       *ins[0], *ins[1], *ins[2], _state(h0, "h0", self.device, (s.n_seqs, Ch)), *ins[3],
                       _state(dlast, "dlast", self.device, (s.n_seqs, Ch)), *pdx, *pdg,
                       None if dh0 is None else dh0.data_ptr())
        return dx, dg, dh0

    def seq_scan_step(self, x: torch.Tensor, gate: torch.Tensor, state: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """gm_seq_scan_step: one more row of every sequence; `state` (fp32) is updated in place, returned rounded to x's type."""
        S, Ch = x.shape
        px, pg = _rows(x, "x", x.dtype, self.device, (S, Ch)), _rows(gate, "gate", x.dtype, self.device, (S, Ch))
        h = torch.empty(S, Ch, dtype=x.dtype, device=self.device) if out is None else out
        ph = _rows(h, "out", x.dtype, self.device, (S, Ch))
        self._seq_call(self.lib.gm_seq_scan_step, (x, gate, state, h), S, Ch, self._seq_dtype(x, "x"), *px, *pg,
                       _state(state, "state", self.device, (S, Ch)), *ph)
        return h

    def _attend_args(self, q, k, v, q_offsets, k_offsets, longest_q, longest_k, scale, k_lengths, key_mask):
        if q.dim() != 3 or k.dim() != 3:
            raise ValueError("q, k and v must be [rows, heads, head_dim]")
        shape, (nk, G, _), dtype, device = q.shape, k.shape, q.dtype, self.device
        nq, H, D = shape
        hd = gm_seq_heads(H, G, D, self._seq_dtype(q, "q"), float(D ** -0.5 if scale is None else scale))
        qs, ks = self._seq(q_offsets, nq, longest_q), self._seq(k_offsets, nk, longest_k, k_lengths)
        if key_mask is not None:
            if key_mask.dtype not in (torch.uint8, torch.bool) or tuple(key_mask.shape) != (nk,) or not key_mask.is_contiguous() or key_mask.device != self.device:
                raise ValueError("key_mask must be a contiguous uint8 or bool tensor with one entry per key row")
        ptrs = _rows(q, "q", dtype, device, shape), _rows(k, "k", dtype, device, (nk, G, D)), _rows(v, "v", dtype, device, (nk, G, D))
        return hd, qs, ks, ptrs, None if key_mask is None else key_mask.data_ptr()

    def seq_attend(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_offsets: torch.Tensor, k_offsets: torch.Tensor, longest_q: int,
                   longest_k: int, scale: Optional[float] = None, k_lengths: Optional[torch.Tensor] = None, key_mask: Optional[torch.Tensor] = None,
                   out: Optional[torch.Tensor] = None):
        """gm_seq_attend: (o, lse); q [queries, heads, head_dim], k and v [keys, kv_heads, head_dim], scale 1 / sqrt(head_dim) unless given."""
        hd, qs, ks, ptrs, pm = self._attend_args(q, k, v, q_offsets, k_offsets, longest_q, longest_k, scale, k_lengths, key_mask)
        o = torch.empty_like(q, memory_format=torch.contiguous_format) if out is None else out
        po = _rows(o, "out", q.dtype, self.device, q.shape)
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=self.device)
        self._seq_call(self.lib.gm_seq_attend, (q, k, v, q_offsets, k_offsets, k_lengths, key_mask, o, lse), C.byref(qs), C.byref(ks), C.byref(hd),
                       *ptrs[0], *ptrs[1], *ptrs[2], pm, *po, lse.data_ptr())
        return o, lse

    def seq_attend_grad(self, dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor, lse: torch.Tensor,
                        q_offsets: torch.Tensor, k_offsets: torch.Tensor, longest_q: int, longest_k: int, scale: Optional[float] = None,
                        key_mask: Optional[torch.Tensor] = None, out=None):
        """gm_seq_attend_grad: (dq, dk, dv) from what seq_attend was given and returned, and the gradient of o; `out` to have these filled."""
        hd, qs, ks, ptrs, pm = self._attend_args(q, k, v, q_offsets, k_offsets, longest_q, longest_k, scale, None, key_mask)
        pd, po = _rows(dout, "dout", q.dtype, self.device, q.shape), _rows(o, "o", q.dtype, self.device, q.shape)
        pl = _state(lse, "lse", self.device, q.shape[:2])
        dq, dk, dv = out if out is not None else (torch.empty_like(t, memory_format=torch.contiguous_format) for t in (q, k, k))
        outs = [_rows(t, n, q.dtype, self.device, like.shape) for t, n, like in ((dq, "dq", q), (dk, "dk", k), (dv, "dv", k))]
        self._seq_call(self.lib.gm_seq_attend_grad, (dout, q, k, v, o, lse, q_offsets, k_offsets, key_mask, dq, dk, dv), C.byref(qs), C.byref(ks), C.byref(hd),
                       *pd, *ptrs[0], *ptrs[1], *ptrs[2], *po, pl, pm, *outs[0], *outs[1], *outs[2])
        return dq, dk, dv
