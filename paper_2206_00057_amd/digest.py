"""Thin Python binding of ``libdigest.so`` (the C ABI declared in include/digest.h).

Functions carry the C names.  They only marshal arguments: tensors become
device pointers (after dtype/device/size checks that keep every kernel
inside the buffers it is given), the stream defaults to torch's current
stream, and a negative status raises ``DigestError``.  All computation runs
in the HIP library; if it is not built, importing this module fails loudly.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
# DIGEST_LIBRARY names another build of the same ABI (e.g. the host-only
# sanitizer build); by default the in-tree libdigest.so.
LIB_PATH = os.environ.get("DIGEST_LIBRARY") or os.path.join(_PKG, "libdigest.so")

OK, EINVAL, ENOMEM, EHIP, ESTATE = 0, -1, -2, -3, -4
MODEL_GCN, MODEL_GAT = 0, 1
ACT_RELU, ACT_IDENTITY = 0, 1
PUSH_BOUNDARY, PUSH_ALL_OWNED = 0, 1
PULL_ROWS, PULL_AGGREGATE = 0, 1
KEEP_F32, KEEP_Q8 = 0, 1
F32, BF16, F16 = 0, 1, 2

_lib = None


class DigestError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"digest status {status}: {message}")
        self.status = status


def lib():
    """Load libdigest.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run `python -m paper_2206_00057_amd.build` "
                               "(or __graft_entry__.build())")
        L = ctypes.CDLL(LIB_PATH)
        P, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        st = ctypes.c_int
        sig = {
            "digest_last_error": ([], ctypes.c_char_p),
            "digest_partition_create": ([i64, P, P, P, P, i64, P, i64, i32, P, P], st),
            "digest_partition_destroy": ([P], None),
            "digest_partition_query": ([P, P, P, P, P], st),
            "digest_partition_bind_workspace": ([P, P, sz, P], st),
            "digest_partition_export_maps": ([P, P, P, P], st),
            "digest_partition_export_transpose": ([P, P, P, P], st),
            "digest_partition_read_halo": ([P, i32, P, P], st),
            "digest_pull": ([P, i32, P, P], st),
            "digest_partition_set_pull_mode": ([P, i32], st),
            "digest_push": ([P, i32, P, P, i32, P], st),
            "digest_layer_forward": ([P, i32, P, P, P, i32, P], st),
            "digest_layer_backward": ([P, i32, P, P, P, P, P, P, P], st),
            "digest_softmax_xent": ([P, P, P, P, P, P], st),
            "digest_softmax_xent_static": ([i64, i32, P, P, P, P, P], st),
            "digest_sgd_average": ([P, P, i32, i64, ctypes.c_float, P], st),
            "digest_halo_gradient": ([P, i32, P, P, P, P, P], st),
            "digest_layer_backward_halo": ([P, i32, P, P, P, P, P, P, P, P], st),
            "digest_gat_query": ([P, P], st),
            "digest_gat_bind_workspace": ([P, P, sz, P], st),
            "digest_gat_forward": ([P, i32, P, P, P, ctypes.c_float, P, i32, P], st),
            "digest_gat_backward": ([P, i32, P, P, P, P, P, P, P, P, P], st),
            "digest_push_add": ([P, i32, P, P, P], st),
            "digest_pull_add": ([P, i32, P, P, P], st),
            "digest_sync_period": ([i32, i64, P, P], st),
            "digest_profile_enable": ([P, i32], st),
            "digest_profile_read": ([P, P, P], st),
            "digest_profile_kernel_count": ([], i32),
            "digest_profile_kernel_name": ([i32], ctypes.c_char_p),
            "digest_partition_plan": ([P, i32, P], st),
            "digest_profile_model": ([P, i32, P, P, P], st),
        }
        for name, (args, res) in sig.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = res
        _lib = L
    return _lib


_train = None


def _train_lib():
    """The library with the operators that belong to no partition (layer norm,
    orthogonalised updates); raises if this build of the ABI lacks them."""
    global _train
    if _train is None or _train is not lib():
        L = lib()
        P, i32, i64, sz, f32 = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t,
                                ctypes.c_float)
        sig = {
            "digest_layer_norm_query": [i64, i32, P],
            "digest_layer_norm_forward": [i64, i32, i32, P, i64, P, P, f32, i32, P, i64, P, P],
            "digest_layer_norm_backward": [i64, i32, i32, P, i64, P, i32, P, i64, P, i64, P, P,
                                           i64, P, P, P, sz, P],
            "digest_orthogonalize_query": [i32, P, P, P],
            "digest_orthogonalize": [i32, P, P, i32, P, P, P, P, i32, P, P, sz, P],
            "digest_muon_average": [i32, P, P, P, P, P, i32, f32, f32, f32, P, i32, i32, P, P, sz,
                                    P],
        }
        for name, args in sig.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = ctypes.c_int
        _train = L
    return _train


def _check(status):
    if status != OK:
        raise DigestError(status, lib().digest_last_error().decode())


def _np(a, dtype):
    a = np.ascontiguousarray(a, dtype=dtype)
    return a, a.ctypes.data_as(ctypes.c_void_p)


def _stream(stream):
    if stream is None:
        import torch
        # (the handle alone: building a torch.cuda.Stream takes longer than a launch)
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    if isinstance(stream, int):
        return ctypes.c_void_p(stream)
    return ctypes.c_void_p(stream.cuda_stream)


def _dev(t, dtype, numel, name):
    """Device pointer of a contiguous CUDA tensor with exactly ``numel`` elements."""
    import torch
    if t is None:
        raise ValueError(f"{name} is required")
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.numel() != numel:
        raise ValueError(f"{name} has {t.numel()} elements, expected {numel}")
    return ctypes.c_void_p(t.data_ptr())


class Partition:
    """Handle of one partition (wraps ``digest_partition*``)."""

    def __init__(self, handle, n_global, n_own, n_halo, widths):
        self.handle = ctypes.c_void_p(handle)
        self.n_global = n_global
        self.n_own = n_own
        self.n_halo = n_halo
        self.widths = list(widths)
        self.L = len(self.widths) - 1
        self.workspace = None
        q = digest_partition_query(self)
        self.n_boundary = q["n_boundary"]
        self.nnz = q["nnz"]
        self.nnz_in = q["nnz_in"]
        self.workspace_bytes = q["workspace_bytes"]

    def __del__(self):
        try:
            digest_partition_destroy(self)
        except Exception:
            pass


def digest_partition_create(n_global, indptr, indices, values, owned, halo, widths):
    indptr, p_indptr = _np(indptr, np.int64)
    indices, p_indices = _np(indices, np.int64)
    values, p_values = _np(values, np.float32)
    owned, p_owned = _np(owned, np.int64)
    halo, p_halo = _np(halo, np.int64)
    widths, p_widths = _np(widths, np.int32)
    if indptr.shape[0] != owned.shape[0] + 1:
        raise ValueError("indptr must have n_owned + 1 entries")
    nnz = int(indptr[-1]) if indptr.size else 0
    if indices.shape[0] < nnz or values.shape[0] < nnz:
        raise ValueError("indices/values shorter than indptr[-1]")
    out = ctypes.c_void_p()
    _check(lib().digest_partition_create(int(n_global), p_indptr, p_indices, p_values, p_owned,
                                         owned.shape[0], p_halo, halo.shape[0],
                                         widths.shape[0] - 1, p_widths, ctypes.byref(out)))
    return Partition(out.value, int(n_global), owned.shape[0], halo.shape[0], widths.tolist())


def digest_partition_destroy(p):
    if p.handle:
        lib().digest_partition_destroy(p.handle)
        p.handle = ctypes.c_void_p()


def digest_partition_query(p):
    nb, nnz, nnz_in = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64()
    ws = ctypes.c_size_t()
    _check(lib().digest_partition_query(p.handle, ctypes.byref(nb), ctypes.byref(nnz),
                                        ctypes.byref(nnz_in), ctypes.byref(ws)))
    return {"n_boundary": nb.value, "nnz": nnz.value, "nnz_in": nnz_in.value,
            "workspace_bytes": ws.value}


def digest_partition_bind_workspace(p, workspace, stream=None):
    """Bind a CUDA uint8 tensor of at least ``p.workspace_bytes`` bytes."""
    import torch
    if not isinstance(workspace, torch.Tensor) or not workspace.is_cuda:
        raise TypeError("workspace must be a CUDA tensor")
    nbytes = workspace.numel() * workspace.element_size()
    _check(lib().digest_partition_bind_workspace(p.handle, ctypes.c_void_p(workspace.data_ptr()),
                                                 nbytes, _stream(stream)))
    p.workspace = workspace


def digest_partition_export_maps(p):
    col = np.empty(p.nnz, np.int32)
    bgid = np.empty(p.n_boundary, np.int64)
    bloc = np.empty(p.n_boundary, np.int32)
    _check(lib().digest_partition_export_maps(p.handle, col.ctypes.data_as(ctypes.c_void_p),
                                              bgid.ctypes.data_as(ctypes.c_void_p),
                                              bloc.ctypes.data_as(ctypes.c_void_p)))
    return col, bgid, bloc


def digest_partition_export_transpose(p):
    ptr = np.empty(p.n_own + 1, np.int64)
    src = np.empty(p.nnz_in, np.int32)
    val = np.empty(p.nnz_in, np.float32)
    _check(lib().digest_partition_export_transpose(p.handle, ptr.ctypes.data_as(ctypes.c_void_p),
                                                   src.ctypes.data_as(ctypes.c_void_p),
                                                   val.ctypes.data_as(ctypes.c_void_p)))
    return ptr, src, val


def digest_partition_read_halo(p, level, out, stream=None):
    import torch
    _check_level(p, level, 0)
    ptr = _dev(out, torch.float32, p.n_halo * p.widths[level], "out")
    _check(lib().digest_partition_read_halo(p.handle, int(level), ptr, _stream(stream)))


def _check_level(p, level, lo):
    if not (lo <= level < p.L):
        raise DigestError(EINVAL, f"level {level} outside [{lo}, {p.L})")


def _check_layer(p, layer):
    if not (1 <= layer <= p.L):
        raise DigestError(EINVAL, f"layer {layer} outside [1, {p.L}]")


def digest_partition_set_pull_mode(p, mode):
    _check(lib().digest_partition_set_pull_mode(p.handle, int(mode)))


def digest_pull(p, level, store, stream=None):
    import torch
    _check_level(p, level, 0)
    ptr = _dev(store, torch.float32, p.n_global * p.widths[level], "store")
    _check(lib().digest_pull(p.handle, int(level), ptr, _stream(stream)))


def digest_push(p, level, h_own, store, mode=PUSH_BOUNDARY, stream=None):
    import torch
    _check_level(p, level, 1)
    d = p.widths[level]
    ph = _dev(h_own, torch.float32, p.n_own * d, "h_own")
    ps = _dev(store, torch.float32, p.n_global * d, "store")
    _check(lib().digest_push(p.handle, int(level), ph, ps, int(mode), _stream(stream)))


def digest_layer_forward(p, layer, h_in, w, h_out, act, stream=None):
    import torch
    _check_layer(p, layer)
    di, do = p.widths[layer - 1], p.widths[layer]
    a = _dev(h_in, torch.float32, p.n_own * di, "h_in")
    b = _dev(w, torch.float32, di * do, "w")
    c = _dev(h_out, torch.float32, p.n_own * do, "h_out")
    _check(lib().digest_layer_forward(p.handle, int(layer), a, b, c, int(act), _stream(stream)))


def digest_layer_backward(p, layer, h_in, h_out, dh_out, w, dw, dh_in=None, stream=None):
    import torch
    _check_layer(p, layer)
    di, do = p.widths[layer - 1], p.widths[layer]
    x = _dev(h_in, torch.float32, p.n_own * di, "h_in")
    a = _dev(h_out, torch.float32, p.n_own * do, "h_out")
    b = _dev(dh_out, torch.float32, p.n_own * do, "dh_out")
    c = _dev(w, torch.float32, di * do, "w")
    e = _dev(dw, torch.float32, di * do, "dw")
    f = _dev(dh_in, torch.float32, p.n_own * di, "dh_in") if dh_in is not None else None
    _check(lib().digest_layer_backward(p.handle, int(layer), x, a, b, c, e, f, _stream(stream)))


def digest_layer_backward_halo(p, layer, h_in, h_out, dh_out, w, dw, dh_in, dh_halo,
                               stream=None):
    """digest_layer_backward plus dh_halo = P_out^T D W^T (layer 2..L)."""
    import torch
    _check_layer(p, layer)
    di, do = p.widths[layer - 1], p.widths[layer]
    _check(lib().digest_layer_backward_halo(
        p.handle, int(layer), _dev(h_in, torch.float32, p.n_own * di, "h_in"),
        _dev(h_out, torch.float32, p.n_own * do, "h_out"),
        _dev(dh_out, torch.float32, p.n_own * do, "dh_out"),
        _dev(w, torch.float32, di * do, "w"), _dev(dw, torch.float32, di * do, "dw"),
        _dev(dh_in, torch.float32, p.n_own * di, "dh_in"),
        _dev(dh_halo, torch.float32, p.n_halo * di, "dh_halo"), _stream(stream)))


GAT_SLOPE = 0.2   # the GAT model's LeakyReLU slope


def digest_gat_query(p):
    """Bytes of the partition's GAT workspace."""
    n = ctypes.c_size_t(0)
    _check(lib().digest_gat_query(p.handle, ctypes.byref(n)))
    return int(n.value)


def digest_gat_bind_workspace(p, workspace, stream=None):
    """Bind a CUDA tensor of at least digest_gat_query(p) bytes."""
    import torch
    if not isinstance(workspace, torch.Tensor) or not workspace.is_cuda:
        raise TypeError("GAT workspace must be a CUDA tensor")
    nbytes = workspace.numel() * workspace.element_size()
    _check(lib().digest_gat_bind_workspace(p.handle, ctypes.c_void_p(workspace.data_ptr()),
                                           nbytes, _stream(stream)))
    p.gat_workspace = workspace   # kept alive with the handle


def digest_gat_forward(p, layer, h_in, w, att, h_out, act, slope=GAT_SLOPE, stream=None):
    import torch
    _check_layer(p, layer)
    di, do = p.widths[layer - 1], p.widths[layer]
    _check(lib().digest_gat_forward(
        p.handle, int(layer), _dev(h_in, torch.float32, p.n_own * di, "h_in"),
        _dev(w, torch.float32, di * do, "w"), _dev(att, torch.float32, do * 2, "att"),
        ctypes.c_float(slope), _dev(h_out, torch.float32, p.n_own * do, "h_out"), int(act),
        _stream(stream)))


def digest_gat_backward(p, layer, h_in, h_out, dh_out, w, att, dw, datt, dh_in=None,
                        stream=None):
    import torch
    _check_layer(p, layer)
    di, do = p.widths[layer - 1], p.widths[layer]
    _check(lib().digest_gat_backward(
        p.handle, int(layer), _dev(h_in, torch.float32, p.n_own * di, "h_in"),
        _dev(h_out, torch.float32, p.n_own * do, "h_out"),
        _dev(dh_out, torch.float32, p.n_own * do, "dh_out"),
        _dev(w, torch.float32, di * do, "w"), _dev(att, torch.float32, do * 2, "att"),
        _dev(dw, torch.float32, di * do, "dw"), _dev(datt, torch.float32, do * 2, "datt"),
        _dev(dh_in, torch.float32, p.n_own * di, "dh_in") if dh_in is not None else None,
        _stream(stream)))


def digest_softmax_xent(p, logits, labels, dlogits, loss, stream=None):
    import torch
    C = p.widths[-1]
    a = _dev(logits, torch.float32, p.n_own * C, "logits")
    b = _dev(labels, torch.int32, p.n_own, "labels")
    c = _dev(dlogits, torch.float32, p.n_own * C, "dlogits")
    d = _dev(loss, torch.float32, 1, "loss")
    _check(lib().digest_softmax_xent(p.handle, a, b, c, d, _stream(stream)))


def digest_softmax_xent_static(logits, labels, dlogits, loss, stream=None):
    """The loss head without a partition or workspace (for callers that
    cannot allocate): logits [n, C], labels int32 [n], dlogits [n, C], loss
    [1]; partial sums in the library's fixed device array."""
    import torch
    if logits.dim() != 2:
        raise ValueError("logits must be [n, C]")
    n, C = int(logits.shape[0]), int(logits.shape[1])
    _check(lib().digest_softmax_xent_static(
        n, C, _dev(logits, torch.float32, n * C, "logits"),
        _dev(labels, torch.int32, n, "labels"), _dev(dlogits, torch.float32, n * C, "dlogits"),
        _dev(loss, torch.float32, 1, "loss"), _stream(stream)))


def digest_halo_gradient(p, layer, h_out, dh_out, w, dh_halo, stream=None):
    """dh_halo = P_out^T D W^T for the halo rows of level layer-1."""
    import torch
    _check_layer(p, layer)
    d_in, d_out = p.widths[layer - 1], p.widths[layer]
    _check(lib().digest_halo_gradient(
        p.handle, int(layer), _dev(h_out, torch.float32, p.n_own * d_out, "h_out"),
        _dev(dh_out, torch.float32, p.n_own * d_out, "dh_out"),
        _dev(w, torch.float32, d_in * d_out, "w"),
        _dev(dh_halo, torch.float32, p.n_halo * d_in, "dh_halo"), _stream(stream)))


def digest_push_add(p, level, dh_halo, gstore, stream=None):
    """gstore[halo] += dh_halo (level 1..L-1)."""
    import torch
    _check_level(p, level, 1)
    d = p.widths[level]
    _check(lib().digest_push_add(p.handle, int(level),
                                 _dev(dh_halo, torch.float32, p.n_halo * d, "dh_halo"),
                                 _dev(gstore, torch.float32, p.n_global * d, "gstore"),
                                 _stream(stream)))


def digest_pull_add(p, level, gstore, dh_own, stream=None):
    """dh_own += gstore[owned]; gstore[owned] = 0 (level 1..L-1)."""
    import torch
    _check_level(p, level, 1)
    d = p.widths[level]
    _check(lib().digest_pull_add(p.handle, int(level),
                                 _dev(gstore, torch.float32, p.n_global * d, "gstore"),
                                 _dev(dh_own, torch.float32, p.n_own * d, "dh_own"),
                                 _stream(stream)))


def digest_sgd_average(w, grads, lr, stream=None):
    """w -= lr * mean(grads), the average of the local models (Algorithm 1, AGG)."""
    import torch
    if not grads:
        raise ValueError("need at least one gradient")
    n = w.numel()
    pw = _dev(w, torch.float32, n, "w")
    ptrs = (ctypes.c_void_p * len(grads))(*[_dev(g, torch.float32, n, f"grads[{m}]").value
                                            for m, g in enumerate(grads)])
    _check(lib().digest_sgd_average(pw, ptrs, len(grads), n, float(lr), _stream(stream)))


def digest_sync_period(K, iteration):
    a, b = ctypes.c_int32(), ctypes.c_int32()
    _check(lib().digest_sync_period(int(K), int(iteration), ctypes.byref(a), ctypes.byref(b)))
    return bool(a.value), bool(b.value)


def digest_profile_enable(p, on=True):
    _check(lib().digest_profile_enable(p.handle, 1 if on else 0))


def kernel_names():
    L = lib()
    return [L.digest_profile_kernel_name(i).decode() for i in range(L.digest_profile_kernel_count())]


def digest_profile_read(p):
    """Per (kernel kind, layer slot): {"kind.lN": (total ms, launches)} since the
    last read (synchronises).  Slot = layer for layer kernels, level for
    pull/push, L for the loss head; entries without launches are omitted."""
    n = lib().digest_profile_kernel_count()
    slots = p.L + 1
    ms = np.zeros(n * slots, np.float64)
    cnt = np.zeros(n * slots, np.int64)
    _check(lib().digest_profile_read(p.handle, ms.ctypes.data_as(ctypes.c_void_p),
                                     cnt.ctypes.data_as(ctypes.c_void_p)))
    out = {}
    for i, name in enumerate(kernel_names()):
        for sl in range(slots):
            j = i * slots + sl
            if cnt[j]:
                out[f"{name}.l{sl}"] = (float(ms[j]), int(cnt[j]))
    return out


class LayerPlan(ctypes.Structure):
    """``digest_layer_plan`` of include/digest.h."""
    _fields_ = [("transform_first", ctypes.c_int32), ("forward_narrow", ctypes.c_int32),
                ("dw_slices", ctypes.c_int32), ("dgrad_narrow_first", ctypes.c_int32),
                ("dgrad_fused", ctypes.c_int32), ("tiers_fwd", ctypes.c_int32),
                ("tiers_bwd", ctypes.c_int32), ("tier_rows_fwd", ctypes.c_int32),
                ("tier_rows_bwd", ctypes.c_int32), ("tier_entries_fwd", ctypes.c_int64),
                ("tier_entries_bwd", ctypes.c_int64), ("forward_fused", ctypes.c_int32),
                ("backward_fused", ctypes.c_int32)]


def digest_partition_plan(p, layer):
    """The library's launch plan of ``layer`` as a dict of the C fields."""
    _check_layer(p, layer)
    out = LayerPlan()
    _check(lib().digest_partition_plan(p.handle, int(layer), ctypes.byref(out)))
    return {name: int(getattr(out, name)) for name, _ in LayerPlan._fields_}


def digest_profile_model(p, model=MODEL_GCN):
    """Algorithmic (bytes, flops, sparse entries) of one launch of each
    (kernel kind, slot) a round makes, keyed like ``digest_profile_read``;
    kinds the round does not launch are omitted."""
    n = lib().digest_profile_kernel_count()
    slots = p.L + 1
    b = np.zeros(n * slots, np.float64)
    f = np.zeros(n * slots, np.float64)
    e = np.zeros(n * slots, np.int64)
    _check(lib().digest_profile_model(p.handle, int(model), b.ctypes.data_as(ctypes.c_void_p),
                                      f.ctypes.data_as(ctypes.c_void_p),
                                      e.ctypes.data_as(ctypes.c_void_p)))
    out = {}
    for i, name in enumerate(kernel_names()):
        for sl in range(slots):
            j = i * slots + sl
            if b[j] or f[j] or e[j]:
                out[f"{name}.l{sl}"] = (float(b[j]), float(f[j]), int(e[j]))
    return out


# Operators that belong to no partition: layer norm, orthogonalised updates.

_TYPES = {}


def _elem_types():
    """torch dtype -> DIGEST_F32, ..."""
    if not _TYPES:
        import torch
        _TYPES.update({torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16})
    return _TYPES


def _device():
    """The current device, where the kernels run."""
    import torch
    return torch.cuda.current_device()


def _here(t, dev, name):
    if getattr(t, "is_cuda", False) is not True:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, the current device is cuda:{dev}")


def _rows(t, shape, dtype, dev, name):
    """(pointer, row stride) of a 2-D tensor of this shape and type whose rows
    are contiguous."""
    _here(t, dev, name)
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    n, d = shape
    if t.is_contiguous():
        return t.data_ptr(), d
    ld, step = t.stride()
    if d > 1 and step != 1:
        raise ValueError(f"{name}: the elements of a row must be contiguous")
    if n <= 1:
        ld = d
    if ld < d:
        raise ValueError(f"{name}: rows must not overlap")
    return t.data_ptr(), ld


def _matrix(t, dev, name):
    """The (shape, dtype) of a 2-D tensor of one of the element types."""
    _here(t, dev, name)
    if t.dim() != 2:
        raise ValueError(f"{name} must be 2-D")
    if t.dtype not in _elem_types():
        raise TypeError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    return t.shape, t.dtype


def _floats(t, numel, dev, name):
    """Pointer of a contiguous float32 tensor of numel elements, None for None."""
    if t is None:
        return None
    _here(t, dev, name)
    if _elem_types().get(t.dtype) != F32:
        raise TypeError(f"{name} must be torch.float32, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.numel() != numel:
        raise ValueError(f"{name} has {t.numel()} elements, expected {numel}")
    return t.data_ptr()


def _workspace(t, dev):
    if t is None:
        return None, 0
    _here(t, dev, "workspace")
    if not t.is_contiguous():
        raise ValueError("workspace must be contiguous")
    return t.data_ptr(), t.numel() * t.element_size()


def digest_layer_norm_query(n_rows, width):
    """Bytes of the layer norm backward's workspace."""
    out = ctypes.c_size_t(0)
    _check(_train_lib().digest_layer_norm_query(int(n_rows), int(width), ctypes.byref(out)))
    return int(out.value)


def digest_layer_norm_forward(x, gain, shift, y, stats=None, eps=1e-5, act=ACT_IDENTITY,
                              stream=None):
    """y = act(layer norm of each row of x [n, d]); gain, shift float32 [d] or
    None; stats float32 [n, 2] keeps (mean, rstd) for the backward."""
    dev = _device()
    shape, dtype = _matrix(x, dev, "x")
    n, d = shape
    px, ldx = _rows(x, shape, dtype, dev, "x")
    py, ldy = _rows(y, shape, dtype, dev, "y")
    _check(_train_lib().digest_layer_norm_forward(
        n, d, _TYPES[dtype], px, ldx, _floats(gain, d, dev, "gain"),
        _floats(shift, d, dev, "shift"), eps, act, py, ldy, _floats(stats, 2 * n, dev, "stats"),
        _stream(stream)))


def digest_layer_norm_backward(x, gain, y, dy, stats, dx, dgain, dshift, workspace,
                               act=ACT_IDENTITY, stream=None):
    """dx, dgain, dshift of digest_layer_norm_forward (each may be None); y, its
    output, is read with ACT_RELU only; workspace: a CUDA tensor of at least
    digest_layer_norm_query(n, d) bytes (None without dgain and dshift)."""
    dev = _device()
    shape, dtype = _matrix(x, dev, "x")
    n, d = shape
    px, ldx = _rows(x, shape, dtype, dev, "x")
    py, ldy = _rows(y, shape, dtype, dev, "y") if act == ACT_RELU else (None, 0)
    pdy, lddy = _rows(dy, shape, dtype, dev, "dy")
    pdx, lddx = _rows(dx, shape, dtype, dev, "dx") if dx is not None else (None, 0)
    ws, nbytes = _workspace(workspace, dev)
    if stats is None:
        raise ValueError("stats is required")
    _check(_train_lib().digest_layer_norm_backward(
        n, d, _TYPES[dtype], px, ldx, _floats(gain, d, dev, "gain"), act, py, ldy, pdy, lddy,
        _floats(stats, 2 * n, dev, "stats"), pdx, lddx, _floats(dgain, d, dev, "dgain"),
        _floats(dshift, d, dev, "dshift"), ws, nbytes, _stream(stream)))


MUON_COEFFS = (3.4445, -4.7750, 2.0315)   # the default odd polynomial of each step


def _sides(shapes):
    n = len(shapes)
    return ((ctypes.c_int32 * n)(*[int(s[0]) for s in shapes]),
            (ctypes.c_int32 * n)(*[int(s[1]) for s in shapes]))


def _coeffs(coeffs, steps):
    """None, (a, b, c) for every step, or one triple per step."""
    if coeffs is None:
        return None
    if not any(hasattr(c, "__len__") for c in coeffs):
        coeffs = [coeffs] * int(steps)
    if len(coeffs) != int(steps) or any(len(c) != 3 for c in coeffs):
        raise ValueError("coeffs must be (a, b, c) or one triple per step")
    flat = [float(v) for c in coeffs for v in c]
    return (ctypes.c_float * len(flat))(*flat)


def digest_orthogonalize_query(shapes):
    """Bytes of the workspace of digest_orthogonalize and digest_muon_average
    for matrices of these (rows, cols)."""
    if not len(shapes):
        raise ValueError("need at least one matrix")
    rows, cols = _sides(shapes)
    out = ctypes.c_size_t(0)
    _check(_train_lib().digest_orthogonalize_query(len(shapes), rows, cols, ctypes.byref(out)))
    return int(out.value)


def digest_orthogonalize(mats, outs, workspace, steps=5, coeffs=None, stream=None):
    """outs[i] = the orthogonalised matrix of mats[i] (2-D, one dtype); outs may
    be mats; workspace: a CUDA tensor of at least digest_orthogonalize_query
    bytes for the same shapes."""
    n = len(mats)
    if n < 1 or len(outs) != n:
        raise ValueError("need as many outputs as matrices, and one at least")
    dev = _device()
    dtype = _matrix(mats[0], dev, "mats[0]")[1]
    ins, outp = [], []
    for i, (m, o) in enumerate(zip(mats, outs)):
        shape, t = _matrix(m, dev, f"mats[{i}]")
        if 0 in shape:
            raise ValueError(f"mats[{i}] has no elements")
        if t != dtype:
            raise TypeError(f"mats[{i}] must be {dtype}, got {t}")
        ins.append(_rows(m, shape, dtype, dev, f"mats[{i}]"))
        outp.append(_rows(o, shape, dtype, dev, f"outs[{i}]"))
    rows, cols = _sides([m.shape for m in mats])
    ptrs, lds = ctypes.c_void_p * n, ctypes.c_int64 * n
    ws, nbytes = _workspace(workspace, dev)
    _check(_train_lib().digest_orthogonalize(
        n, rows, cols, _TYPES[dtype], ptrs(*[p for p, _ in ins]), lds(*[l for _, l in ins]),
        ptrs(*[p for p, _ in outp]), lds(*[l for _, l in outp]), int(steps),
        _coeffs(coeffs, steps), ws, nbytes, _stream(stream)))


def digest_muon_average(ws, momenta, grads, workspace, lr, beta=0.95, decay=0.0, scales=None,
                        nesterov=True, steps=5, coeffs=None, stream=None):
    """The Muon update of the weight matrices ws (with their momenta, float32,
    in place) by the mean of each one's gradients: grads[i] lists the M
    gradients of ws[i]."""
    n = len(ws)
    if n < 1 or len(momenta) != n or len(grads) != n:
        raise ValueError("need a momentum and a list of gradients for each matrix, and one at "
                         "least")
    M = len(grads[0])
    if M < 1 or any(len(g) != M for g in grads):
        raise ValueError("need the same number of gradients for each matrix, and one at least")
    if scales is not None and len(scales) != n:
        raise ValueError("need one scale for each matrix")
    dev = _device()
    flat = {"ws": [], "momenta": [], "grads": []}
    shapes = [w.shape for w in ws]
    for i, shape in enumerate(shapes):
        if len(shape) != 2 or 0 in shape:
            raise ValueError(f"ws[{i}] must be a matrix with rows and columns")
        for name, ts in (("ws", [ws[i]]), ("momenta", [momenta[i]]), ("grads", grads[i])):
            for t in ts:
                if t.shape != shape:
                    raise ValueError(f"{name}[{i}] must be {list(shape)}, got {list(t.shape)}")
                flat[name].append(_floats(t, t.numel(), dev, f"{name}[{i}]"))
    rows, cols = _sides(shapes)
    arr = lambda v: (ctypes.c_void_p * len(v))(*v)
    work, nbytes = _workspace(workspace, dev)
    _check(_train_lib().digest_muon_average(
        n, rows, cols, arr(flat["ws"]), arr(flat["momenta"]), arr(flat["grads"]), M, float(lr),
        float(beta), float(decay),
        (ctypes.c_float * n)(*[float(v) for v in scales]) if scales is not None else None,
        int(bool(nesterov)), int(steps), _coeffs(coeffs, steps), work, nbytes, _stream(stream)))


# Rows held in 8 bits.

_q8 = None
_I8 = _F32T = _I64 = None   # torch.int8, torch.float32, torch.int64
_raw_stream = None           # a device's current stream, as a number


def _q8_lib():
    """The library with the calls on rows held in 8 bits; raises if this build
    of the ABI lacks them."""
    global _q8, _I8, _F32T, _I64, _raw_stream
    if _q8 is None or _q8 is not _lib:
        import torch
        _I8, _F32T, _I64 = torch.int8, torch.float32, torch.int64
        _raw_stream = torch._C._cuda_getCurrentRawStream
        L = lib()
        P, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        sig = {
            "digest_quantize_rows": [i64, i32, i32, P, i64, P, i64, P, i64, P, P],
            "digest_quantize_columns": [i32, i32, i32, P, i64, P, i64, P, P],
            "digest_dequantize_rows": [i64, i32, P, i64, P, P, i64, i32, P, i64, P],
            "digest_q8_product": [i64, i32, i32, P, i64, P, P, i64, P, i32, i32, P, i64, P],
            "digest_q8_weight_grad_query": [i64, i32, i32, P],
            "digest_q8_weight_grad": [i64, i32, i32, P, i64, P, i32, P, i64, i32, P, i64, P, P, sz,
                                      P],
            "digest_push_q8": [P, i32, P, P, P, i32, P],
            "digest_pull_q8": [P, i32, P, P, P],
            "digest_partition_set_keep_mode": [P, i32],
            "digest_layer_forward_q8": [P, i32, P, P, P, P, i32, P],
        }
        for name, args in sig.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = ctypes.c_int
        _q8 = L
    return _q8


def digest_q8_stride(width):
    """Row stride of the codes of rows of `width` elements (DIGEST_Q8_STRIDE)."""
    return (int(width) + 15) // 16 * 16


# (The checks below take the common case first, a contiguous tensor of what is
# asked for: they cost as much as a launch.)

def _row_array(t, shape, dtype, dev, name):
    """As _rows."""
    if (getattr(t, "dtype", None) is dtype and t.shape == shape and t.get_device() == dev and
            t.is_contiguous()):
        return t.data_ptr(), shape[1]
    return _rows(t, shape, dtype, dev, name)


def _codes(t, scales, n, width, dev, name, scales_name):
    """(pointer, row stride, pointer of the scales) of the codes [n,
    digest_q8_stride(width)] and scales [n] of n rows."""
    p, ld = _row_array(t, (n, (width + 15) // 16 * 16), _I8, dev, name)
    if (getattr(scales, "dtype", None) is _F32T and scales.numel() == n and
            scales.get_device() == dev and scales.is_contiguous()):
        return p, ld, scales.data_ptr()
    return p, ld, _need(_floats(scales, n, dev, scales_name), scales_name)


def _stream_of(stream, dev):
    """As _stream, of the device dev, the current one."""
    return _raw_stream(dev) if stream is None else _stream(stream)


def _need(p, name):
    if p is None:
        raise ValueError(f"{name} is required")
    return p


def _list(rows, n, dev):
    """Pointer of n row numbers (int64), None for None."""
    if rows is None:
        return None
    _here(rows, dev, "rows")
    if rows.dtype is not _I64:
        raise TypeError(f"rows must be torch.int64, got {rows.dtype}")
    if rows.dim() != 1 or not rows.is_contiguous() or rows.numel() != n:
        raise ValueError(f"rows must be {n} contiguous numbers")
    return rows.data_ptr()


def digest_quantize_rows(x, codes, scales, rows=None, stream=None):
    """codes, scales = the rows of x [m, d] (those that rows, int64, lists, in
    its order) held in 8 bits: codes int8 [n, digest_q8_stride(d)], scales
    float32 [n]."""
    L, dev = _q8_lib(), _device()
    shape, dtype = _matrix(x, dev, "x")
    m, d = shape
    n = m if rows is None else rows.numel()
    px, ldx = _row_array(x, shape, dtype, dev, "x")
    pq, ldq, ps = _codes(codes, scales, n, d, dev, "codes", "scales")
    _check(L.digest_quantize_rows(n, d, _TYPES[dtype], px, ldx, _list(rows, n, dev), m, pq,
                                          ldq, ps, _stream_of(stream, dev)))


def digest_quantize_columns(w, codes, scales, stream=None):
    """codes, scales = the columns of w [k, m] held in 8 bits: codes int8 [m,
    digest_q8_stride(k)], scales float32 [m]."""
    L, dev = _q8_lib(), _device()
    shape, dtype = _matrix(w, dev, "w")
    k, m = shape
    pw, ldw = _row_array(w, shape, dtype, dev, "w")
    pq, ldq, ps = _codes(codes, scales, m, k, dev, "codes", "scales")
    _check(L.digest_quantize_columns(k, m, _TYPES[dtype], pw, ldw, pq, ldq, ps,
                                             _stream_of(stream, dev)))


def digest_dequantize_rows(codes, scales, y, rows=None, stream=None):
    """y [n, d] = the values of the rows (those that rows, int64, lists, in its
    order) that codes [m, digest_q8_stride(d)] and scales [m] hold."""
    L, dev = _q8_lib(), _device()
    shape, dtype = _matrix(y, dev, "y")
    n, d = shape
    m = n if rows is None else codes.shape[0]
    pq, ldq, ps = _codes(codes, scales, m, d, dev, "codes", "scales")
    py, ldy = _row_array(y, shape, dtype, dev, "y")
    _check(L.digest_dequantize_rows(n, d, pq, ldq, ps, _list(rows, n, dev), m,
                                            _TYPES[dtype], py, ldy, _stream_of(stream, dev)))


def digest_q8_product(codes, scales, w_codes, w_scales, y, act=ACT_IDENTITY, stream=None):
    """y [n, d_out] = act(the product of the rows in 8 bits (codes [n, k], scales
    [n]) by the weight matrix whose columns w_codes [d_out, k], w_scales [d_out]
    hold)."""
    L, dev = _q8_lib(), _device()
    shape, dtype = _matrix(y, dev, "y")
    n, m = shape
    k = codes.shape[-1]
    pq, ldq, ps = _codes(codes, scales, n, k, dev, "codes", "scales")
    pw, ldw, pt = _codes(w_codes, w_scales, m, k, dev, "w_codes", "w_scales")
    py, ldy = _row_array(y, shape, dtype, dev, "y")
    _check(L.digest_q8_product(n, k, m, pq, ldq, ps, pw, ldw, pt, act, _TYPES[dtype], py,
                                       ldy, _stream_of(stream, dev)))


def digest_q8_weight_grad_query(n_rows, d_in, d_out):
    """Bytes of the workspace of digest_q8_weight_grad."""
    out = ctypes.c_size_t(0)
    _check(_q8_lib().digest_q8_weight_grad_query(int(n_rows), int(d_in), int(d_out),
                                                 ctypes.byref(out)))
    return int(out.value)


def digest_q8_weight_grad(codes, scales, dy, dw, workspace, act=ACT_IDENTITY, y=None, stream=None):
    """dw [d_in, d_out], float32 = the transpose of the rows that codes [n,
    digest_q8_stride(d_in)] and scales [n] hold, times dy [n, d_out], with
    ACT_RELU masked by y > 0; workspace: a CUDA tensor of at least
    digest_q8_weight_grad_query(n, d_in, d_out) bytes."""
    L, dev = _q8_lib(), _device()
    shape, dtype = _matrix(dy, dev, "dy")
    n, m = shape
    if getattr(dw, "ndim", 0) != 2 or dw.shape[1] != m:
        raise ValueError(f"dw must be [d_in, {m}]")
    k = dw.shape[0]
    pq, ldq, ps = _codes(codes, scales, n, k, dev, "codes", "scales")
    pdy, lddy = _row_array(dy, shape, dtype, dev, "dy")
    if act == ACT_RELU and y is None:
        raise ValueError("y is required with ACT_RELU")
    py, ldy = _row_array(y, shape, dtype, dev, "y") if act == ACT_RELU else (None, 0)
    ws, nbytes = _workspace(workspace, dev)
    _check(L.digest_q8_weight_grad(n, k, m, pq, ldq, ps, _TYPES[dtype], pdy, lddy, act,
                                           py, ldy, _floats(dw, k * m, dev, "dw"), ws, nbytes,
                                           _stream_of(stream, dev)))


def digest_push_q8(p, level, h_own, codes, scales, mode=PUSH_BOUNDARY, stream=None):
    """digest_push into a store in 8 bits: codes int8 [n_global,
    digest_q8_stride(d)], scales float32 [n_global]."""
    import torch
    _check_level(p, level, 1)
    d = p.widths[level]
    ph = _dev(h_own, torch.float32, p.n_own * d, "h_own")
    pq = _dev(codes, torch.int8, p.n_global * digest_q8_stride(d), "codes")
    ps = _dev(scales, torch.float32, p.n_global, "scales")
    _check(_q8_lib().digest_push_q8(p.handle, int(level), ph, pq, ps, int(mode), _stream(stream)))


def digest_pull_q8(p, level, codes, scales, stream=None):
    """digest_pull out of a store in 8 bits."""
    import torch
    _check_level(p, level, 0)
    pq = _dev(codes, torch.int8, p.n_global * digest_q8_stride(p.widths[level]), "codes")
    ps = _dev(scales, torch.float32, p.n_global, "scales")
    _check(_q8_lib().digest_pull_q8(p.handle, int(level), pq, ps, _stream(stream)))


def digest_partition_set_keep_mode(p, mode):
    """KEEP_F32 or KEEP_Q8; a change unbinds the workspace and changes
    p.workspace_bytes."""
    _check(_q8_lib().digest_partition_set_keep_mode(p.handle, int(mode)))
    p.workspace_bytes = digest_partition_query(p)["workspace_bytes"]


def digest_layer_forward_q8(p, layer, h_in, w_codes, w_scales, h_out, act, stream=None):
    """The layer forward with the product in 8 bits (KEEP_Q8): w_codes int8 [d_out,
    digest_q8_stride(d_in)], w_scales float32 [d_out] hold W's columns."""
    import torch
    _check_layer(p, layer)
    di, do = p.widths[layer - 1], p.widths[layer]
    a = _dev(h_in, torch.float32, p.n_own * di, "h_in")
    b = _dev(w_codes, torch.int8, do * digest_q8_stride(di), "w_codes")
    c = _dev(w_scales, torch.float32, do, "w_scales")
    e = _dev(h_out, torch.float32, p.n_own * do, "h_out")
    _check(_q8_lib().digest_layer_forward_q8(p.handle, int(layer), a, b, c, e, int(act),
                                             _stream(stream)))
