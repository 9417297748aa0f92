"""ctypes binding of libgsplit.so: argument marshalling only.

Every function has the name and the argument order of its C entry point in include/gsplit.h;
tensors are passed as raw device pointers and the current torch stream as a hipStream_t.  There is
no computation here and no fallback: if the HIP library is missing or a call fails, an exception
is raised.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import List, Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgsplit.so")

GSPLIT_F32, GSPLIT_BF16 = 0, 1
MAX_SPLITS = 8

EXPORTS = [
    "gsplit_create", "gsplit_destroy", "gsplit_last_error", "gsplit_max_rows", "gsplit_sample_split",
    "gsplit_batch_sizes", "gsplit_batch_level", "gsplit_batch_layer", "gsplit_gather_features",
    "gsplit_sage_fwd", "gsplit_sage_bwd", "gsplit_softmax_xent", "gsplit_timing_enable",
    "gsplit_timing_read", "gsplit_presample_accumulate", "gsplit_presample_weights",
    "gsplit_gat_fwd", "gsplit_gat_bwd", "gsplit_batch_stats", "gsplit_sample_split_dev",
    "gsplit_input_counts_accumulate", "gsplit_cache_build", "gsplit_gather_features_cached",
    "gsplit_batch_shuffle", "gsplit_sage_activations", "gsplit_gat_score_terms", "gsplit_sample_split_noalloc",
    "gsplit_sample_split_multi", "gsplit_sage_step", "gsplit_gather_features_multi",
    "gsplit_policy_loss", "gsplit_preference_loss", "gsplit_grad_norm", "gsplit_clip_grads", "gsplit_adamw_step",
    "gsplit_group_rows", "gsplit_grouped_linear_fwd", "gsplit_grouped_linear_work", "gsplit_grouped_linear_bwd",
    "gsplit_orthogonalize_work", "gsplit_orthogonalize", "gsplit_muon_work", "gsplit_muon_step",
]


class GsplitError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"gsplit error {code}: {msg}")
        self.code = code


class _Graph(C.Structure):
    _fields_ = [("n_vertices", C.c_int64), ("n_edges", C.c_int64), ("d_indptr", C.c_void_p),
                ("indptr_is_64", C.c_int32), ("d_indices", C.c_void_p), ("d_pmap", C.c_void_p),
                ("n_splits", C.c_int32)]


class _Config(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("fanouts", C.POINTER(C.c_int32)), ("max_targets", C.c_int64),
                ("keep_edge_ids", C.c_int32), ("gat_index", C.c_int32), ("sampler_blocks_per_cu", C.c_int32),
                ("table_mode", C.c_int32)]


class _LevelView(C.Structure):
    _fields_ = [("d_local_cat", C.c_void_p), ("d_local_off", C.c_void_p)]


class _LayerView(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("d_nbr", "d_cnt", "d_mixed_cat", "d_mixed_off", "d_blk_indptr",
                                          "d_blk_src", "d_shuffle_src_row", "d_recv_cat", "d_recv_off")]


class _ShuffleView(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("d_self_row", "d_edge_row", "d_rev_ptr", "d_rev_cnt", "d_rev_list",
                                          "d_rev_eid")]


MAX_LAYERS = 8


class _BatchOut(C.Structure):
    _fields_ = [("d_local_cat", C.c_void_p * (MAX_LAYERS + 1)), ("d_local_off", C.c_void_p),
                ("d_nbr", C.c_void_p * MAX_LAYERS), ("d_cnt", C.c_void_p * MAX_LAYERS),
                ("d_mixed_cat", C.c_void_p * MAX_LAYERS), ("d_mixed_off", C.c_void_p),
                ("d_blk_indptr", C.c_void_p * MAX_LAYERS), ("d_blk_src", C.c_void_p * MAX_LAYERS),
                ("d_shuffle_src_row", C.c_void_p * MAX_LAYERS), ("d_recv_cat", C.c_void_p * MAX_LAYERS),
                ("d_recv_off", C.c_void_p)]


class _SageParams(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("dims", C.POINTER(C.c_int32)), ("d_w_self", C.POINTER(C.c_void_p)),
                ("d_w_neigh", C.POINTER(C.c_void_p)), ("d_bias", C.POINTER(C.c_void_p))]


class _GatParams(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("dims", C.POINTER(C.c_int32)), ("heads", C.POINTER(C.c_int32)),
                ("d_w", C.POINTER(C.c_void_p)), ("d_a_src", C.POINTER(C.c_void_p)),
                ("d_a_dst", C.POINTER(C.c_void_p)), ("d_bias", C.POINTER(C.c_void_p))]


class _PolicyConfig(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("clip_low", C.c_float), ("clip_high", C.c_float), ("kl_coef", C.c_float)]


class _PreferenceConfig(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("beta", C.c_float), ("label_smoothing", C.c_float)]


class _GradTensor(C.Structure):
    _fields_ = [("d_grad", C.c_void_p), ("d_out", C.c_void_p), ("n", C.c_int64), ("dtype", C.c_int32)]


class _AdamwTensor(C.Structure):
    _fields_ = [("d_param", C.c_void_p), ("d_master", C.c_void_p), ("d_grad", C.c_void_p), ("d_m", C.c_void_p),
                ("d_v", C.c_void_p), ("n", C.c_int64), ("param_dtype", C.c_int32), ("grad_dtype", C.c_int32)]


class _AdamwConfig(C.Structure):
    _fields_ = [(n, C.c_double) for n in ("lr", "beta1", "beta2", "eps", "weight_decay", "max_norm")] + [
        ("step", C.c_int64), ("d_step", C.c_void_p), ("d_lr", C.c_void_p)]


class _GroupedConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "n_groups", "n_in", "n_out")]


class _MatrixTensor(C.Structure):
    _fields_ = [("d_in", C.c_void_p), ("d_out", C.c_void_p), ("count", C.c_int64)] + [
        (n, C.c_int32) for n in ("rows", "cols", "in_dtype", "out_dtype")]


class _NewtonConfig(C.Structure):
    _fields_ = [(n, C.c_double) for n in ("a", "b", "c", "eps")] + [("steps", C.c_int32)]


class _MuonTensor(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("d_param", "d_master", "d_grad", "d_momentum")] + [("count", C.c_int64)] + [
        (n, C.c_int32) for n in ("rows", "cols", "param_dtype", "grad_dtype")]


class _MuonConfig(C.Structure):
    _fields_ = [("newton", _NewtonConfig), ("lr", C.c_double), ("momentum", C.c_double), ("weight_decay", C.c_double), ("d_lr", C.c_void_p),
                ("nesterov", C.c_int32), ("scaling", C.c_int32)]


_lib = None


def load_library():
    """dlopen the in-tree HIP library; never falls back to anything else."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: run `python -c 'import __graft_entry__ as g; g.build()'` "
                          "(hipcc, gfx950) first; there is no non-HIP path")
    L = C.CDLL(LIB_PATH)
    vp, i32, i64, u64 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64
    L.gsplit_create.argtypes = [C.POINTER(vp), C.POINTER(_Graph), C.POINTER(_Config)]
    L.gsplit_destroy.argtypes = [vp]
    L.gsplit_last_error.argtypes = [vp]
    L.gsplit_last_error.restype = C.c_char_p
    L.gsplit_max_rows.argtypes = [vp, i32]
    L.gsplit_max_rows.restype = i64
    L.gsplit_sample_split.argtypes = [vp, vp, i64, u64, u64, vp]
    L.gsplit_sample_split_dev.argtypes = [vp, vp, i64, vp, vp]
    L.gsplit_batch_sizes.argtypes = [vp, C.POINTER(i64), C.POINTER(i64), C.POINTER(i64), C.POINTER(i64)]
    L.gsplit_batch_level.argtypes = [vp, i32, C.POINTER(_LevelView)]
    L.gsplit_batch_layer.argtypes = [vp, i32, C.POINTER(_LayerView)]
    L.gsplit_sample_split_multi.argtypes = [C.POINTER(vp), i32, C.POINTER(vp), C.POINTER(i64), u64, C.POINTER(u64), vp]
    L.gsplit_sample_split_noalloc.argtypes = [C.POINTER(_Graph), C.POINTER(_Config), vp, i64, u64, u64,
                                              C.POINTER(_BatchOut), vp]
    L.gsplit_batch_shuffle.argtypes = [vp, i32, C.POINTER(_ShuffleView)]
    L.gsplit_sage_activations.argtypes = [vp, i32, C.POINTER(vp)]
    L.gsplit_gat_score_terms.argtypes = [vp, i32, C.POINTER(vp), C.POINTER(i64), C.POINTER(i64), C.POINTER(i64)]
    L.gsplit_gather_features.argtypes = [vp, vp, i32, i64, i64, vp, vp]
    L.gsplit_gather_features_multi.argtypes = [C.POINTER(vp), i32, vp, i32, i64, i64, C.POINTER(vp), vp]
    L.gsplit_sage_fwd.argtypes = [vp, C.POINTER(_SageParams), vp, vp, vp]
    L.gsplit_sage_bwd.argtypes = [vp, C.POINTER(_SageParams), vp, C.POINTER(vp), C.POINTER(vp),
                                  C.POINTER(vp), vp]
    L.gsplit_softmax_xent.argtypes = [vp, vp, i32, vp, vp, vp, vp]
    L.gsplit_sage_step.argtypes = [vp, C.POINTER(_SageParams), vp, vp, vp, vp, C.POINTER(vp), C.POINTER(vp),
                                   C.POINTER(vp), vp]
    L.gsplit_timing_enable.argtypes = [vp, i32]
    L.gsplit_timing_read.argtypes = [vp, C.c_char_p, i64]
    L.gsplit_timing_read.restype = i64
    L.gsplit_presample_accumulate.argtypes = [vp, vp, vp, vp]
    L.gsplit_presample_weights.argtypes = [vp, vp, i64, i64, vp, vp]
    L.gsplit_batch_stats.argtypes = [vp, vp, vp, vp]
    L.gsplit_input_counts_accumulate.argtypes = [vp, vp, vp]
    L.gsplit_cache_build.argtypes = [vp, vp, i32, i64, i64, vp, C.POINTER(i64), vp]
    L.gsplit_gather_features_cached.argtypes = [vp, vp, vp, vp, vp]
    L.gsplit_gat_fwd.argtypes = [vp, C.POINTER(_GatParams), vp, vp, vp]
    L.gsplit_gat_bwd.argtypes = [vp, C.POINTER(_GatParams), vp, vp, C.POINTER(vp), C.POINTER(vp), C.POINTER(vp),
                                 C.POINTER(vp), vp]
    L.gsplit_policy_loss.argtypes = [vp, C.POINTER(_PolicyConfig), vp, i64, i32, i64, vp, vp, vp, vp, vp, vp, i64, vp, vp,
                                     vp, vp]
    L.gsplit_preference_loss.argtypes = [vp, C.POINTER(_PreferenceConfig), vp, i64, i32, i64, vp, vp, i64, vp, vp, vp, i64,
                                         vp, vp, vp, vp, vp]
    L.gsplit_grad_norm.argtypes = [vp, C.POINTER(_GradTensor), i64, vp, vp]
    L.gsplit_clip_grads.argtypes = [vp, C.POINTER(_GradTensor), i64, C.c_double, vp, vp]
    L.gsplit_adamw_step.argtypes = [vp, C.POINTER(_AdamwConfig), C.POINTER(_AdamwTensor), i64, vp, vp]
    L.gsplit_group_rows.argtypes = [vp, vp, i64, i32, vp, vp, vp]
    L.gsplit_grouped_linear_fwd.argtypes = [vp, C.POINTER(_GroupedConfig), vp, i64, i64, vp, vp, vp, vp, vp, i64, vp]
    L.gsplit_grouped_linear_work.argtypes = [vp, C.POINTER(_GroupedConfig), i64]
    L.gsplit_grouped_linear_work.restype = i64
    L.gsplit_grouped_linear_bwd.argtypes = [vp, C.POINTER(_GroupedConfig), vp, i64, i64, vp, vp, vp, vp, i64, vp, i64, vp, vp, vp, vp]
    L.gsplit_orthogonalize_work.argtypes = [C.POINTER(_MatrixTensor), i64]
    L.gsplit_orthogonalize_work.restype = i64
    L.gsplit_orthogonalize.argtypes = [vp, C.POINTER(_NewtonConfig), C.POINTER(_MatrixTensor), i64, vp, vp]
    L.gsplit_muon_work.argtypes = [C.POINTER(_MuonTensor), i64]
    L.gsplit_muon_work.restype = i64
    L.gsplit_muon_step.argtypes = [vp, C.POINTER(_MuonConfig), C.POINTER(_MuonTensor), i64, vp, vp]
    for name in EXPORTS:
        if name not in ("gsplit_last_error", "gsplit_max_rows", "gsplit_timing_read", "gsplit_grouped_linear_work", "gsplit_orthogonalize_work",
                        "gsplit_muon_work"):
            getattr(L, name).restype = C.c_int
    _lib = L
    return L


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _view(ptr: int, n: int, device, dtype=torch.int32) -> torch.Tensor:
    """Copy n values from a raw device pointer into a fresh tensor (test/inspection only)."""
    out = torch.empty(max(n, 0), dtype=dtype, device=device)
    if n > 0:
        hip = _hip_runtime()
        rc = hip.hipMemcpy(C.c_void_p(out.data_ptr()), C.c_void_p(ptr), C.c_size_t(out.element_size() * n), 3)
        if rc != 0:
            raise GsplitError(-4, f"hipMemcpy failed ({rc})")
    return out


def _view_i32(ptr: int, n: int, device) -> torch.Tensor:
    return _view(ptr, n, device, torch.int32)


_hip = None


def _hip_runtime():
    global _hip
    if _hip is None:
        for name in ("libamdhip64.so.7", "libamdhip64.so"):   # the runtime torch already loaded
            try:
                _hip = C.CDLL(name)
                break
            except OSError:
                continue
        if _hip is None:
            raise ImportError("libamdhip64.so not found")
        _hip.hipMemcpy.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_int]
        _hip.hipMemcpy.restype = C.c_int
    return _hip


def noalloc_output_sizes(n_vertices: int, n_splits: int, fanouts: Sequence[int], max_targets: int) -> dict:
    """Entries of every output buffer of gsplit_sample_split_noalloc, as include/gsplit.h states them."""
    L, S = len(fanouts), n_splits
    ub = [0] * (L + 1)
    ub[L] = max_targets
    for l in range(L - 1, -1, -1):
        ub[l] = min(n_vertices, ub[l + 1] * (1 + fanouts[l]))
    return {"local_cat": ub, "local_off": (L + 1) * (S + 1), "mixed_off": L * (S + 1), "recv_off": L * (S + 1),
            "nbr": [ub[l + 1] * fanouts[l] for l in range(L)], "cnt": [ub[l + 1] for l in range(L)],
            "blk_indptr": [ub[l + 1] + 1 for l in range(L)], "blk_src": [ub[l + 1] * fanouts[l] for l in range(L)],
            "recv_cat": [ub[l + 1] * fanouts[l] for l in range(L)],
            "mixed_cat": [ub[l + 1] * (1 + fanouts[l]) for l in range(L)],
            "shuffle_src_row": [ub[l + 1] * (1 + fanouts[l]) for l in range(L)]}


def gsplit_sample_split_noalloc(indptr: torch.Tensor, indices: torch.Tensor, pmap: torch.Tensor, n_splits: int,
                                fanouts: Sequence[int], max_targets: int, targets: torch.Tensor, seed: int, it: int,
                                out: dict):
    """gsplit_sample_split without a context and without any allocation inside the library.  `out` maps
    the field names of gsplit_batch_out (without the d_ prefix) to int32 device tensors (lists of
    tensors for the per-level / per-layer fields), sized as noalloc_output_sizes says."""
    lib = load_library()
    L = len(fanouts)
    assert indptr.is_cuda and indices.is_cuda and pmap.is_cuda and targets.is_cuda
    assert indptr.dtype in (torch.int32, torch.int64) and indices.dtype == torch.int32 and pmap.dtype == torch.uint8
    assert targets.dtype == torch.int32 and targets.is_contiguous()
    want = noalloc_output_sizes(indptr.numel() - 1, n_splits, fanouts, max_targets)
    o = _BatchOut()
    for name, sizes in want.items():
        t = out[name]
        if isinstance(sizes, list):
            assert len(t) == len(sizes)
            for k, (x, n) in enumerate(zip(t, sizes)):
                assert x.is_cuda and x.dtype == torch.int32 and x.is_contiguous() and x.numel() >= n, (name, k)
                getattr(o, "d_" + name)[k] = x.data_ptr()
        else:
            assert t.is_cuda and t.dtype == torch.int32 and t.is_contiguous() and t.numel() >= sizes, name
            setattr(o, "d_" + name, t.data_ptr())
    fan = (C.c_int32 * L)(*[int(f) for f in fanouts])
    g = _Graph(indptr.numel() - 1, indices.numel(), indptr.data_ptr(), int(indptr.dtype == torch.int64),
               indices.data_ptr(), pmap.data_ptr(), int(n_splits))
    c = _Config(L, fan, int(max_targets), 0, 0, 0, 0)
    with torch.cuda.device(indptr.device):
        rc = lib.gsplit_sample_split_noalloc(C.byref(g), C.byref(c), targets.data_ptr(), targets.numel(),
                                             C.c_uint64(seed), C.c_uint64(it), C.byref(o), _stream())
    if rc != 0:
        raise GsplitError(rc, (lib.gsplit_last_error(None) or b"").decode())


def gsplit_sample_split_multi(ctxs, targets, seed: int, iters):
    """Samples targets[b] into ctxs[b] for all b in one set of launches (contexts over the same graph
    and configuration)."""
    n = len(ctxs)
    assert n >= 1 and len(targets) == n and len(iters) == n
    for t in targets:
        assert t.is_cuda and t.dtype == torch.int32 and t.is_contiguous()
    hs = (C.c_void_p * n)(*[c.h.value for c in ctxs])
    tg = (C.c_void_p * n)(*[t.data_ptr() for t in targets])
    nt = (C.c_int64 * n)(*[t.numel() for t in targets])
    its = (C.c_uint64 * n)(*[int(i) for i in iters])
    for c, t in zip(ctxs, targets):
        c._targets = t
    rc = ctxs[0].lib.gsplit_sample_split_multi(hs, n, tg, nt, C.c_uint64(seed), its, _stream())
    ctxs[0]._check(rc)


def gsplit_gather_features_multi(ctxs, table: torch.Tensor, outs):
    """The loading step of ctxs[b] into outs[b] for all b in one launch."""
    n = len(ctxs)
    assert n >= 1 and len(outs) == n
    assert table.is_cuda and table.dim() == 2 and table.stride(1) == 1
    for o in outs:
        assert o.is_cuda and o.is_contiguous() and o.dtype == table.dtype and o.shape[1] == table.shape[1]
    dt = {torch.float32: GSPLIT_F32, torch.bfloat16: GSPLIT_BF16}[table.dtype]
    hs = (C.c_void_p * n)(*[c.h.value for c in ctxs])
    ps = (C.c_void_p * n)(*[o.data_ptr() for o in outs])
    rc = ctxs[0].lib.gsplit_gather_features_multi(hs, n, table.data_ptr(), dt, table.shape[1],
                                                  table.stride(0) * table.element_size(), ps, _stream())
    ctxs[0]._check(rc)


class SageParams:
    """Holds the marshalled gsplit_sage_params block (and keeps the tensors alive)."""

    def __init__(self, dims: Sequence[int], w_self: List[torch.Tensor], w_neigh: List[torch.Tensor],
                 bias: List[torch.Tensor], dtype: int = GSPLIT_F32):
        L = len(dims) - 1
        assert len(w_self) == len(w_neigh) == len(bias) == L
        for l in range(L):
            for w in (w_self[l], w_neigh[l]):
                assert w.is_cuda and w.dtype == torch.float32 and w.is_contiguous()
                assert tuple(w.shape) == (dims[l], dims[l + 1])
            assert bias[l].is_cuda and bias[l].dtype == torch.float32 and bias[l].numel() == dims[l + 1]
        self.dims = list(dims)
        self.tensors = (list(w_self), list(w_neigh), list(bias))
        self._dims = (C.c_int32 * (L + 1))(*dims)
        self._ws = (C.c_void_p * L)(*[w.data_ptr() for w in w_self])
        self._wn = (C.c_void_p * L)(*[w.data_ptr() for w in w_neigh])
        self._b = (C.c_void_p * L)(*[b.data_ptr() for b in bias])
        self.c = _SageParams(dtype, self._dims, self._ws, self._wn, self._b)
        self.dtype = dtype


class GatParams:
    """Holds the marshalled gsplit_gat_params block (and keeps the tensors alive)."""

    def __init__(self, dims: Sequence[int], heads: Sequence[int], w: List[torch.Tensor], a_src: List[torch.Tensor],
                 a_dst: List[torch.Tensor], bias: List[torch.Tensor]):
        L = len(dims) - 1
        assert len(heads) == len(w) == len(a_src) == len(a_dst) == len(bias) == L
        for l in range(L):
            width = heads[l] * dims[l + 1] if l == L - 1 else dims[l + 1]
            for t, n in ((w[l], dims[l] * width), (a_src[l], width), (a_dst[l], width), (bias[l], dims[l + 1])):
                assert t.is_cuda and t.dtype == torch.float32 and t.is_contiguous() and t.numel() == n
        self.dims, self.heads = list(dims), list(heads)
        self.widths = [heads[l] * dims[l + 1] if l == L - 1 else dims[l + 1] for l in range(L)]
        self.tensors = (list(w), list(a_src), list(a_dst), list(bias))
        self._dims = (C.c_int32 * (L + 1))(*dims)
        self._heads = (C.c_int32 * L)(*heads)
        self._ptrs = [(C.c_void_p * L)(*[t.data_ptr() for t in lst]) for lst in self.tensors]
        self.c = _GatParams(GSPLIT_F32, self._dims, self._heads, *self._ptrs)


_F32 = torch.float32
_DTYPES = {torch.float32: GSPLIT_F32, torch.bfloat16: GSPLIT_BF16}


def _same_device(ts):
    assert all(t.is_cuda and t.device == ts[0].device for t in ts)
    return ts[0].device if ts else None


def _assert_apart(written, read):
    """No tensor that is written overlaps another one."""
    runs = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size(), w)
                  for ts, w in ((written, True), (read, False)) for t in ts if t is not None and t.numel())
    end = end_written = 0
    for lo, hi, w in runs:
        assert lo >= (end if w else end_written), "tensors of a call overlap"
        end = max(end, hi)
        end_written = max(end_written, hi if w else 0)


class GradTensors:
    """Holds the marshalled gradient tensors of gsplit_grad_norm and gsplit_clip_grads (and keeps them
    alive).  outs: where the clipped gradients go; None, or the gradients themselves: in place.  norm_only: a
    table for gsplit_grad_norm alone, which writes none of its tensors: they may overlap, or be listed twice."""

    def __init__(self, grads: Sequence[torch.Tensor], outs: Optional[Sequence[torch.Tensor]] = None, norm_only: bool = False):
        assert not (norm_only and outs is not None)
        self.norm_only = norm_only
        outs = grads if outs is None else outs
        assert len(outs) == len(grads)
        self.device = _same_device([*grads, *outs])
        for g, o in zip(grads, outs):
            assert g.dtype in _DTYPES and g.is_contiguous()
            assert o.dtype == g.dtype and o.is_contiguous() and o.numel() == g.numel()
        if not norm_only:
            _assert_apart(outs, [g for g, o in zip(grads, outs) if g.data_ptr() != o.data_ptr()])
        self.tensors = (list(grads), list(outs))
        self.n = len(self.tensors[0])
        self.c = (_GradTensor * max(1, self.n))(*[_GradTensor(g.data_ptr(), o.data_ptr(), g.numel(), _DTYPES[g.dtype])
                                                  for g, o in zip(grads, outs)])


class AdamwTensors:
    """Holds the marshalled tensors of gsplit_adamw_step (and keeps them alive).  masters: the float copies
    of the bfloat16 parameters, None for the float ones (or None if there are none)."""

    def __init__(self, params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], m: Sequence[torch.Tensor],
                 v: Sequence[torch.Tensor], masters: Optional[Sequence[Optional[torch.Tensor]]] = None):
        masters = [None] * len(params) if masters is None else masters
        assert len(grads) == len(m) == len(v) == len(masters) == len(params)
        self.device = _same_device([*params, *grads, *m, *v, *[t for t in masters if t is not None]])
        for p, g, a, b, w in zip(params, grads, m, v, masters):
            assert p.dtype in _DTYPES and g.dtype in _DTYPES and (w is not None) == (p.dtype == torch.bfloat16)
            for t in (p, g, a, b, w):
                assert t is None or (t.is_contiguous() and t.numel() == p.numel())
            assert all(t is None or t.dtype == torch.float32 for t in (a, b, w))
        _assert_apart([*params, *masters, *m, *v], grads)
        self.tensors = (list(params), list(grads), list(m), list(v), list(masters))
        self.n = len(self.tensors[0])
        self.c = (_AdamwTensor * max(1, self.n))(*[
            _AdamwTensor(p.data_ptr(), None if w is None else w.data_ptr(), g.data_ptr(), a.data_ptr(), b.data_ptr(),
                         p.numel(), _DTYPES[p.dtype], _DTYPES[g.dtype])
            for p, g, a, b, w in zip(params, grads, m, v, masters)])


NEWTON_COEFFICIENTS = (3.4445, -4.7750, 2.0315)
MUON_SCALINGS = {"plain": 0, "shape": 1, "rms": 2}


def _stack_shape(t):
    """(count, rows, cols) of a matrix or a stack of them."""
    assert t.dim() in (2, 3) and t.is_contiguous()
    return (1, *t.shape) if t.dim() == 2 else tuple(t.shape)


def _newton_work(bytes_, device):
    if bytes_ < 0:
        raise GsplitError(int(bytes_), "sizes out of range")
    return torch.empty(bytes_, dtype=torch.uint8, device=device)


class MatrixTensors:
    """Holds the marshalled matrices of gsplit_orthogonalize, [rows, cols] or stacks [count, rows, cols], and the working memory of
    a call (and keeps them alive).  outs: where the results go; None, or the matrices themselves: in place."""

    def __init__(self, matrices: Sequence[torch.Tensor], outs: Optional[Sequence[torch.Tensor]] = None):
        outs = matrices if outs is None else outs
        assert len(outs) == len(matrices)
        self.device = _same_device([*matrices, *outs])
        for g, o in zip(matrices, outs):
            assert g.dtype in _DTYPES and o.dtype in _DTYPES and o.shape == g.shape and o.is_contiguous()
            assert g.data_ptr() != o.data_ptr() or g.dtype == o.dtype or g.numel() == 0
        _assert_apart(outs, [g for g, o in zip(matrices, outs) if g.data_ptr() != o.data_ptr()])
        self.tensors = (list(matrices), list(outs))
        self.n = len(self.tensors[0])
        self.c = (_MatrixTensor * max(1, self.n))(*[
            _MatrixTensor(g.data_ptr(), o.data_ptr(), *_stack_shape(g), _DTYPES[g.dtype], _DTYPES[o.dtype]) for g, o in zip(matrices, outs)])
        self.work = _newton_work(load_library().gsplit_orthogonalize_work(self.c, self.n), self.device)


class MuonTensors:
    """Holds the marshalled tensors of gsplit_muon_step, [rows, cols] or stacks [count, rows, cols], and the working memory of a
    call (and keeps them alive).  masters: the float copies of the bfloat16 parameters, None for the float ones (or None if there
    are none)."""

    def __init__(self, params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], momenta: Sequence[torch.Tensor],
                 masters: Optional[Sequence[Optional[torch.Tensor]]] = None):
        masters = [None] * len(params) if masters is None else masters
        assert len(grads) == len(momenta) == len(masters) == len(params)
        self.device = _same_device([*params, *grads, *momenta, *[t for t in masters if t is not None]])
        for p, g, m, w in zip(params, grads, momenta, masters):
            assert p.dtype in _DTYPES and g.dtype in _DTYPES and (w is not None) == (p.dtype == torch.bfloat16)
            assert all(t is None or (t.is_contiguous() and t.shape == p.shape) for t in (g, m, w))
            assert all(t is None or t.dtype == torch.float32 for t in (m, w))
        _assert_apart([*params, *masters, *momenta], grads)
        self.tensors = (list(params), list(grads), list(momenta), list(masters))
        self.n = len(self.tensors[0])
        self.c = (_MuonTensor * max(1, self.n))(*[
            _MuonTensor(p.data_ptr(), None if w is None else w.data_ptr(), g.data_ptr(), m.data_ptr(), *_stack_shape(p), _DTYPES[p.dtype],
                        _DTYPES[g.dtype]) for p, g, m, w in zip(params, grads, momenta, masters)])
        self.work = _newton_work(load_library().gsplit_muon_work(self.c, self.n), self.device)


class Context:
    """gsplit_ctx wrapper.  Methods mirror the C entry points one to one."""

    def __init__(self, indptr: torch.Tensor, indices: torch.Tensor, pmap: torch.Tensor, n_splits: int,
                 fanouts: Sequence[int], max_targets: int, keep_edge_ids: bool = False,
                 gat_index: bool = False, sampler_blocks_per_cu: int = 0, table_mode: int = 0):
        self.lib = load_library()
        assert indptr.is_cuda and indices.is_cuda and pmap.is_cuda
        assert indptr.dtype in (torch.int32, torch.int64) and indices.dtype == torch.int32
        assert pmap.dtype == torch.uint8
        assert indptr.is_contiguous() and indices.is_contiguous() and pmap.is_contiguous()
        self.device = indptr.device
        self.n_vertices = indptr.numel() - 1
        assert pmap.numel() == self.n_vertices
        self.S, self.L = int(n_splits), len(fanouts)
        self.fanouts = list(int(f) for f in fanouts)
        self._keep = (indptr, indices, pmap)
        self._fan = (C.c_int32 * self.L)(*self.fanouts)
        g = _Graph(self.n_vertices, indices.numel(), indptr.data_ptr(), int(indptr.dtype == torch.int64),
                   indices.data_ptr(), pmap.data_ptr(), self.S)
        self.n_edges = indices.numel()
        c = _Config(self.L, self._fan, int(max_targets), int(keep_edge_ids), int(gat_index), int(sampler_blocks_per_cu),
                    int(table_mode))
        h = C.c_void_p()
        with torch.cuda.device(self.device):
            rc = self.lib.gsplit_create(C.byref(h), C.byref(g), C.byref(c))
        if rc != 0:
            raise GsplitError(rc, (self.lib.gsplit_last_error(None) or b"").decode())
        self.h = h

    # -- plumbing ------------------------------------------------------------------------
    def _check(self, rc: int):
        if rc != 0:
            raise GsplitError(rc, (self.lib.gsplit_last_error(self.h) or b"").decode())

    def close(self):
        if getattr(self, "h", None):
            self.lib.gsplit_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- entry points ----------------------------------------------------------------------
    def gsplit_max_rows(self, level: int) -> int:
        r = self.lib.gsplit_max_rows(self.h, level)
        if r < 0:
            raise GsplitError(int(r), "gsplit_max_rows")
        return int(r)

    def gsplit_sample_split(self, targets: torch.Tensor, seed: int, it: int):
        assert targets.is_cuda and targets.dtype == torch.int32 and targets.is_contiguous()
        self._targets = targets
        self._check(self.lib.gsplit_sample_split(self.h, targets.data_ptr(), targets.numel(),
                                                 C.c_uint64(seed), C.c_uint64(it), _stream()))

    def gsplit_sample_split_dev(self, targets: torch.Tensor, seed_iter: torch.Tensor):
        """seed_iter: int64 device tensor [seed, iteration] read when the kernels run."""
        assert targets.is_cuda and targets.dtype == torch.int32 and targets.is_contiguous()
        assert seed_iter.is_cuda and seed_iter.dtype == torch.int64 and seed_iter.numel() == 2
        self._check(self.lib.gsplit_sample_split_dev(self.h, targets.data_ptr(), targets.numel(),
                                                     seed_iter.data_ptr(), _stream()))

    def gsplit_batch_sizes(self):
        S, L = self.S, self.L
        nl = (C.c_int64 * ((L + 1) * S))()
        nm = (C.c_int64 * (L * S))()
        ne = (C.c_int64 * (L * S))()
        bk = (C.c_int64 * (L * S * S))()
        self._check(self.lib.gsplit_batch_sizes(self.h, nl, nm, ne, bk))
        n_local = [[nl[l * S + s] for s in range(S)] for l in range(L + 1)]
        n_mixed = [[nm[l * S + s] for s in range(S)] for l in range(L)]
        n_edges = [[ne[l * S + s] for s in range(S)] for l in range(L)]
        bucket = [[[bk[(l * S + s) * S + t] for t in range(S)] for s in range(S)] for l in range(L)]
        return n_local, n_mixed, n_edges, bucket

    def gsplit_batch_level(self, level: int) -> _LevelView:
        v = _LevelView()
        self._check(self.lib.gsplit_batch_level(self.h, level, C.byref(v)))
        return v

    def gsplit_batch_layer(self, layer: int) -> _LayerView:
        v = _LayerView()
        self._check(self.lib.gsplit_batch_layer(self.h, layer, C.byref(v)))
        return v

    def gsplit_batch_shuffle(self, layer: int) -> _ShuffleView:
        v = _ShuffleView()
        self._check(self.lib.gsplit_batch_shuffle(self.h, layer, C.byref(v)))
        return v

    def gsplit_sage_activations(self, level: int) -> int:
        """Raw device pointer of the stored activations of local_cat[level]."""
        p = C.c_void_p()
        self._check(self.lib.gsplit_sage_activations(self.h, level, C.byref(p)))
        return int(p.value or 0)

    def gsplit_gat_score_terms(self, layer: int):
        """(raw device pointer, row stride, column of the src terms, column of the dst terms)."""
        p, st, sc, dc = C.c_void_p(), C.c_int64(), C.c_int64(), C.c_int64()
        self._check(self.lib.gsplit_gat_score_terms(self.h, layer, C.byref(p), C.byref(st), C.byref(sc), C.byref(dc)))
        return int(p.value or 0), int(st.value), int(sc.value), int(dc.value)

    def gsplit_gather_features(self, table: torch.Tensor, out: torch.Tensor):
        assert table.is_cuda and out.is_cuda and table.dim() == 2 and table.stride(1) == 1
        assert out.is_contiguous() and out.dtype == table.dtype and out.shape[1] == table.shape[1]
        dt = {torch.float32: GSPLIT_F32, torch.bfloat16: GSPLIT_BF16}[table.dtype]
        self._check(self.lib.gsplit_gather_features(self.h, table.data_ptr(), dt, table.shape[1],
                                                    table.stride(0) * table.element_size(),
                                                    out.data_ptr(), _stream()))

    def gsplit_sage_fwd(self, params: SageParams, feat_local: torch.Tensor, logits: torch.Tensor):
        assert feat_local.is_cuda and feat_local.is_contiguous() and logits.is_cuda and logits.is_contiguous()
        assert logits.dtype == torch.float32
        assert feat_local.dtype == (torch.bfloat16 if params.dtype == GSPLIT_BF16 else torch.float32)
        self._fwd_keep = (params, feat_local)
        self._check(self.lib.gsplit_sage_fwd(self.h, C.byref(params.c), feat_local.data_ptr(),
                                             logits.data_ptr(), _stream()))

    def gsplit_sage_bwd(self, params: SageParams, grad_logits: torch.Tensor, gw_self, gw_neigh, gbias):
        L = self.L
        assert grad_logits.is_cuda and grad_logits.dtype == torch.float32 and grad_logits.is_contiguous()
        for lst in (gw_self, gw_neigh, gbias):
            assert len(lst) == L and all(t.is_cuda and t.dtype == torch.float32 and t.is_contiguous()
                                         for t in lst)
        a = (C.c_void_p * L)(*[t.data_ptr() for t in gw_self])
        b = (C.c_void_p * L)(*[t.data_ptr() for t in gw_neigh])
        c = (C.c_void_p * L)(*[t.data_ptr() for t in gbias])
        self._check(self.lib.gsplit_sage_bwd(self.h, C.byref(params.c), grad_logits.data_ptr(), a, b, c,
                                             _stream()))

    def gsplit_sage_step(self, params: SageParams, feat_local: torch.Tensor, labels: torch.Tensor, logits: torch.Tensor,
                         gw_self, gw_neigh, gbias, row_loss: Optional[torch.Tensor] = None):
        L = self.L
        assert feat_local.is_cuda and feat_local.is_contiguous() and logits.is_cuda and logits.is_contiguous()
        assert logits.dtype == torch.float32
        assert feat_local.dtype == (torch.bfloat16 if params.dtype == GSPLIT_BF16 else torch.float32)
        assert labels.is_cuda and labels.dtype == torch.int64 and labels.numel() == self.n_vertices
        for lst in (gw_self, gw_neigh, gbias):
            assert len(lst) == L and all(t.is_cuda and t.dtype == torch.float32 and t.is_contiguous() for t in lst)
        if row_loss is not None:
            assert row_loss.is_cuda and row_loss.dtype == torch.float32 and row_loss.numel() >= logits.shape[0]
        a = (C.c_void_p * L)(*[t.data_ptr() for t in gw_self])
        b = (C.c_void_p * L)(*[t.data_ptr() for t in gw_neigh])
        c = (C.c_void_p * L)(*[t.data_ptr() for t in gbias])
        self._fwd_keep = (params, feat_local)
        self._check(self.lib.gsplit_sage_step(self.h, C.byref(params.c), feat_local.data_ptr(), labels.data_ptr(),
                                              logits.data_ptr(), row_loss.data_ptr() if row_loss is not None else None,
                                              a, b, c, _stream()))

    def gsplit_gat_fwd(self, params: GatParams, feat_local: torch.Tensor, logits: torch.Tensor):
        assert feat_local.is_cuda and feat_local.is_contiguous() and feat_local.dtype == torch.float32
        assert feat_local.shape[1] == params.dims[0]
        assert logits.is_cuda and logits.dtype == torch.float32 and logits.is_contiguous()
        assert logits.shape[1] == params.dims[-1]
        self._check(self.lib.gsplit_gat_fwd(self.h, C.byref(params.c), feat_local.data_ptr(), logits.data_ptr(),
                                            _stream()))

    def gsplit_gat_bwd(self, params: GatParams, feat_local: torch.Tensor, grad_logits: torch.Tensor, gw, ga_src,
                       ga_dst, gbias):
        L = self.L
        assert feat_local.is_cuda and feat_local.is_contiguous() and feat_local.dtype == torch.float32
        assert grad_logits.is_cuda and grad_logits.dtype == torch.float32 and grad_logits.is_contiguous()
        for lst in (gw, ga_src, ga_dst, gbias):
            assert len(lst) == L and all(t.is_cuda and t.dtype == torch.float32 and t.is_contiguous() for t in lst)
        for l in range(L):
            assert gw[l].numel() == params.dims[l] * params.widths[l] and gbias[l].numel() == params.dims[l + 1]
            assert ga_src[l].numel() == params.widths[l] and ga_dst[l].numel() == params.widths[l]
        ptrs = [(C.c_void_p * L)(*[t.data_ptr() for t in lst]) for lst in (gw, ga_src, ga_dst, gbias)]
        self._check(self.lib.gsplit_gat_bwd(self.h, C.byref(params.c), feat_local.data_ptr(), grad_logits.data_ptr(),
                                            *ptrs, _stream()))

    def gsplit_softmax_xent(self, logits: torch.Tensor, labels: torch.Tensor, grad_logits: torch.Tensor,
                            row_loss: Optional[torch.Tensor] = None):
        assert logits.is_cuda and logits.dtype == torch.float32 and logits.is_contiguous()
        assert labels.is_cuda and labels.dtype == torch.int64 and labels.numel() == self.n_vertices
        assert grad_logits.is_cuda and grad_logits.dtype == torch.float32 and grad_logits.is_contiguous()
        assert grad_logits.shape == logits.shape
        if row_loss is not None:
            assert row_loss.is_cuda and row_loss.dtype == torch.float32 and row_loss.numel() >= logits.shape[0]
        self._check(self.lib.gsplit_softmax_xent(self.h, logits.data_ptr(), logits.shape[1], labels.data_ptr(),
                                                 grad_logits.data_ptr(),
                                                 row_loss.data_ptr() if row_loss is not None else None,
                                                 _stream()))

    # The calls below need no batch: tensors on the context's device, whichever device is current
    def _own_stream(self) -> int:
        # (the raw handle: torch.cuda.current_stream() builds a Stream object, 2 us of a call that takes 7)
        return torch._C._cuda_getCurrentRawStream(self.device.index)

    # (a small call is the host's time: one pass over the tensors checks them and takes their addresses)
    def _vectors(self, tensors, n):
        """Addresses of float32 vectors of n values (None: absent)."""
        dev, out = self.device.index, []
        for t in tensors:
            if t is None:
                out.append(None)
            else:
                assert t.dtype is _F32 and t.numel() == n and t.is_contiguous() and t.get_device() == dev
                out.append(t.data_ptr())
        return out

    def _rows(self, logits, grad_logits, actions):
        """(dtype, rows, classes, logits stride, address of the gradient, its stride)"""
        dt = _DTYPES.get(logits.dtype)
        assert dt is not None and logits.dim() == 2
        dev = self.device.index
        rows, classes = logits.shape
        ld, step = logits.stride()
        assert (step == 1 or classes == 1) and logits.get_device() == dev
        assert actions.dtype is torch.int64 and actions.numel() == rows and actions.is_contiguous() and actions.get_device() == dev
        grad, gld = None, classes
        if grad_logits is not None:
            assert grad_logits.dtype is logits.dtype and grad_logits.shape == logits.shape and grad_logits.get_device() == dev
            gld, step = grad_logits.stride()
            assert step == 1 or classes == 1
            grad = grad_logits.data_ptr()
        if rows <= 1:
            ld = gld = classes          # (one row: any stride)
        return dt, rows, classes, ld, grad, gld

    def gsplit_policy_loss(self, logits: torch.Tensor, actions: torch.Tensor, old_logp: torch.Tensor,
                           advantages: torch.Tensor, grad_logits: Optional[torch.Tensor],
                           ref_logp: Optional[torch.Tensor] = None, row_weight: Optional[torch.Tensor] = None,
                           clip_low: float = 0.2, clip_high: float = 0.2, kl_coef: float = 0.0,
                           row_loss: Optional[torch.Tensor] = None, row_logp: Optional[torch.Tensor] = None,
                           row_kl: Optional[torch.Tensor] = None):
        """Clipped policy loss with a KL term of every row of logits, and its gradient."""
        dt, rows, classes, ld, grad, gld = self._rows(logits, grad_logits, actions)
        old, adv, ref, w, loss, logp, kl = self._vectors((old_logp, advantages, ref_logp, row_weight, row_loss, row_logp, row_kl), rows)
        rc = self.lib.gsplit_policy_loss(self.h, C.byref(_PolicyConfig(dt, clip_low, clip_high, kl_coef)), logits.data_ptr(), rows,
                                         classes, ld, actions.data_ptr(), old, ref, adv, w, grad, gld, loss, logp, kl, self._own_stream())
        if rc:
            self._check(rc)

    def gsplit_preference_loss(self, logits: torch.Tensor, actions: torch.Tensor, seq_ptr: torch.Tensor,
                               grad_logits: Optional[torch.Tensor], row_work: torch.Tensor,
                               ref_logp: Optional[torch.Tensor] = None, pair_weight: Optional[torch.Tensor] = None,
                               beta: float = 0.1, label_smoothing: float = 0.0,
                               pair_loss: Optional[torch.Tensor] = None, pair_margin: Optional[torch.Tensor] = None,
                               row_logp: Optional[torch.Tensor] = None):
        """Preference loss of pairs of sequences of rows (2 p preferred to 2 p + 1), and its gradient.
        row_work: float32, 4 values a row."""
        dt, rows, classes, ld, grad, gld = self._rows(logits, grad_logits, actions)
        n = seq_ptr.numel()
        assert n % 2 == 1 and seq_ptr.dtype is torch.int64 and seq_ptr.is_contiguous() and seq_ptr.get_device() == self.device.index
        w, loss, margin = self._vectors((pair_weight, pair_loss, pair_margin), n // 2)
        ref, = self._vectors((ref_logp,), n - 1)
        logp, = self._vectors((row_logp,), rows)
        work, = self._vectors((row_work,), 4 * rows)
        rc = self.lib.gsplit_preference_loss(self.h, C.byref(_PreferenceConfig(dt, beta, label_smoothing)), logits.data_ptr(), rows,
                                             classes, ld, actions.data_ptr(), seq_ptr.data_ptr(), n // 2, ref, w, grad, gld, logp, loss,
                                             margin, work, self._own_stream())
        if rc:
            self._check(rc)

    def _table(self, table, norm):
        """Address of the norm, for a table of this device."""
        assert table.device is None or table.device == self.device
        return self._vectors((norm,), 1)[0]

    def gsplit_grad_norm(self, grads: GradTensors, norm: torch.Tensor):
        self._check(self.lib.gsplit_grad_norm(self.h, grads.c, grads.n, self._table(grads, norm), self._own_stream()))

    def gsplit_clip_grads(self, grads: GradTensors, max_norm: float, norm: Optional[torch.Tensor] = None):
        """Gradients times min(1, max_norm / their global norm) into the table's outputs."""
        assert not grads.norm_only
        self._check(self.lib.gsplit_clip_grads(self.h, grads.c, grads.n, max_norm, self._table(grads, norm), self._own_stream()))

    def gsplit_adamw_step(self, tensors: AdamwTensors, lr: float = 1e-3, beta1: float = 0.9, beta2: float = 0.999,
                          eps: float = 1e-8, weight_decay: float = 0.01, step: int = 0, max_norm: float = 0.0,
                          norm: Optional[torch.Tensor] = None, step_dev: Optional[torch.Tensor] = None,
                          lr_dev: Optional[torch.Tensor] = None):
        """AdamW step number `step` (from 1), gradients clipped to max_norm (0: as they are).  step_dev (int64)
        and lr_dev (float32): the step and the learning rate in device memory, for captured steps."""
        norm = self._table(tensors, norm)
        if step_dev is not None:
            assert step_dev.dtype is torch.int64 and step_dev.numel() == 1 and step_dev.device == self.device
        cfg = _AdamwConfig(lr, beta1, beta2, eps, weight_decay, max_norm, step, None if step_dev is None else step_dev.data_ptr(),
                           self._vectors((lr_dev,), 1)[0])
        self._check(self.lib.gsplit_adamw_step(self.h, C.byref(cfg), tensors.c, tensors.n, norm, self._own_stream()))

    def gsplit_group_rows(self, group: torch.Tensor, group_ptr: torch.Tensor, rows: torch.Tensor):
        """Rows sorted by their group: group [n] int32 -> group_ptr [groups + 1], rows [n] int32."""
        dev = self.device.index
        for t in (group, group_ptr, rows):
            assert t.dtype is torch.int32 and t.is_contiguous() and t.get_device() == dev
        assert rows.numel() == group.numel() and (group.numel() == 0 or rows.data_ptr() != group.data_ptr())
        rc = self.lib.gsplit_group_rows(self.h, group.data_ptr(), group.numel(), group_ptr.numel() - 1, group_ptr.data_ptr(),
                                        rows.data_ptr(), self._own_stream())
        if rc:
            self._check(rc)

    def _grouped(self, x, group_ptr, rows, w):
        """(config, n_rows, address of the offsets, of the list of rows or None)"""
        dt, dev = _DTYPES.get(x.dtype), self.device.index
        assert dt is not None and x.dim() == 2 and w.dim() == 3 and w.dtype is x.dtype and w.is_contiguous() and w.get_device() == dev
        groups, n_in, n_out = w.shape
        assert group_ptr.dtype is torch.int32 and group_ptr.is_contiguous() and group_ptr.numel() == groups + 1 and group_ptr.get_device() == dev
        if rows is not None:
            assert rows.dtype is torch.int32 and rows.is_contiguous() and rows.numel() == x.shape[0] and rows.get_device() == dev
        return _GroupedConfig(dt, groups, n_in, n_out), x.shape[0], group_ptr.data_ptr(), None if rows is None else rows.data_ptr()

    def _matrix(self, t, like, width):
        """(address, row stride) of a matrix of `like`'s rows and type."""
        assert t.dtype is like.dtype and t.dim() == 2 and t.shape[0] == like.shape[0] and t.shape[1] == width and t.get_device() == self.device.index
        ld, step = t.stride()
        assert step == 1 or width == 1
        return t.data_ptr(), ld if t.shape[0] > 1 else width

    def gsplit_grouped_linear_fwd(self, x: torch.Tensor, group_ptr: torch.Tensor, rows: Optional[torch.Tensor], w: torch.Tensor,
                                  bias: Optional[torch.Tensor], y: torch.Tensor):
        """y[r] = x[r] W[g] + bias[g] for the rows r of every group g; rows None: they lie sorted by group."""
        cfg, n, ptr, order = self._grouped(x, group_ptr, rows, w)
        xp, ldx = self._matrix(x, x, cfg.n_in)
        yp, ldy = self._matrix(y, x, cfg.n_out)
        assert n == 0 or yp != xp           # (rows are written while others still read them)
        b, = self._vectors((bias,), cfg.n_groups * cfg.n_out)
        rc = self.lib.gsplit_grouped_linear_fwd(self.h, C.byref(cfg), xp, n, ldx, ptr, order, w.data_ptr(), b, yp, ldy, self._own_stream())
        if rc:
            self._check(rc)

    def gsplit_grouped_linear_work(self, x: torch.Tensor, w: torch.Tensor) -> torch.Tensor:
        """Working memory for gsplit_grouped_linear_bwd with these rows and weights."""
        cfg = _GroupedConfig(_DTYPES[x.dtype], *w.shape)
        n = self.lib.gsplit_grouped_linear_work(self.h, C.byref(cfg), x.shape[0])
        if n < 0:
            self._check(int(n))
        return torch.empty(n // 4, dtype=torch.float32, device=self.device)

    def gsplit_grouped_linear_bwd(self, x: torch.Tensor, group_ptr: torch.Tensor, rows: Optional[torch.Tensor], w: torch.Tensor,
                                  dy: torch.Tensor, dx: Optional[torch.Tensor], dw: Optional[torch.Tensor],
                                  dbias: Optional[torch.Tensor], work: Optional[torch.Tensor] = None):
        """The gradients of gsplit_grouped_linear_fwd (None: not asked for); dw and dbias are float32."""
        cfg, n, ptr, order = self._grouped(x, group_ptr, rows, w)
        xp, ldx = self._matrix(x, x, cfg.n_in)
        dyp, lddy = self._matrix(dy, x, cfg.n_out)
        dxp, lddx = (None, 0) if dx is None else self._matrix(dx, x, cfg.n_in)
        assert n == 0 or dxp not in (xp, dyp)
        dwp, = self._vectors((dw,), w.numel())
        dbp, = self._vectors((dbias,), cfg.n_groups * cfg.n_out)
        if dw is not None:
            need = self.lib.gsplit_grouped_linear_work(self.h, C.byref(cfg), n)
            assert need <= 0 or (work is not None and work.is_contiguous() and work.numel() * work.element_size() >= need
                                 and work.get_device() == self.device.index)
        rc = self.lib.gsplit_grouped_linear_bwd(self.h, C.byref(cfg), xp, n, ldx, ptr, order, w.data_ptr(), dyp, lddy, dxp, lddx, dwp, dbp,
                                                None if work is None else work.data_ptr(), self._own_stream())
        if rc:
            self._check(rc)

    def gsplit_orthogonalize(self, matrices: MatrixTensors, steps: int = 5,
                             coefficients: Sequence[float] = NEWTON_COEFFICIENTS, eps: float = 1e-7):
        """Newton-Schulz steps X <- (a I + b X X^T + c (X X^T)^2) X from every matrix over its norm, into the table's outputs."""
        assert matrices.device is None or matrices.device == self.device
        cfg = _NewtonConfig(*coefficients, eps, steps)
        self._check(self.lib.gsplit_orthogonalize(self.h, C.byref(cfg), matrices.c, matrices.n, matrices.work.data_ptr(), self._own_stream()))

    def gsplit_muon_step(self, tensors: MuonTensors, lr: float = 0.02, momentum: float = 0.95, nesterov: bool = True,
                         weight_decay: float = 0.0, scaling: str = "shape", steps: int = 5,
                         coefficients: Sequence[float] = NEWTON_COEFFICIENTS, eps: float = 1e-7, lr_dev: Optional[torch.Tensor] = None):
        """One step of orthogonalised momentum for matrices.  scaling: "plain", "shape" or "rms" (see gsplit.h); lr_dev (float32): the
        learning rate in device memory, for captured steps."""
        assert tensors.device is None or tensors.device == self.device
        cfg = _MuonConfig(_NewtonConfig(*coefficients, eps, steps), lr, momentum, weight_decay, self._vectors((lr_dev,), 1)[0], int(nesterov),
                          MUON_SCALINGS[scaling])
        self._check(self.lib.gsplit_muon_step(self.h, C.byref(cfg), tensors.c, tensors.n, tensors.work.data_ptr(), self._own_stream()))

    def gsplit_presample_accumulate(self, vertex_count: Optional[torch.Tensor], edge_count: Optional[torch.Tensor]):
        # torch has no unsigned 32-bit arithmetic: int32 tensors carry the uint32 counters
        for t, n in ((vertex_count, self.n_vertices), (edge_count, self.n_edges)):
            if t is not None:
                assert t.is_cuda and t.dtype == torch.int32 and t.is_contiguous() and t.numel() == n
        self._check(self.lib.gsplit_presample_accumulate(
            self.h, vertex_count.data_ptr() if vertex_count is not None else None,
            edge_count.data_ptr() if edge_count is not None else None, _stream()))

    def gsplit_batch_stats(self, edges: torch.Tensor, cross_edges: torch.Tensor):
        # int64 tensors carry the uint64 counters
        for t in (edges, cross_edges):
            assert t.is_cuda and t.dtype == torch.int64 and t.is_contiguous() and t.numel() == self.L * self.S
        self._check(self.lib.gsplit_batch_stats(self.h, edges.data_ptr(), cross_edges.data_ptr(), _stream()))

    def gsplit_input_counts_accumulate(self, count: torch.Tensor):
        assert count.is_cuda and count.dtype == torch.int32 and count.is_contiguous() and count.numel() == self.n_vertices
        self._check(self.lib.gsplit_input_counts_accumulate(self.h, count.data_ptr(), _stream()))

    def gsplit_cache_build(self, table: torch.Tensor, cache_ids: torch.Tensor, n_cache: Sequence[int]):
        """table: [n_vertices, dim] float32 / bfloat16, on the device or in pinned host memory."""
        assert table.dim() == 2 and table.stride(1) == 1 and table.shape[0] == self.n_vertices
        assert table.dtype in (torch.float32, torch.bfloat16) and (table.is_cuda or table.is_pinned())
        assert cache_ids.is_cuda and cache_ids.dtype == torch.int32 and cache_ids.is_contiguous()
        assert len(n_cache) == self.S and sum(n_cache) == cache_ids.numel()
        self._cache_keep = (table, cache_ids)
        self._cache_dim, self._cache_dtype = table.shape[1], table.dtype
        self._check(self.lib.gsplit_cache_build(
            self.h, table.data_ptr(), GSPLIT_F32 if table.dtype == torch.float32 else GSPLIT_BF16, table.shape[1],
            table.stride(0) * table.element_size(), cache_ids.data_ptr(), (C.c_int64 * self.S)(*[int(x) for x in n_cache]),
            _stream()))

    def gsplit_gather_features_cached(self, out: torch.Tensor, hits: Optional[torch.Tensor] = None,
                                      misses: Optional[torch.Tensor] = None):
        assert out.is_cuda and out.is_contiguous() and out.dtype == self._cache_dtype and out.shape[1] == self._cache_dim
        for t in (hits, misses):      # int64 tensors carry the uint64 counters
            assert t is None or (t.is_cuda and t.dtype == torch.int64 and t.is_contiguous() and t.numel() == self.S)
        self._check(self.lib.gsplit_gather_features_cached(
            self.h, out.data_ptr(), hits.data_ptr() if hits is not None else None,
            misses.data_ptr() if misses is not None else None, _stream()))

    def gsplit_presample_weights(self, count: torch.Tensor, n_samples: int, weight: torch.Tensor):
        assert count.is_cuda and count.dtype == torch.int32 and count.is_contiguous()
        assert weight.is_cuda and weight.dtype == torch.float32 and weight.is_contiguous()
        assert weight.numel() == count.numel()
        self._check(self.lib.gsplit_presample_weights(self.h, count.data_ptr(), count.numel(), int(n_samples),
                                                      weight.data_ptr(), _stream()))

    def gsplit_timing_enable(self, enable: bool):
        self._check(self.lib.gsplit_timing_enable(self.h, int(enable)))

    def gsplit_timing_read(self) -> dict:
        """{label: (launches, total_ms)} since the last read."""
        buf = C.create_string_buffer(1 << 16)
        n = self.lib.gsplit_timing_read(self.h, buf, len(buf))
        if n < 0:
            self._check(int(n))
        out = {}
        for line in buf.value.decode().splitlines():
            name, cnt, ms = line.split()
            out[name] = (int(cnt), float(ms))
        return out

    # -- inspection helpers for tests (copies of the device views; they synchronise) -------
    def fetch_batch(self) -> dict:
        """Copies the whole current batch to torch tensors, split by split (tests only)."""
        S, L = self.S, self.L
        n_local, n_mixed, n_edges, bucket = self.gsplit_batch_sizes()
        dev = self.device
        out = {"n_local": n_local, "n_mixed": n_mixed, "n_edges": n_edges, "bucket": bucket,
               "local_front": [], "layers": []}
        for l in range(L + 1):
            v = self.gsplit_batch_level(l)
            cat = _view_i32(v.d_local_cat, sum(n_local[l]), dev)
            off = _view_i32(v.d_local_off, S + 1, dev)
            assert off.tolist() == [sum(n_local[l][:s]) for s in range(S + 1)]
            out["local_front"].append(list(torch.split(cat, n_local[l])))
        for l in range(L):
            v = self.gsplit_batch_layer(l)
            fan = self.fanouts[l]
            n_dst = sum(n_local[l + 1])
            lay = {
                "nbr": _view_i32(v.d_nbr, n_dst * fan, dev).view(n_dst, fan),
                "cnt": _view_i32(v.d_cnt, n_dst, dev),
                "mixed": list(torch.split(_view_i32(v.d_mixed_cat, sum(n_mixed[l]), dev), n_mixed[l])),
                "blk_indptr": _view_i32(v.d_blk_indptr, n_dst + 1, dev),
                "blk_src": _view_i32(v.d_blk_src, sum(n_edges[l]), dev),
                "shuffle_src_row": list(torch.split(_view_i32(v.d_shuffle_src_row, sum(n_mixed[l]), dev),
                                                    n_mixed[l])),
                "recv": _view_i32(v.d_recv_cat, sum(sum(r) for r in bucket[l]), dev),
                "recv_off": _view_i32(v.d_recv_off, S + 1, dev),
            }
            out["layers"].append(lay)
        return out

    def fetch_shuffle(self, layer: int) -> dict:
        """Copies of the composed gather side and of the scatter side of shuffle_idx[layer] (tests only)."""
        n_local, _, n_edges, _ = self.gsplit_batch_sizes()
        dev = self.device
        v = self.gsplit_batch_shuffle(layer)
        n_dst, nnz, n_lo = sum(n_local[layer + 1]), sum(n_edges[layer]), sum(n_local[layer])
        out = {"self_row": _view_i32(v.d_self_row, n_dst, dev), "edge_row": _view_i32(v.d_edge_row, nnz, dev),
               "rev_ptr": None, "rev_cnt": None, "rev_list": None, "rev_eid": None}
        if v.d_rev_list:
            out["rev_ptr"] = _view_i32(v.d_rev_ptr, n_lo, dev)
            out["rev_cnt"] = _view_i32(v.d_rev_cnt, n_lo, dev)
            out["rev_list"] = _view_i32(v.d_rev_list, n_dst + nnz, dev)
            if v.d_rev_eid:
                out["rev_eid"] = _view_i32(v.d_rev_eid, n_dst + nnz, dev)
        return out

    def fetch_sage_activations(self, level: int, width: int, dtype=torch.float32) -> torch.Tensor:
        """Copy of the stored activations of local_cat[level] as [rows, width] (tests only)."""
        n_local, _, _, _ = self.gsplit_batch_sizes()
        rows = sum(n_local[level])
        return _view(self.gsplit_sage_activations(level), rows * width, self.device, dtype).view(rows, width)

    def fetch_gat_score_terms(self, layer: int, heads: int):
        """Copies of the per-row score terms of a GAT layer: (src [rows, K], dst [rows, K]) (tests only)."""
        n_local, _, _, _ = self.gsplit_batch_sizes()
        rows = sum(n_local[layer])
        ptr, stride, sc, dc = self.gsplit_gat_score_terms(layer)
        raw = _view(ptr, rows * stride, self.device, torch.float32).view(rows, stride)
        return raw[:, sc:sc + heads].contiguous(), raw[:, dc:dc + heads].contiguous()
