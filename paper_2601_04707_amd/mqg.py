"""ctypes binding of libmqg.so - argument marshalling only.

The four operations keep the names of the C ABI (``include/mqg.h``):
``mqg_build_cache``, ``mqg_sample_blocks``, ``mqg_gather_features`` and
``mqg_sage_mean_aggregate``, and so do the calls of a layer (``mqg_rms_norm``,
``mqg_adamw_step`` and those between them in this file).  Torch is used for device memory, pinned host
memory and streams; every step of the path runs in the library's kernels.
There is no fallback: if the shared library is missing, importing this module
raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import List, Optional, Sequence

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libmqg.so")

MQG_OK, MQG_ERR_INVALID_ARG, MQG_ERR_CAPACITY, MQG_ERR_HIP, MQG_ERR_UNSUPPORTED = 0, -1, -2, -3, -4
MQG_F32, MQG_F16, MQG_BF16 = 0, 1, 2
MQG_Q_E4M3, MQG_Q_INT8 = 0, 1
MQG_NORM_MAX_DIM = 16384
MQG_STATE_F32, MQG_STATE_E4M3, MQG_ADAMW_BLOCK = 0, 1, 128
MQG_ORTH_MAX_STEPS, MQG_ORTH_MAX_SIDE, MQG_ORTH_MAX_MATS = 32, 65536, 65535
MQG_I32, MQG_I64 = 0, 1
MQG_OPT_FORCE_SLOW_SELECT, MQG_OPT_PROFILE, MQG_OPT_MISS_INFLIGHT_BYTES, MQG_OPT_HEAVY_DEGREE, MQG_OPT_DEDUP_HASH = 1, 2, 3, 4, 5
MQG_OPT_LAYERWISE_CANDIDATES = 6
MQG_MAX_FANOUT, MQG_MAX_LAYERS = 64, 8
MQG_CACHE_TOP_DEGREE, MQG_CACHE_DEGREE_SAMPLED, MQG_CACHE_RANDOM_WALK, MQG_CACHE_RANDOM_WALK_SAMPLED = 0, 1, 2, 3
MQG_WALK_PUSH, MQG_WALK_PRINTED = 0, 1

EXPORTS = [
    "mqg_version", "mqg_ctx_create", "mqg_ctx_destroy", "mqg_last_error", "mqg_ctx_set_option",
    "mqg_ctx_kernel_time", "mqg_ctx_reset_profile", "mqg_ctx_kernel_names", "mqg_build_cache",
    "mqg_sample_blocks", "mqg_gather_features", "mqg_sage_mean_aggregate", "mqg_sage_mean_aggregate_backward",
    "mqg_queue_size", "mqg_build_cache_ex", "mqg_gcn_edge_weights", "mqg_weighted_aggregate",
    "mqg_weighted_aggregate_backward", "mqg_ctx_set_sampling_priority", "mqg_sample_layerwise",
    "mqg_select_smallest_keys", "mqg_select_row_candidates", "mqg_sample_blocks_seed_dev",
    "mqg_gather_features_static", "mqg_exp_tickets", "mqg_gather_features_cached", "mqg_gather_features_missed",
    "mqg_ctx_reserve", "mqg_ctx_reserve_layer", "mqg_rms_norm", "mqg_rms_norm_backward", "mqg_sage_mean_aggregate_q8",
    "mqg_orthogonalize", "mqg_muon_step", "mqg_layer_norm", "mqg_layer_norm_backward", "mqg_grad_norm", "mqg_adamw_step",
]

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2601_04707_amd.build` "
                      "(hipcc, gfx950).  There is no CPU fallback.")

lib = ctypes.CDLL(LIB_PATH)

_i64, _i32, _vp = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p


class CGraph(ctypes.Structure):
    _fields_ = [("num_nodes", _i64), ("num_edges", _i64), ("ptr_type", _i32), ("idx_type", _i32),
                ("row_ptr", _vp), ("col_idx", _vp)]


class CCache(ctypes.Structure):
    _fields_ = [("num_nodes", _i64), ("num_cached", _i64), ("dim", _i32), ("dtype", _i32),
                ("feats", _vp), ("feat_stride", _i64), ("cache_rows", _vp), ("cache_stride", _i64),
                ("slot_of", _vp), ("cached_ids", _vp)]


class CBlock(ctypes.Structure):
    _fields_ = [("cap_dst", _i64), ("cap_src", _i64), ("cap_nnz", _i64), ("src_ids", _vp),
                ("indptr", _vp), ("indices", _vp), ("sizes", _vp)]


class CCachePlan(ctypes.Structure):
    _fields_ = [("policy", _i32), ("num_steps", _i32), ("seed", ctypes.c_uint64), ("train_ids", _vp),
                ("num_train", _i64), ("step_fanouts", ctypes.POINTER(_i32)), ("scores_out", _vp),
                ("walk_form", _i32), ("graph_symmetric", _i32)]


class CMatrices(ctypes.Structure):
    _fields_ = [("num_mats", _i32), ("rows", _i32), ("cols", _i32), ("dtype", _i32), ("data", _vp),
                ("row_stride", _i64), ("mat_stride", _i64)]


class COrth(ctypes.Structure):
    _fields_ = [("steps", _i32), ("eps", ctypes.c_float), ("coeffs", ctypes.POINTER(ctypes.c_float))]


class CParam(ctypes.Structure):
    _fields_ = [("numel", _i64), ("weight", _vp), ("grad", _vp), ("copy", _vp), ("m", _vp), ("v", _vp), ("m_scale", _vp), ("v_scale", _vp),
                ("weight_type", _i32), ("grad_type", _i32), ("copy_type", _i32), ("state_type", _i32), ("lr_scale", ctypes.c_float),
                ("decay_scale", ctypes.c_float)]


class CAdamw(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("weight_decay", ctypes.c_double), ("step", _i64), ("step_dev", _vp), ("lr_dev", _vp), ("grad_scale_dev", _vp)]


lib.mqg_version.restype = _i32
lib.mqg_version.argtypes = []
lib.mqg_ctx_create.restype = ctypes.c_int
lib.mqg_ctx_create.argtypes = [ctypes.POINTER(_vp), ctypes.POINTER(CGraph), _i32, ctypes.POINTER(_i32), _i32]
lib.mqg_ctx_destroy.restype = ctypes.c_int
lib.mqg_ctx_destroy.argtypes = [_vp]
lib.mqg_last_error.restype = ctypes.c_char_p
lib.mqg_last_error.argtypes = [_vp]
lib.mqg_ctx_set_option.restype = ctypes.c_int
lib.mqg_ctx_set_option.argtypes = [_vp, _i32, _i64]
lib.mqg_ctx_reserve.restype = ctypes.c_int
lib.mqg_ctx_reserve.argtypes = [_vp, _i32, _i64]
MQG_RESERVE_BACKWARD, MQG_RESERVE_LAYERWISE, MQG_RESERVE_DEDUP_HASH, MQG_RESERVE_SAMPLING_PRIORITY, MQG_RESERVE_CACHE_BUILD = 1, 2, 4, 8, 16
lib.mqg_ctx_kernel_time.restype = ctypes.c_int
lib.mqg_ctx_kernel_time.argtypes = [_vp, ctypes.c_char_p, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(_i64)]
lib.mqg_ctx_reset_profile.restype = ctypes.c_int
lib.mqg_ctx_reset_profile.argtypes = [_vp]
lib.mqg_ctx_kernel_names.restype = ctypes.c_int
lib.mqg_ctx_kernel_names.argtypes = [_vp, ctypes.c_char_p, _i64]
lib.mqg_build_cache.restype = ctypes.c_int
lib.mqg_build_cache.argtypes = [_vp, ctypes.POINTER(CGraph), ctypes.POINTER(CCache), _vp]
lib.mqg_build_cache_ex.restype = ctypes.c_int
lib.mqg_build_cache_ex.argtypes = [_vp, ctypes.POINTER(CGraph), ctypes.POINTER(CCache), ctypes.POINTER(CCachePlan), _vp]
lib.mqg_sample_blocks.restype = ctypes.c_int
lib.mqg_sample_blocks.argtypes = [_vp, ctypes.POINTER(CGraph), _vp, _i32, ctypes.POINTER(_i32), _i32,
                                  ctypes.c_uint64, ctypes.POINTER(CBlock), _vp]
lib.mqg_gather_features.restype = ctypes.c_int
lib.mqg_gather_features.argtypes = [_vp, ctypes.POINTER(CCache), _i32, _vp, _vp, _i64, _vp, _i64, _vp, _vp]
for _name in ("mqg_gather_features_cached", "mqg_gather_features_missed"):
    getattr(lib, _name).restype = ctypes.c_int
    getattr(lib, _name).argtypes = [_vp, ctypes.POINTER(CCache), _i32, _vp, _vp, _i64, _vp, _i64, _vp, _vp]
lib.mqg_gather_features_static.restype = ctypes.c_int
lib.mqg_gather_features_static.argtypes = [ctypes.POINTER(CCache), _i32, _vp, _vp, _i64, _vp, _i64, _vp, _vp]
MQG_GATHER_STATIC_MAX_IDS = 1 << 20
lib.mqg_sage_mean_aggregate.restype = ctypes.c_int
lib.mqg_sage_mean_aggregate.argtypes = [_vp, ctypes.POINTER(CBlock), _vp, _i64, _vp, _i64, _i32, _i32, _vp]
lib.mqg_sage_mean_aggregate_backward.restype = ctypes.c_int
lib.mqg_sage_mean_aggregate_backward.argtypes = [_vp, ctypes.POINTER(CBlock), _vp, _i64, _vp, _i64, _i32, _i32, _vp]
lib.mqg_queue_size.restype = ctypes.c_int
lib.mqg_gcn_edge_weights.restype = ctypes.c_int
lib.mqg_gcn_edge_weights.argtypes = [_vp, ctypes.POINTER(CGraph), ctypes.POINTER(CBlock), _vp, _vp, _vp]
lib.mqg_weighted_aggregate.restype = ctypes.c_int
lib.mqg_weighted_aggregate.argtypes = [_vp, ctypes.POINTER(CBlock), _vp, _vp, _vp, _i64, _vp, _i64, _i32, _i32, _vp]
lib.mqg_weighted_aggregate_backward.restype = ctypes.c_int
lib.mqg_weighted_aggregate_backward.argtypes = [_vp, ctypes.POINTER(CBlock), _vp, _vp, _vp, _i64, _vp, _i64, _i32, _i32, _vp]
lib.mqg_ctx_set_sampling_priority.restype = ctypes.c_int
lib.mqg_ctx_set_sampling_priority.argtypes = [_vp, ctypes.POINTER(CGraph), ctypes.POINTER(CCache), _vp]
lib.mqg_sample_layerwise.restype = ctypes.c_int
lib.mqg_sample_layerwise.argtypes = [_vp, ctypes.POINTER(CGraph), _vp, _i32, ctypes.POINTER(_i32), _i32, ctypes.c_uint64,
                                     _i32, _i32, ctypes.POINTER(CBlock), ctypes.POINTER(_vp), _vp]
MQG_LAYERWISE_LADIES, MQG_LAYERWISE_FASTGCN, MQG_LAYERWISE_DEBIAS, MQG_LAYERWISE_FLAT = 0, 1, 2, 4
lib.mqg_select_smallest_keys.restype = ctypes.c_int
lib.mqg_select_smallest_keys.argtypes = [_vp, _vp, _i64, _i64, _vp, _vp]
lib.mqg_select_row_candidates.restype = ctypes.c_int
lib.mqg_select_row_candidates.argtypes = [_vp, _vp, _vp, _i32, _i32, _i32, _i32, _vp, _vp]
lib.mqg_exp_tickets.restype = ctypes.c_int
lib.mqg_exp_tickets.argtypes = [_vp, ctypes.c_uint64, _i64, _i64, _i64, _vp, _vp]
lib.mqg_sample_blocks_seed_dev.restype = ctypes.c_int
lib.mqg_sample_blocks_seed_dev.argtypes = [_vp, ctypes.POINTER(CGraph), _vp, _i32, ctypes.POINTER(_i32), _i32, _vp,
                                           ctypes.POINTER(CBlock), _vp]
lib.mqg_queue_size.argtypes = [ctypes.c_double, ctypes.c_double, _i64, _i64, _i32, _i64, ctypes.POINTER(_i64),
                               ctypes.POINTER(_i64)]


_f32 = ctypes.c_float
lib.mqg_ctx_reserve_layer.restype = ctypes.c_int
lib.mqg_ctx_reserve_layer.argtypes = [_vp, _i32, _i32, _i32, _i32]
lib.mqg_rms_norm.restype = ctypes.c_int
lib.mqg_rms_norm.argtypes = [_vp, _vp, _i64, _vp, _i64, _vp, _f32, _vp, _i64, _i32, _i32, _vp, _i64, _vp, _i64, _vp, _i64, _i32, _i32, _vp,
                             _i64, _vp]
lib.mqg_rms_norm_backward.restype = ctypes.c_int
lib.mqg_rms_norm_backward.argtypes = [_vp, _vp, _i64, _vp, _i64, _vp, _vp, _i64, _f32, _vp, _i64, _i32, _i32, _vp, _i64, _vp, _vp]
lib.mqg_layer_norm.restype = ctypes.c_int
lib.mqg_layer_norm.argtypes = [_vp, _vp, _i64, _vp, _i64, _vp, _vp, _f32, _vp, _i64, _i32, _i32, _vp, _i64, _vp, _i64, _vp, _i64, _i32, _i32, _vp,
                               _i64, _vp]
lib.mqg_layer_norm_backward.restype = ctypes.c_int
lib.mqg_layer_norm_backward.argtypes = [_vp, _vp, _i64, _vp, _i64, _vp, _vp, _i64, _f32, _vp, _i64, _i32, _i32, _vp, _i64, _vp, _vp, _vp]
lib.mqg_grad_norm.restype = ctypes.c_int
lib.mqg_grad_norm.argtypes = [_vp, ctypes.POINTER(CParam), _i32, _f32, _f32, _vp, _vp, _vp]
lib.mqg_adamw_step.restype = ctypes.c_int
lib.mqg_adamw_step.argtypes = [_vp, ctypes.POINTER(CParam), _i32, ctypes.POINTER(CAdamw), _vp]
lib.mqg_sage_mean_aggregate_q8.restype = ctypes.c_int
lib.mqg_sage_mean_aggregate_q8.argtypes = [_vp, ctypes.POINTER(CBlock), _vp, _i64, _i32, _i32, _vp, _i64, _vp, _i64, _i32, _i32, _vp]
lib.mqg_orthogonalize.restype = ctypes.c_int
lib.mqg_orthogonalize.argtypes = [_vp, ctypes.POINTER(CMatrices), ctypes.POINTER(CMatrices), ctypes.POINTER(COrth), _vp]
lib.mqg_muon_step.restype = ctypes.c_int
lib.mqg_muon_step.argtypes = [_vp, ctypes.POINTER(CMatrices), ctypes.POINTER(CMatrices), ctypes.POINTER(CMatrices), _f32, _f32, _i32, _f32, _f32,
                              ctypes.POINTER(COrth), _vp]


class MqgError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"mqg error {code}: {msg}")
        self.code = code


def _itype(t: torch.Tensor) -> int:
    if t.dtype == torch.int32:
        return MQG_I32
    if t.dtype == torch.int64:
        return MQG_I64
    raise TypeError(f"index tensors must be int32 or int64, got {t.dtype}")


def _dtype(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return MQG_F32
    if t.dtype == torch.float16:
        return MQG_F16
    raise TypeError(f"features must be float32 or float16, got {t.dtype}")


_LAYER_DTYPES = {torch.float32: MQG_F32, torch.float16: MQG_F16, torch.bfloat16: MQG_BF16}
_Q_TYPES = {torch.float8_e4m3fn: MQG_Q_E4M3, torch.int8: MQG_Q_INT8}


def _layer_dtype(t: torch.Tensor) -> int:
    try:
        return _LAYER_DTYPES[t.dtype]
    except KeyError:
        raise TypeError(f"rows and matrices of a layer must be float32, float16 or bfloat16, got {t.dtype}") from None


def _q_type(t: torch.Tensor) -> int:
    try:
        return _Q_TYPES[t.dtype]
    except KeyError:
        raise TypeError(f"8-bit rows must be float8_e4m3fn or int8, got {t.dtype}") from None


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


# The current stream's handle alone: 0.4 us of host time; the Stream object around it takes 2.9 us, and small calls are
# bound by the host.  The function is not part of torch's public interface: without it the object will do.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> Optional[int]:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream if _raw_stream is None else _raw_stream(torch.cuda.current_device())
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


class Graph:
    """CSR graph resident on the GPU (the tensors are kept alive here)."""

    def __init__(self, row_ptr: torch.Tensor, col_idx: torch.Tensor):
        assert row_ptr.is_cuda and col_idx.is_cuda and row_ptr.is_contiguous() and col_idx.is_contiguous()
        self.row_ptr, self.col_idx = row_ptr, col_idx
        self.num_nodes = row_ptr.numel() - 1
        self.c = CGraph(self.num_nodes, col_idx.numel(), _itype(row_ptr), _itype(col_idx),
                        row_ptr.data_ptr(), col_idx.data_ptr())

    @property
    def idx_dtype(self):
        return self.col_idx.dtype


class Context:
    def __init__(self, graph: Graph, max_seeds: int, max_fanouts: Sequence[int]):
        self.graph = graph
        self.max_fanouts = list(max_fanouts)
        self.max_seeds = int(max_seeds)
        h = _vp()
        arr = (_i32 * len(max_fanouts))(*max_fanouts)
        rc = lib.mqg_ctx_create(ctypes.byref(h), ctypes.byref(graph.c), max_seeds, arr, len(max_fanouts))
        if rc != MQG_OK:
            raise MqgError(rc, lib.mqg_last_error(None).decode())
        self.h = h

    def check(self, rc: int):
        if rc != MQG_OK:
            raise MqgError(rc, lib.mqg_last_error(self.h).decode())

    def set_option(self, option: int, value: int):
        self.check(lib.mqg_ctx_set_option(self.h, option, value))

    def reserve(self, what: int, layerwise_rows: int = 0):
        """Allocate optional-path scratch now (a sum of MQG_RESERVE_*)."""
        self.check(lib.mqg_ctx_reserve(self.h, what, layerwise_rows))

    def reserve_layer(self, norm_dim: int = 0, num_mats: int = 0, rows: int = 0, cols: int = 0):
        """Allocate now the scratch of a layer's calls: mqg_rms_norm_backward and mqg_layer_norm_backward for rows of up to norm_dim columns,
        mqg_orthogonalize and mqg_muon_step for stacks of num_mats matrices of rows x cols."""
        self.check(lib.mqg_ctx_reserve_layer(self.h, norm_dim, num_mats, rows, cols))

    def set_sampling_priority(self, cache, stream=None):
        """Draw cached neighbours first (cache: a Cache, or None for the uniform draw)."""
        self.check(lib.mqg_ctx_set_sampling_priority(self.h, ctypes.byref(self.graph.c),
                                                     ctypes.byref(cache.c) if cache is not None else None,
                                                     _stream(stream)))

    def kernel_time(self, name: str):
        ms, n = ctypes.c_double(0), _i64(0)
        self.check(lib.mqg_ctx_kernel_time(self.h, name.encode(), ctypes.byref(ms), ctypes.byref(n)))
        return ms.value, n.value

    def kernel_names(self) -> List[str]:
        buf = ctypes.create_string_buffer(8192)
        self.check(lib.mqg_ctx_kernel_names(self.h, buf, 8192))
        return [s for s in buf.value.decode().split("\n") if s]

    def reset_profile(self):
        self.check(lib.mqg_ctx_reset_profile(self.h))

    def close(self):
        if getattr(self, "h", None):
            lib.mqg_ctx_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def block_bounds(num_nodes: int, num_seeds: int, fanouts: Sequence[int]):
    """Worst-case (cap_dst, cap_src, cap_nnz) per block, the bounds the library checks."""
    L = len(fanouts)
    out = [None] * L
    dst = num_seeds
    for l in range(L - 1, -1, -1):
        nnz = dst * fanouts[l]
        src = max(dst, min(num_nodes, dst + nnz))
        out[l] = (dst, src, nnz)
        dst = src
    return out


class Blocks:
    """Device buffers of the L blocks of one mini-batch, sized by the worst-case bounds."""

    def __init__(self, graph: Graph, max_seeds: int, fanouts: Sequence[int], device=None):
        device = device or graph.col_idx.device
        self.fanouts = list(fanouts)
        self.L = len(fanouts)
        self.bounds = block_bounds(graph.num_nodes, max_seeds, fanouts)
        self.src_ids, self.indptr, self.indices = [], [], []
        self.sizes = torch.zeros((self.L, 4), dtype=torch.int64, device=device)
        self.c = (CBlock * self.L)()
        for l, (cd, cs, cn) in enumerate(self.bounds):
            self.src_ids.append(torch.empty(max(cs, 1), dtype=graph.idx_dtype, device=device))
            self.indptr.append(torch.empty(cd + 1, dtype=torch.int32, device=device))
            self.indices.append(torch.empty(max(cn, 1), dtype=torch.int32, device=device))
            self.c[l] = CBlock(cd, cs, cn, self.src_ids[l].data_ptr(), self.indptr[l].data_ptr(),
                               self.indices[l].data_ptr(), self.sizes[l].data_ptr())

    def host_sizes(self):
        """[(num_dst, num_src, nnz, flags)] - synchronises."""
        return [tuple(int(x) for x in row) for row in self.sizes.cpu().tolist()]


class BlockView:
    """One block (number 0) over tensors that the caller has: indptr and indices int32, sizes int64 [4] on the device,
    num_src the number of source rows."""

    def __init__(self, indptr: torch.Tensor, indices: torch.Tensor, sizes: torch.Tensor, num_src: int):
        assert indptr.is_cuda and indptr.dtype == torch.int32 and indptr.is_contiguous() and indptr.numel() >= 1
        assert indices.is_cuda and indices.dtype == torch.int32 and indices.is_contiguous()
        assert sizes.is_cuda and sizes.dtype == torch.int64 and sizes.is_contiguous() and sizes.numel() >= 4
        self.L = 1
        self.indptr, self.indices, self.sizes = [indptr], [indices], sizes.view(-1, 4)
        self.bounds = [(indptr.numel() - 1, int(num_src), indices.numel())]
        self.c = (CBlock * 1)(CBlock(indptr.numel() - 1, int(num_src), indices.numel(), None, indptr.data_ptr(), indices.data_ptr(),
                                     sizes.data_ptr()))


class LayerwiseBlocks(Blocks):
    """Buffers of the L weighted blocks of one layer-wise mini-batch: rows of block L-1 = the seeds,
    sources of block l = the layer_sizes[l] drawn nodes = the rows of block l-1."""

    def __init__(self, graph: Graph, max_seeds: int, layer_sizes: Sequence[int], nnz_per_row: Optional[int] = None,
                 device=None):
        device = device or graph.col_idx.device
        self.layer_sizes = list(layer_sizes)
        self.L = len(layer_sizes)
        n = graph.num_nodes
        self.bounds = []
        rows = max_seeds
        for l in range(self.L - 1, -1, -1):
            src = min(n, layer_sizes[l])
            per_row = src if nnz_per_row is None else min(src, nnz_per_row)
            self.bounds.insert(0, (rows, src, max(1, rows * per_row)))
            rows = src
        self.src_ids, self.indptr, self.indices, self.edge_w = [], [], [], []
        self.sizes = torch.zeros((self.L, 4), dtype=torch.int64, device=device)
        self.c = (CBlock * self.L)()
        for l, (cd, cs, cn) in enumerate(self.bounds):
            self.src_ids.append(torch.empty(max(cs, 1), dtype=graph.idx_dtype, device=device))
            self.indptr.append(torch.empty(cd + 1, dtype=torch.int32, device=device))
            self.indices.append(torch.empty(cn, dtype=torch.int32, device=device))
            self.edge_w.append(torch.empty(cn, dtype=torch.float32, device=device))
            self.c[l] = CBlock(cd, cs, cn, self.src_ids[l].data_ptr(), self.indptr[l].data_ptr(),
                               self.indices[l].data_ptr(), self.sizes[l].data_ptr())
        self.edge_w_ptrs = (_vp * self.L)(*[t.data_ptr() for t in self.edge_w])


class Cache:
    """Feature storage plus the HBM cache of hot rows.  `feats` may be a pinned host tensor
    or a device tensor; with num_cached=None there is no cache and feats is read directly."""

    def __init__(self, graph: Graph, feats: torch.Tensor, num_cached: Optional[int], cache_stride: Optional[int] = None):
        assert feats.dim() == 2 and feats.stride(1) == 1
        assert feats.is_cuda or feats.is_pinned(), "feats must be device or pinned host memory"
        self.feats = feats
        self.dim = feats.shape[1]
        dev = graph.col_idx.device
        self.num_cached = num_cached
        if num_cached is None:
            self.cache_rows = self.slot_of = self.cached_ids = None
            self.cache_stride = 0
            nc = 0
        else:
            nc = int(num_cached)
            self.cache_stride = int(cache_stride or self.dim)
            self.cache_rows = torch.zeros((max(nc, 1), self.cache_stride), dtype=feats.dtype, device=dev)
            self.slot_of = torch.empty(max(graph.num_nodes, 1), dtype=torch.int32, device=dev)
            self.cached_ids = torch.empty(max(nc, 1), dtype=graph.idx_dtype, device=dev)
        self.c = CCache(graph.num_nodes, nc, self.dim, _dtype(feats), feats.data_ptr(), feats.stride(0),
                        _ptr(self.cache_rows), self.cache_stride, _ptr(self.slot_of), _ptr(self.cached_ids))


# ---------------------------------------------------------------------------------- the four calls

def mqg_build_cache(ctx: Context, graph: Graph, cache: Cache, stream=None) -> None:
    ctx.check(lib.mqg_build_cache(ctx.h, ctypes.byref(graph.c), ctypes.byref(cache.c), _stream(stream)))


def mqg_build_cache_ex(ctx: Context, graph: Graph, cache: Cache, policy: int, *, seed: int = 0,
                       train_ids: Optional[torch.Tensor] = None, step_fanouts: Sequence[int] = (),
                       scores_out: Optional[torch.Tensor] = None, walk_form: int = MQG_WALK_PUSH,
                       graph_symmetric: bool = False, stream=None) -> None:
    """Cache filled by one of the policies MQG_CACHE_*."""
    fo = (_i32 * max(1, len(step_fanouts)))(*step_fanouts)
    if train_ids is not None:
        assert train_ids.is_cuda and train_ids.dtype == graph.idx_dtype and train_ids.is_contiguous()
    if scores_out is not None:
        assert scores_out.is_cuda and scores_out.dtype == torch.float64 and scores_out.numel() >= graph.num_nodes
    plan = CCachePlan(policy, len(step_fanouts), seed & 0xFFFFFFFFFFFFFFFF, _ptr(train_ids),
                      0 if train_ids is None else train_ids.numel(), fo, _ptr(scores_out), walk_form,
                      1 if graph_symmetric else 0)
    ctx.check(lib.mqg_build_cache_ex(ctx.h, ctypes.byref(graph.c), ctypes.byref(cache.c), ctypes.byref(plan),
                                     _stream(stream)))


def mqg_sample_blocks(ctx: Context, graph: Graph, seeds: torch.Tensor, fanouts: Sequence[int], rng_seed: int,
                      blocks: Blocks, stream=None) -> None:
    assert seeds.is_cuda and seeds.dtype == graph.idx_dtype and seeds.is_contiguous()
    arr = (_i32 * len(fanouts))(*fanouts)
    ctx.check(lib.mqg_sample_blocks(ctx.h, ctypes.byref(graph.c), seeds.data_ptr(), seeds.numel(), arr,
                                    len(fanouts), ctypes.c_uint64(rng_seed & 0xFFFFFFFFFFFFFFFF), blocks.c,
                                    _stream(stream)))


def mqg_sample_blocks_seed_dev(ctx: Context, graph: Graph, seeds: torch.Tensor, fanouts: Sequence[int],
                               rng_seed_dev: torch.Tensor, blocks: Blocks, stream=None) -> None:
    """As mqg_sample_blocks, the seed read from a one-element device int64 tensor at run time."""
    assert seeds.is_cuda and seeds.dtype == graph.idx_dtype and seeds.is_contiguous()
    assert rng_seed_dev.is_cuda and rng_seed_dev.dtype == torch.int64 and rng_seed_dev.numel() >= 1
    arr = (_i32 * len(fanouts))(*fanouts)
    ctx.check(lib.mqg_sample_blocks_seed_dev(ctx.h, ctypes.byref(graph.c), seeds.data_ptr(), seeds.numel(), arr,
                                             len(fanouts), rng_seed_dev.data_ptr(), blocks.c, _stream(stream)))


def mqg_sample_layerwise(ctx: Context, graph: Graph, seeds: torch.Tensor, layer_sizes: Sequence[int], rng_seed: int,
                         blocks: "LayerwiseBlocks", normalise: bool = True, method: int = 0, stream=None) -> None:
    assert seeds.is_cuda and seeds.dtype == graph.idx_dtype and seeds.is_contiguous()
    arr = (_i32 * len(layer_sizes))(*layer_sizes)
    ctx.check(lib.mqg_sample_layerwise(ctx.h, ctypes.byref(graph.c), seeds.data_ptr() if seeds.numel() else None,
                                       seeds.numel(), arr, len(layer_sizes), rng_seed & 0xFFFFFFFFFFFFFFFF,
                                       1 if normalise else 0, method, blocks.c, blocks.edge_w_ptrs, _stream(stream)))


def mqg_select_smallest_keys(ctx: Context, keys: torch.Tensor, k: int, stream=None) -> torch.Tensor:
    """keys: device int64 tensor holding unsigned 64-bit patterns.  Returns a bool tensor: selected."""
    assert keys.is_cuda and keys.dtype == torch.int64 and keys.is_contiguous()
    n = keys.numel()
    words = torch.empty(max(1, (n + 31) // 32), dtype=torch.int32, device=keys.device)
    ctx.check(lib.mqg_select_smallest_keys(ctx.h, keys.data_ptr() if n else None, n, k, words.data_ptr(), _stream(stream)))
    bits = (words.view(-1, 1) >> torch.arange(32, device=keys.device, dtype=torch.int32)) & 1
    return bits.reshape(-1)[:n].bool()


def mqg_select_row_candidates(ctx: Context, keys: torch.Tensor, slot_words: torch.Tensor, k: int, prioritised: bool = False,
                              ordered: bool = True, stream=None) -> torch.Tensor:
    """keys: device int64 (unsigned 64-bit patterns); slot_words: device int32 (bit 31 = comes after
    every unmarked candidate when prioritised).  Returns a bool tensor: candidate chosen."""
    assert keys.is_cuda and keys.dtype == torch.int64 and keys.is_contiguous()
    assert slot_words.is_cuda and slot_words.dtype == torch.int32 and slot_words.numel() == keys.numel()
    n = keys.numel()
    words = torch.zeros(8, dtype=torch.int32, device=keys.device)
    ctx.check(lib.mqg_select_row_candidates(ctx.h, keys.data_ptr(), slot_words.data_ptr(), n, k, int(prioritised), int(ordered),
                                            words.data_ptr(), _stream(stream)))
    bits = (words.view(-1, 1) >> torch.arange(32, device=keys.device, dtype=torch.int32)) & 1
    return bits.reshape(-1)[:n].bool()


def mqg_exp_tickets(ctx: Context, seed: int, tag: int, first: int, n: int, stream=None) -> torch.Tensor:
    """The race tickets of nodes first .. first + n - 1 in key domain `tag`, as int64 bit patterns."""
    out = torch.empty(max(1, n), dtype=torch.int64, device="cuda")
    ctx.check(lib.mqg_exp_tickets(ctx.h, ctypes.c_uint64(seed & 0xFFFFFFFFFFFFFFFF), tag, first, n, out.data_ptr(),
                                  _stream(stream)))
    return out[:n]


def mqg_gather_features(ctx: Context, cache: Cache, ids: torch.Tensor, num_ids: torch.Tensor, out: torch.Tensor,
                        stats: Optional[torch.Tensor] = None, cap_ids: Optional[int] = None, stream=None) -> None:
    """ids: device id tensor; num_ids: device int64 scalar tensor (e.g. blocks.sizes[0, 1:2])."""
    assert ids.is_cuda and num_ids.is_cuda and num_ids.dtype == torch.int64 and out.is_cuda
    assert out.dtype == cache.feats.dtype and out.stride(1) == 1
    cap = int(cap_ids if cap_ids is not None else min(ids.numel(), out.shape[0]))
    assert cap <= ids.numel() and cap <= out.shape[0]
    ctx.check(lib.mqg_gather_features(ctx.h, ctypes.byref(cache.c), _itype(ids), ids.data_ptr(), num_ids.data_ptr(),
                                      cap, out.data_ptr(), out.stride(0), _ptr(stats), _stream(stream)))


def _gather_half(fn, ctx, cache, ids, num_ids, out, stats, cap_ids, stream):
    assert ids.is_cuda and num_ids.is_cuda and num_ids.dtype == torch.int64 and out.is_cuda
    assert out.dtype == cache.feats.dtype and out.stride(1) == 1
    cap = int(cap_ids if cap_ids is not None else min(ids.numel(), out.shape[0]))
    assert cap <= ids.numel() and cap <= out.shape[0]
    ctx.check(fn(ctx.h, ctypes.byref(cache.c), _itype(ids), ids.data_ptr(), num_ids.data_ptr(), cap, out.data_ptr(),
                 out.stride(0), _ptr(stats), _stream(stream)))


def mqg_gather_features_cached(ctx: Context, cache: Cache, ids: torch.Tensor, num_ids: torch.Tensor, out: torch.Tensor,
                               stats: Optional[torch.Tensor] = None, cap_ids: Optional[int] = None, stream=None) -> None:
    """First half of mqg_gather_features: classify the ids, copy the cached rows."""
    _gather_half(lib.mqg_gather_features_cached, ctx, cache, ids, num_ids, out, stats, cap_ids, stream)


def mqg_gather_features_missed(ctx: Context, cache: Cache, ids: torch.Tensor, num_ids: torch.Tensor, out: torch.Tensor,
                               stats: Optional[torch.Tensor] = None, cap_ids: Optional[int] = None, stream=None) -> None:
    """Second half: copy the rows the first half did not find in the cache."""
    _gather_half(lib.mqg_gather_features_missed, ctx, cache, ids, num_ids, out, stats, cap_ids, stream)


def mqg_gather_features_static(cache: Cache, ids: torch.Tensor, num_ids: torch.Tensor, out: torch.Tensor,
                               stats: Optional[torch.Tensor] = None, cap_ids: Optional[int] = None, stream=None) -> None:
    """mqg_gather_features without a context: the library's fixed device array holds the lists."""
    assert ids.is_cuda and num_ids.is_cuda and num_ids.dtype == torch.int64 and out.is_cuda
    assert out.dtype == cache.feats.dtype and out.stride(1) == 1
    cap = int(cap_ids if cap_ids is not None else min(ids.numel(), out.shape[0]))
    assert cap <= ids.numel() and cap <= out.shape[0]
    rc = lib.mqg_gather_features_static(ctypes.byref(cache.c), _itype(ids), ids.data_ptr(), num_ids.data_ptr(), cap,
                                        out.data_ptr(), out.stride(0), _ptr(stats), _stream(stream))
    if rc != MQG_OK:
        raise MqgError(rc, lib.mqg_last_error(None).decode())


def mqg_sage_mean_aggregate(ctx: Context, blocks: Blocks, l: int, x_src: torch.Tensor, out: torch.Tensor,
                            stream=None) -> None:
    assert x_src.is_cuda and out.is_cuda and x_src.dtype == out.dtype
    assert x_src.stride(1) == 1 and out.stride(1) == 1 and x_src.shape[1] == out.shape[1]
    assert out.shape[0] >= blocks.c[l].cap_dst
    ctx.check(lib.mqg_sage_mean_aggregate(ctx.h, ctypes.byref(blocks.c[l]), x_src.data_ptr(), x_src.stride(0),
                                          out.data_ptr(), out.stride(0), x_src.shape[1], _dtype(x_src),
                                          _stream(stream)))


def mqg_sage_mean_aggregate_backward(ctx: Context, blocks: Blocks, l: int, grad_out: torch.Tensor, grad_x: torch.Tensor,
                                     stream=None) -> None:
    """grad_out: [>= num_dst, dim] gradient of the block's output; grad_x: [>= cap_src, dim] receives the
    gradient with respect to the block's source rows."""
    assert grad_out.is_cuda and grad_x.is_cuda and grad_out.dtype == grad_x.dtype
    assert grad_out.stride(1) == 1 and grad_x.stride(1) == 1 and grad_out.shape[1] == grad_x.shape[1]
    assert grad_x.shape[0] >= blocks.c[l].cap_src
    ctx.check(lib.mqg_sage_mean_aggregate_backward(ctx.h, ctypes.byref(blocks.c[l]), grad_out.data_ptr(),
                                                   grad_out.stride(0), grad_x.data_ptr(), grad_x.stride(0),
                                                   grad_x.shape[1], _dtype(grad_x), _stream(stream)))


def mqg_gcn_edge_weights(ctx: Context, graph: Graph, blocks: Blocks, l: int, edge_w: torch.Tensor, self_w: torch.Tensor,
                         stream=None) -> None:
    """edge_w: [>= cap_nnz] float32, self_w: [>= cap_dst] float32 (device)."""
    for t, cap in ((edge_w, blocks.c[l].cap_nnz), (self_w, blocks.c[l].cap_dst)):
        assert t.is_cuda and t.dtype == torch.float32 and t.is_contiguous() and t.numel() >= cap
    ctx.check(lib.mqg_gcn_edge_weights(ctx.h, ctypes.byref(graph.c), ctypes.byref(blocks.c[l]), edge_w.data_ptr(),
                                       self_w.data_ptr(), _stream(stream)))


def _weights(edge_w, self_w):
    assert edge_w.is_cuda and edge_w.dtype == torch.float32 and edge_w.is_contiguous()
    if self_w is not None:
        assert self_w.is_cuda and self_w.dtype == torch.float32 and self_w.is_contiguous()
    return edge_w.data_ptr(), (self_w.data_ptr() if self_w is not None else None)


def mqg_weighted_aggregate(ctx: Context, blocks: Blocks, l: int, edge_w: torch.Tensor, self_w: Optional[torch.Tensor],
                           x: torch.Tensor, out: torch.Tensor, stream=None) -> None:
    assert x.is_cuda and out.is_cuda and x.dtype == out.dtype and x.stride(1) == 1 and out.stride(1) == 1
    assert x.shape[1] == out.shape[1] and out.shape[0] >= blocks.c[l].cap_dst
    assert edge_w.numel() >= blocks.c[l].cap_nnz and (self_w is None or self_w.numel() >= blocks.c[l].cap_dst)
    ew, sw = _weights(edge_w, self_w)
    ctx.check(lib.mqg_weighted_aggregate(ctx.h, ctypes.byref(blocks.c[l]), ew, sw, x.data_ptr(), x.stride(0),
                                         out.data_ptr(), out.stride(0), x.shape[1], _dtype(x), _stream(stream)))


def mqg_weighted_aggregate_backward(ctx: Context, blocks: Blocks, l: int, edge_w: torch.Tensor,
                                    self_w: Optional[torch.Tensor], grad_out: torch.Tensor, grad_x: torch.Tensor,
                                    stream=None) -> None:
    assert grad_out.is_cuda and grad_x.is_cuda and grad_out.dtype == grad_x.dtype
    assert grad_out.stride(1) == 1 and grad_x.stride(1) == 1 and grad_out.shape[1] == grad_x.shape[1]
    assert grad_x.shape[0] >= blocks.c[l].cap_src
    assert edge_w.numel() >= blocks.c[l].cap_nnz and (self_w is None or self_w.numel() >= blocks.c[l].cap_dst)
    ew, sw = _weights(edge_w, self_w)
    ctx.check(lib.mqg_weighted_aggregate_backward(ctx.h, ctypes.byref(blocks.c[l]), ew, sw, grad_out.data_ptr(),
                                                  grad_out.stride(0), grad_x.data_ptr(), grad_x.stride(0),
                                                  grad_x.shape[1], _dtype(grad_x), _stream(stream)))


# ---------------------------------------------------------------------------------- the calls of a layer

def _rows(t: torch.Tensor, dtype, shape) -> int:
    """The row stride of a [rows, dim] tensor, checked."""
    assert t.is_cuda and t.dtype is dtype and t.shape == shape, f"expected {tuple(shape)} of {dtype} on the GPU, got {tuple(t.shape)} of {t.dtype}"
    row, col = t.stride()
    assert col == 1 or shape[1] == 1
    return row if shape[0] > 1 else max(row, shape[1])


def _norm_inputs(weight, num_rows, dim):
    if weight is not None:
        assert weight.is_cuda and weight.dtype == torch.float32 and weight.is_contiguous() and weight.numel() == dim
    if num_rows is not None:
        assert num_rows.is_cuda and num_rows.dtype == torch.int64 and num_rows.numel() >= 1


def _scales(q, q_scale, group, shape):
    assert q_scale is not None and q_scale.is_cuda and q_scale.dtype == torch.float32 and q_scale.dim() == 2
    assert q_scale.shape[0] >= shape[0] and (q_scale.shape[1] <= 1 or q_scale.stride(1) == 1)
    per_row = -(-shape[1] // group) if group else 1
    assert q_scale.shape[1] >= per_row, f"{per_row} scales per row are wanted, got {q_scale.shape[1]}"
    return q_scale.stride(0) if q_scale.shape[0] > 1 else max(q_scale.stride(0), per_row)


def mqg_rms_norm(ctx: Context, x: torch.Tensor, weight: Optional[torch.Tensor] = None, *, residual: Optional[torch.Tensor] = None,
                 sum_out: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None,
                 q_scale: Optional[torch.Tensor] = None, group: int = 0, eps: float = 1e-6, num_rows: Optional[torch.Tensor] = None,
                 stream=None) -> None:
    """y = (x + residual) / rms * weight, row by row; q and q_scale receive it in 8 bits (float8_e4m3fn or int8), one scale
    per row or per `group` columns; sum_out receives x + residual.  num_rows: device int64, rows past it are left alone."""
    shape, dtype = x.shape, x.dtype
    assert x.dim() == 2
    xs = _rows(x, dtype, shape)
    rs = _rows(residual, dtype, shape) if residual is not None else 0
    ss = _rows(sum_out, dtype, shape) if sum_out is not None else 0
    ys = _rows(y, dtype, shape) if y is not None else 0
    _norm_inputs(weight, num_rows, shape[1])
    qs = qt = cs = 0
    if q is not None:
        qt, qs, cs = _q_type(q), _rows(q, q.dtype, shape), _scales(q, q_scale, group, shape)
    ctx.check(lib.mqg_rms_norm(ctx.h, x.data_ptr(), xs, _ptr(residual), rs, _ptr(weight), eps, _ptr(num_rows), shape[0], shape[1],
                               _layer_dtype(x), _ptr(sum_out), ss, _ptr(y), ys, _ptr(q), qs, qt, group, _ptr(q_scale) if q is not None else None, cs,
                               _stream(stream)))


def mqg_rms_norm_backward(ctx: Context, grad_y: torch.Tensor, s: torch.Tensor, weight: Optional[torch.Tensor], grad_x: torch.Tensor, *,
                          grad_weight: Optional[torch.Tensor] = None, grad_sum: Optional[torch.Tensor] = None, eps: float = 1e-6,
                          num_rows: Optional[torch.Tensor] = None, stream=None) -> None:
    """Gradient of mqg_rms_norm at the stored sum s (x where there was no residual): grad_x, the same for x and residual, and
    grad_weight ([dim] float32, written).  grad_sum: the gradient that reaches s by its other uses."""
    shape, dtype = s.shape, s.dtype
    assert s.dim() == 2
    ss, gys, gxs = _rows(s, dtype, shape), _rows(grad_y, dtype, shape), _rows(grad_x, dtype, shape)
    gss = _rows(grad_sum, dtype, shape) if grad_sum is not None else 0
    _norm_inputs(weight, num_rows, shape[1])
    if grad_weight is not None:
        assert grad_weight.is_cuda and grad_weight.dtype == torch.float32 and grad_weight.is_contiguous() and grad_weight.numel() == shape[1]
    ctx.check(lib.mqg_rms_norm_backward(ctx.h, grad_y.data_ptr(), gys, s.data_ptr(), ss, _ptr(weight), _ptr(grad_sum), gss, eps, _ptr(num_rows),
                                        shape[0], shape[1], _layer_dtype(s), grad_x.data_ptr(), gxs, _ptr(grad_weight), _stream(stream)))


def mqg_layer_norm(ctx: Context, x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, *,
                   residual: Optional[torch.Tensor] = None, sum_out: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None,
                   q: Optional[torch.Tensor] = None, q_scale: Optional[torch.Tensor] = None, group: int = 0, eps: float = 1e-5,
                   num_rows: Optional[torch.Tensor] = None, stream=None) -> None:
    """y = (s - mean) / sqrt(variance + eps) * weight + bias of s = x + residual, row by row; the other arguments as mqg_rms_norm's."""
    shape, dtype = x.shape, x.dtype
    assert x.dim() == 2
    xs = _rows(x, dtype, shape)
    rs = _rows(residual, dtype, shape) if residual is not None else 0
    ss = _rows(sum_out, dtype, shape) if sum_out is not None else 0
    ys = _rows(y, dtype, shape) if y is not None else 0
    _norm_inputs(weight, num_rows, shape[1])
    _norm_inputs(bias, None, shape[1])
    qs = qt = cs = 0
    if q is not None:
        qt, qs, cs = _q_type(q), _rows(q, q.dtype, shape), _scales(q, q_scale, group, shape)
    ctx.check(lib.mqg_layer_norm(ctx.h, x.data_ptr(), xs, _ptr(residual), rs, _ptr(weight), _ptr(bias), eps, _ptr(num_rows), shape[0], shape[1],
                                 _layer_dtype(x), _ptr(sum_out), ss, _ptr(y), ys, _ptr(q), qs, qt, group, _ptr(q_scale) if q is not None else None, cs,
                                 _stream(stream)))


def mqg_layer_norm_backward(ctx: Context, grad_y: torch.Tensor, s: torch.Tensor, weight: Optional[torch.Tensor], grad_x: torch.Tensor, *,
                            grad_weight: Optional[torch.Tensor] = None, grad_bias: Optional[torch.Tensor] = None,
                            grad_sum: Optional[torch.Tensor] = None, eps: float = 1e-5, num_rows: Optional[torch.Tensor] = None, stream=None) -> None:
    """Gradient of mqg_layer_norm at the stored sum s (x where there was no residual): grad_x, the same for x and residual, grad_weight
    and grad_bias ([dim] float32, written).  grad_sum: the gradient that reaches s by its other uses."""
    shape, dtype = s.shape, s.dtype
    assert s.dim() == 2
    ss, gys, gxs = _rows(s, dtype, shape), _rows(grad_y, dtype, shape), _rows(grad_x, dtype, shape)
    gss = _rows(grad_sum, dtype, shape) if grad_sum is not None else 0
    _norm_inputs(weight, num_rows, shape[1])
    _norm_inputs(grad_weight, None, shape[1])
    _norm_inputs(grad_bias, None, shape[1])
    ctx.check(lib.mqg_layer_norm_backward(ctx.h, grad_y.data_ptr(), gys, s.data_ptr(), ss, _ptr(weight), _ptr(grad_sum), gss, eps, _ptr(num_rows),
                                          shape[0], shape[1], _layer_dtype(s), grad_x.data_ptr(), gxs, _ptr(grad_weight), _ptr(grad_bias),
                                          _stream(stream)))


def mqg_sage_mean_aggregate_q8(ctx: Context, blocks, l: int, q: torch.Tensor, q_scale: torch.Tensor, out: torch.Tensor, *, group: int = 0,
                               stream=None) -> None:
    """mqg_sage_mean_aggregate of source rows in 8 bits with scales, as mqg_rms_norm writes them; out: float32, float16 or bfloat16."""
    assert q.dim() == 2 and out.dim() == 2 and q.shape[0] >= blocks.bounds[l][1] and out.shape[0] >= blocks.bounds[l][0]
    assert q.shape[1] == out.shape[1]
    qs, cs, os_ = _rows(q, q.dtype, q.shape), _scales(q, q_scale, group, q.shape), _rows(out, out.dtype, out.shape)
    ctx.check(lib.mqg_sage_mean_aggregate_q8(ctx.h, ctypes.byref(blocks.c[l]), q.data_ptr(), qs, _q_type(q), group, q_scale.data_ptr(), cs,
                                             out.data_ptr(), os_, out.shape[1], _layer_dtype(out), _stream(stream)))


def _matrices(t: torch.Tensor) -> CMatrices:
    """A [rows, cols] matrix or a [mats, rows, cols] stack of them, rows contiguous."""
    assert t.is_cuda and t.dim() in (2, 3)
    m, (r, c) = (1, t.shape) if t.dim() == 2 else (t.shape[0], t.shape[1:])
    assert c <= 1 or t.stride(-1) == 1
    rs = t.stride(-2) if r > 1 else max(t.stride(-2), c)
    return CMatrices(m, r, c, _layer_dtype(t), t.data_ptr(), rs, t.stride(0) if t.dim() == 3 and m > 1 else rs * r)


def _orth(steps, coeffs, eps) -> COrth:
    """coeffs: None, one (a, b, c) for all steps, or one for each."""
    if coeffs is None:
        return COrth(steps, eps, None)
    flat = [float(v) for row in coeffs for v in row] if hasattr(coeffs[0], "__len__") else [float(v) for v in coeffs] * steps
    assert len(flat) == 3 * steps, "coeffs: (a, b, c), or one such triple for each step"
    return COrth(steps, eps, (_f32 * len(flat))(*flat))


def mqg_orthogonalize(ctx: Context, update: torch.Tensor, out: torch.Tensor, *, steps: int = 5, coeffs=None, eps: float = 1e-7,
                      stream=None) -> None:
    """out = the orthogonal factor of every matrix of `update` ([rows, cols] or [mats, rows, cols]), by Newton-Schulz steps."""
    assert update.shape == out.shape
    u, o, p = _matrices(update), _matrices(out), _orth(steps, coeffs, eps)
    ctx.check(lib.mqg_orthogonalize(ctx.h, ctypes.byref(u), ctypes.byref(o), ctypes.byref(p), _stream(stream)))


def mqg_muon_step(ctx: Context, grad: torch.Tensor, momentum: torch.Tensor, weight: torch.Tensor, *, lr: float, beta: float = 0.95,
                  nesterov: bool = True, weight_decay: float = 0.0, scale: Optional[float] = None, steps: int = 5, coeffs=None,
                  eps: float = 1e-7, stream=None) -> None:
    """momentum = beta momentum + grad; weight = (1 - lr weight_decay) weight - lr scale orthogonalize(grad + beta momentum, or momentum),
    in place (float32).  scale: sqrt(max(1, rows / cols)) if none is given."""
    assert grad.shape == momentum.shape == weight.shape
    if scale is None:
        scale = max(1.0, grad.shape[-2] / max(1, grad.shape[-1])) ** 0.5
    g, m, w, p = _matrices(grad), _matrices(momentum), _matrices(weight), _orth(steps, coeffs, eps)
    ctx.check(lib.mqg_muon_step(ctx.h, ctypes.byref(g), ctypes.byref(m), ctypes.byref(w), lr, beta, int(nesterov), weight_decay, scale,
                                ctypes.byref(p), _stream(stream)))


class Params:
    """The tensors that mqg_adamw_step steps and whose gradients mqg_grad_norm reads: made once, kept by the program.

    weights, grads: lists of contiguous tensors of the same shapes (a gradient of None: the tensor is left alone); without weights the list
    serves mqg_grad_norm only.  m, v: the moments, zeros of state_dtype if not given - float32, or float8_e4m3fn (v: its root) with
    m_scale, v_scale, a float32 per MQG_ADAMW_BLOCK elements (both zeros if not given: moments of zero, whatever m and v hold).  copies: tensors that receive the weights rounded to their type.
    lr_scale, decay_scale: a number for every tensor."""

    def __init__(self, weights=None, grads=None, *, m=None, v=None, m_scale=None, v_scale=None, copies=None, state_dtype=torch.float32,
                 lr_scale=None, decay_scale=None):
        assert weights is not None or grads is not None
        # lists of its own: the library has the addresses of these tensors, whatever the caller puts into its lists later
        weights, m, v, m_scale, v_scale, copies = (None if given is None else list(given) for given in (weights, m, v, m_scale, v_scale, copies))
        like = weights if weights is not None else grads
        n = len(like)
        eight = (m[0].dtype if m else state_dtype) == torch.float8_e4m3fn
        if weights is not None:
            assert (m is None) == (v is None)
            if m is None:
                m, v = ([torch.zeros(w.shape, dtype=state_dtype, device=w.device) for w in weights] for _ in range(2))
            if eight and m_scale is None and v_scale is None:
                m_scale, v_scale = ([torch.zeros(-(-w.numel() // MQG_ADAMW_BLOCK), device=w.device) for w in weights] for _ in range(2))
        self.weights, self.copies, self.m, self.v, self.m_scale, self.v_scale = weights, copies, m, v, m_scale, v_scale
        self.c = (CParam * n)()
        for given in (m, v, copies, lr_scale, decay_scale) + ((m_scale, v_scale) if eight else ()):
            assert given is None or len(given) == n, "one of each for every tensor"
        for i, p in enumerate(self.c):
            p.lr_scale, p.decay_scale = lr_scale[i] if lr_scale else 1.0, decay_scale[i] if decay_scale else 1.0
            if like[i] is None:
                continue
            p.numel = like[i].numel()
            if weights is None:
                continue
            p.weight, p.weight_type = self._data(weights[i], like[i].shape), _layer_dtype(weights[i])
            if copies is not None and copies[i] is not None:
                p.copy, p.copy_type = self._data(copies[i], like[i].shape), _layer_dtype(copies[i])
            state = torch.float8_e4m3fn if eight else torch.float32
            p.m, p.v, p.state_type = self._data(m[i], like[i].shape, state), self._data(v[i], like[i].shape, state), int(eight)
            if eight:
                blocks = (-(-p.numel // MQG_ADAMW_BLOCK),)
                p.m_scale, p.v_scale = self._data(m_scale[i], blocks, torch.float32), self._data(v_scale[i], blocks, torch.float32)
        self.grads = None
        if grads is not None:
            self.set_grads(grads)

    @staticmethod
    def _data(t: torch.Tensor, shape, dtype=None) -> int:
        assert t.is_cuda and t.is_contiguous() and t.shape == shape and (dtype is None or t.dtype is dtype), \
            f"expected {tuple(shape)} of {dtype or t.dtype}, contiguous on the GPU, got {tuple(t.shape)} of {t.dtype}"
        return t.data_ptr()

    def set_grads(self, grads) -> None:
        """The gradients of the steps that follow."""
        grads = list(grads)
        assert len(grads) == len(self.c)
        like = self.weights if self.weights is not None else grads
        # (looked at before anything is changed: `grads` keeps alive what the addresses are of)
        new = [None if g is None else (self._data(g, like[i].shape), _layer_dtype(g), g.numel()) for i, g in enumerate(grads)]
        for p, g in zip(self.c, new):
            if g is None:
                p.grad = None
            else:
                p.grad, p.grad_type, p.numel = g
        self.grads = grads


def _one(t, dtype) -> Optional[int]:
    if t is None:
        return None
    assert t.is_cuda and t.dtype is dtype and t.numel() >= 1
    return t.data_ptr()


def mqg_grad_norm(ctx: Context, params: Params, *, max_norm: float = float("inf"), mul: float = 1.0, norm: Optional[torch.Tensor] = None,
                  scale: Optional[torch.Tensor] = None, stream=None) -> None:
    """norm = mul * the norm of all gradients, scale = mul * min(1, max_norm / norm): float32 tensors on the GPU, either may be None."""
    ctx.check(lib.mqg_grad_norm(ctx.h, params.c, len(params.c), mul, max_norm, _one(norm, torch.float32), _one(scale, torch.float32), _stream(stream)))


def mqg_adamw_step(ctx: Context, params: Params, *, lr, step, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                   weight_decay: float = 0.01, grad_scale: Optional[torch.Tensor] = None, stream=None) -> None:
    """An AdamW step of all tensors.  lr: a number, or a float32 tensor on the GPU; step: 1, 2, ..., or an int64 tensor on the GPU, read when the step
    runs; grad_scale: a float32 tensor on the GPU that the gradients are multiplied by (mqg_grad_norm's scale)."""
    plan = CAdamw(beta1=beta1, beta2=beta2, eps=eps, weight_decay=weight_decay, grad_scale_dev=_one(grad_scale, torch.float32))
    if isinstance(lr, torch.Tensor):
        plan.lr_dev = _one(lr, torch.float32)
    else:
        plan.lr = lr
    if isinstance(step, torch.Tensor):
        plan.step_dev = _one(step, torch.int64)
    else:
        plan.step = step
    ctx.check(lib.mqg_adamw_step(ctx.h, params.c, len(params.c), ctypes.byref(plan), _stream(stream)))


def mqg_queue_size(max_prepare_ms: float, mean_compute_ms: float, total_mem_bytes: int, peak_mem_bytes: int,
                   margin_percent: int, mem_per_batch_bytes: int):
    """Returns (queue_size, cap) of the paper's queue-sizing rule; host arithmetic in the library."""
    cap, q = _i64(0), _i64(0)
    rc = lib.mqg_queue_size(max_prepare_ms, mean_compute_ms, total_mem_bytes, peak_mem_bytes, margin_percent,
                            mem_per_batch_bytes, ctypes.byref(cap), ctypes.byref(q))
    if rc != MQG_OK:
        raise MqgError(rc, lib.mqg_last_error(None).decode())
    return q.value, cap.value
