"""Thin ctypes binding of the C ABI in include/gs.h.

Argument marshalling only: every function takes torch tensors (device memory)
or numpy arrays (host memory), checks dtype/device/contiguity, passes raw
pointers and the current CUDA stream to the library, and raises GsError on a
non-zero status.  Nothing here computes anything; if the shared library has
not been built the first call raises.
"""
from __future__ import annotations

import ctypes
import functools
import struct
from dataclasses import dataclass
from pathlib import Path

import numpy as np
import torch

_LIB_PATH = Path(__file__).resolve().parent / "libgs_b200.so"
_lib = None

GS_VALIDATE, GS_REQUIRE_SORTED, GS_BUILD_WALK_INDEX, GS_BUILD_EDGE_SET = 1, 2, 4, 8
GS_DETERMINISTIC, GS_HOGWILD, GS_HOGWILD_RED = 0, 1, 2
GS_PAIRS_FORWARD_ONLY = 0x100
GS_WINDOW_SHRINK = 0x200
GS_ROUND_STOCHASTIC = 0x400
GS_WALK_UNIFORM, GS_WALK_NODE2VEC = 0, 1
GS_LR_CONSTANT, GS_LR_LINEAR = 0, 1
GS_TABLE_F32, GS_TABLE_F16, GS_TABLE_BF16 = 0, 1, 2
GS_OPT_SGD, GS_OPT_MOMENTUM, GS_OPT_ADAM = 0, 1, 2

EXPORTS = [
    "gs_last_error", "gs_graph_load_csr", "gs_graph_free", "gs_graph_info", "gs_build_alias",
    "gs_init_embeddings", "gs_random_walks", "gs_node2vec_walks", "gs_sgns_step",
    "gs_sgns_epoch", "gs_release_workspace", "gs_tune_node2vec_group", "gs_sgns_step_static", "gs_sgns_step_momentum", "gs_momentum_flush",
    "gs_init_embeddings_f16", "gs_sgns_step_f16", "gs_sgns_step_adam", "gs_build_keep_thresholds",
    "gs_subsample_walks", "gs_shuffled_starts", "gs_refused_ids",
    "gs_init_embeddings_bf16", "gs_sgns_step_bf16",
    "gs_attention_forward", "gs_attention_backward", "gs_attention_backward_work",
    "gs_stalled_kernels", "gs_stall_drill", "gs_gradient_norm_work", "gs_gradient_norm", "gs_clip_gradients",
    "gs_layer_norm_forward", "gs_layer_norm_backward", "gs_layer_norm_backward_work",
    "gs_recurrence_states", "gs_recurrence_work", "gs_recurrence_forward", "gs_recurrence_backward",
    "gs_checkpoint_pack", "gs_checkpoint_unpack",
]


class GsError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"gs status {status}: {message}")
        self.status = status


class SgnsConfig(ctypes.Structure):
    _fields_ = [
        ("dim", ctypes.c_int32), ("walks_per_node", ctypes.c_int32), ("walk_len", ctypes.c_int32),
        ("window", ctypes.c_int32), ("n_neg", ctypes.c_int32), ("walk_kind", ctypes.c_int32),
        ("lr_schedule", ctypes.c_int32), ("mode", ctypes.c_int32), ("max_rounds", ctypes.c_int32),
        ("table_dtype", ctypes.c_int32), ("p", ctypes.c_double), ("q", ctypes.c_double),
        ("lr0", ctypes.c_double), ("batch_walks", ctypes.c_int64), ("first_batch", ctypes.c_int64),
        ("num_batches", ctypes.c_int64), ("seed", ctypes.c_uint64),
        ("d_keep_thr", ctypes.c_void_p), ("shuffle_starts", ctypes.c_int32), ("epoch", ctypes.c_uint32),
        ("optimizer", ctypes.c_int32), ("momentum", ctypes.c_float), ("beta2", ctypes.c_float),
        ("eps", ctypes.c_float), ("iteration_base", ctypes.c_int64),
        ("d_m_in", ctypes.c_void_p), ("d_m_out", ctypes.c_void_p), ("d_v_in", ctypes.c_void_p),
        ("d_v_out", ctypes.c_void_p), ("d_last_in", ctypes.c_void_p), ("d_last_out", ctypes.c_void_p),
    ]


class AttentionConfig(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("q_heads", ctypes.c_int32),
        ("kv_heads", ctypes.c_int32), ("batch", ctypes.c_int64), ("q_len", ctypes.c_int32),
        ("k_len", ctypes.c_int32), ("window_left", ctypes.c_int32), ("window_right", ctypes.c_int32),
        ("scale", ctypes.c_float), ("reserved", ctypes.c_int32),
        ("d_q_lens", ctypes.c_void_p), ("d_k_lens", ctypes.c_void_p),
    ] + [(f"{t}_stride", ctypes.c_int64 * 3) for t in ("q", "k", "v", "out", "dout", "dq", "dk", "dv")]


class LayerNormConfig(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int32), ("weight_dtype", ctypes.c_int32), ("batch", ctypes.c_int64),
        ("length", ctypes.c_int64), ("columns", ctypes.c_int32), ("eps", ctypes.c_float), ("d_lens", ctypes.c_void_p),
    ] + [(f"{t}_stride", ctypes.c_int64 * 2) for t in ("x", "y", "dy", "dx")]


class RecurrenceConfig(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int32), ("length", ctypes.c_int32), ("batch", ctypes.c_int64), ("channels", ctypes.c_int64),
        ("d_lens", ctypes.c_void_p),
    ] + [(f"{t}_stride", ctypes.c_int64 * 2) for t in ("gate", "x", "out", "dout", "dgate", "dx")]


class TensorEntry(ctypes.Structure):
    _fields_ = [("d_data", ctypes.c_void_p), ("numel", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class EpochStats(ctypes.Structure):
    _fields_ = [
        ("loss_sum", ctypes.c_double), ("pairs", ctypes.c_int64), ("steps", ctypes.c_int64),
        ("cap_hits", ctypes.c_int64), ("batches", ctypes.c_int64), ("masked_negs", ctypes.c_int64),
        ("ms_walk", ctypes.c_float),
        ("ms_sgns", ctypes.c_float), ("ms_total", ctypes.c_float), ("ms_prepare", ctypes.c_float),
        ("refused_ids", ctypes.c_int64),
    ]


def library_path() -> Path:
    return _LIB_PATH


def lib():
    """Loads libgs_b200.so; fails loudly if it is missing (there is no fallback path)."""
    global _lib
    if _lib is None:
        if not _LIB_PATH.exists():
            raise FileNotFoundError(
                f"{_LIB_PATH} not built; run `python -m paper_2407_15452_b200.build`")
        L = ctypes.CDLL(str(_LIB_PATH))
        L.gs_last_error.restype = ctypes.c_char_p
        L.gs_graph_free.restype = None
        for name in EXPORTS:
            if name not in ("gs_last_error", "gs_graph_free"):
                getattr(L, name).restype = ctypes.c_int32
        p, i64 = ctypes.c_void_p, ctypes.c_int64
        L.gs_attention_forward.argtypes = [p] * 7
        L.gs_attention_backward.argtypes = [p] * 12
        L.gs_attention_backward_work.argtypes, L.gs_attention_backward_work.restype = [p], i64
        L.gs_gradient_norm_work.argtypes, L.gs_gradient_norm_work.restype = [i64], i64
        L.gs_gradient_norm.argtypes = [p, i64, p, p, p]
        L.gs_clip_gradients.argtypes = [p, p, i64, ctypes.c_float, p, p, p]
        i32 = ctypes.c_int32
        L.gs_layer_norm_forward.argtypes = [p] * 9
        L.gs_layer_norm_backward_work.argtypes, L.gs_layer_norm_backward_work.restype = [p], i64
        L.gs_layer_norm_backward.argtypes = [p] * 12
        L.gs_recurrence_states.argtypes, L.gs_recurrence_states.restype = [p], i64
        L.gs_recurrence_work.argtypes, L.gs_recurrence_work.restype = [p], i64
        L.gs_recurrence_forward.argtypes = [p] * 9
        L.gs_recurrence_backward.argtypes = [p] * 12
        L.gs_checkpoint_pack.argtypes = [i32, p, i64, i64, i64, p, p, p]
        L.gs_checkpoint_unpack.argtypes = [i32, p, p, i64, i64, i64, p, p]
        _lib = L
    return _lib


def _check(status: int):
    if status != 0:
        raise GsError(status, lib().gs_last_error().decode())


def _stream() -> ctypes.c_void_p:
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _dev(t, dtype, name, allow_none=False) -> ctypes.c_void_p:
    if t is None:
        if allow_none:
            return ctypes.c_void_p(0)
        raise TypeError(f"{name} is required")
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise TypeError(f"{name} must be a contiguous CUDA tensor of {dtype}")
    return ctypes.c_void_p(t.data_ptr())


class Graph:
    """Owns a gs_graph handle and keeps the CSR tensors alive."""

    def __init__(self, offsets: torch.Tensor, cols: torch.Tensor, flags: int = GS_VALIDATE):
        if offsets.dtype not in (torch.int32, torch.int64):
            raise TypeError("offsets must be int32 or int64")
        self.offsets, self.cols = offsets, cols
        self.n_nodes = offsets.numel() - 1
        self.n_edges = cols.numel()
        self._h = ctypes.c_void_p(0)
        _check(lib().gs_graph_load_csr(
            ctypes.c_int64(self.n_nodes), ctypes.c_int64(self.n_edges),
            _dev(offsets, offsets.dtype, "offsets"), ctypes.c_int32(offsets.dtype == torch.int64),
            _dev(cols, torch.int32, "cols", allow_none=self.n_edges == 0),
            ctypes.c_uint32(flags), _stream(), ctypes.byref(self._h)))

    def info(self):
        n, e, m, s = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int32()
        _check(lib().gs_graph_info(self._h, ctypes.byref(n), ctypes.byref(e), ctypes.byref(m),
                                   ctypes.byref(s)))
        return {"n_nodes": n.value, "n_edges": e.value, "max_degree": m.value,
                "rows_sorted": bool(s.value)}

    def close(self):
        if self._h:
            lib().gs_graph_free(self._h)
            self._h = ctypes.c_void_p(0)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def gs_graph_load_csr(offsets, cols, flags=GS_VALIDATE) -> Graph:
    return Graph(offsets, cols, flags)


def gs_build_alias(weights: np.ndarray, power: float = 0.75) -> np.ndarray:
    """Host call.  Returns the packed table (uint64: thr low, alias high)."""
    w = np.ascontiguousarray(weights, dtype=np.float64)
    out = np.empty(len(w), dtype=np.uint64)
    _check(lib().gs_build_alias(w.ctypes.data_as(ctypes.c_void_p), ctypes.c_int64(len(w)),
                                ctypes.c_double(power), out.ctypes.data_as(ctypes.c_void_p)))
    return out


def gs_init_embeddings(w_in, w_out, seed: int):
    ref = w_in if w_in is not None else w_out
    n, d = ref.shape
    _check(lib().gs_init_embeddings(_dev(w_in, torch.float32, "w_in", True),
                                    _dev(w_out, torch.float32, "w_out", True),
                                    ctypes.c_int64(n), ctypes.c_int32(d), ctypes.c_uint64(seed),
                                    _stream()))


def gs_random_walks(graph: Graph, starts, n_walks: int, walk_id_base: int, walk_len: int,
                    seed: int, out=None, steps=None):
    """Returns walks[n_walks, walk_len] (int32, CUDA).  steps: optional uint64/int64[1] counter."""
    if out is None:
        out = torch.empty((n_walks, walk_len), dtype=torch.int32, device=graph.cols.device)
    _check(lib().gs_random_walks(
        graph._h, _dev(starts, torch.int32, "starts", True), ctypes.c_int64(n_walks),
        ctypes.c_int64(walk_id_base), ctypes.c_int32(walk_len), ctypes.c_uint64(seed),
        _dev(out, torch.int32, "out"), _dev(steps, torch.int64, "steps", True), _stream()))
    return out


def gs_node2vec_walks(graph: Graph, starts, n_walks: int, walk_id_base: int, walk_len: int,
                      seed: int, p: float, q: float, max_rounds: int = 1024, out=None,
                      steps=None, cap_hits=None):
    if out is None:
        out = torch.empty((n_walks, walk_len), dtype=torch.int32, device=graph.cols.device)
    _check(lib().gs_node2vec_walks(
        graph._h, _dev(starts, torch.int32, "starts", True), ctypes.c_int64(n_walks),
        ctypes.c_int64(walk_id_base), ctypes.c_int32(walk_len), ctypes.c_uint64(seed),
        ctypes.c_double(p), ctypes.c_double(q), ctypes.c_int32(max_rounds),
        _dev(out, torch.int32, "out"), _dev(steps, torch.int64, "steps", True),
        _dev(cap_hits, torch.int64, "cap_hits", True), _stream()))
    return out


def gs_sgns_step(w_in, w_out, walks, walk_id_base: int, window: int, n_neg: int, alias,
                 lr: float, seed: int, mode: int, loss_sum=None, pair_count=None,
                 pairs_dump=None, negs_dump=None):
    """One SGNS update over walks[n_walks, walk_len]; loss_sum (float64[1]) and pair_count
    (int64[1]) are accumulated into; dumps are optional int32 tensors (see gs.h)."""
    n_nodes, dim = w_in.shape
    n_walks, walk_len = walks.shape
    _check(lib().gs_sgns_step(
        _dev(w_in, torch.float32, "w_in"), _dev(w_out, torch.float32, "w_out"),
        ctypes.c_int64(n_nodes), ctypes.c_int32(dim), _dev(walks, torch.int32, "walks", n_walks == 0),
        ctypes.c_int64(n_walks), ctypes.c_int64(walk_id_base), ctypes.c_int32(walk_len),
        ctypes.c_int32(window), ctypes.c_int32(n_neg), _dev(alias, torch.int64, "alias", n_neg == 0),
        ctypes.c_float(lr), ctypes.c_uint64(seed), ctypes.c_int32(mode),
        _dev(loss_sum, torch.float64, "loss_sum", True), _dev(pair_count, torch.int64, "pair_count", True),
        _dev(pairs_dump, torch.int32, "pairs_dump", True), _dev(negs_dump, torch.int32, "negs_dump", True),
        _stream()))


def gs_init_embeddings_f16(w_in, w_out, seed: int):
    """Start values of gs_init_embeddings rounded to half; tables are torch.float16."""
    ref = w_in if w_in is not None else w_out
    n, d = ref.shape
    _check(lib().gs_init_embeddings_f16(_dev(w_in, torch.float16, "w_in", True),
                                        _dev(w_out, torch.float16, "w_out", True),
                                        ctypes.c_int64(n), ctypes.c_int32(d), ctypes.c_uint64(seed),
                                        _stream()))


def gs_sgns_step_f16(w_in, w_out, walks, walk_id_base: int, window: int, n_neg: int, alias,
                     lr: float, seed: int, mode: int, loss_sum=None, pair_count=None,
                     pairs_dump=None, negs_dump=None):
    """gs_sgns_step on torch.float16 tables (fp32 arithmetic, round-to-nearest write-back)."""
    n_nodes, dim = w_in.shape
    n_walks, walk_len = walks.shape
    _check(lib().gs_sgns_step_f16(
        _dev(w_in, torch.float16, "w_in"), _dev(w_out, torch.float16, "w_out"),
        ctypes.c_int64(n_nodes), ctypes.c_int32(dim), _dev(walks, torch.int32, "walks", n_walks == 0),
        ctypes.c_int64(n_walks), ctypes.c_int64(walk_id_base), ctypes.c_int32(walk_len),
        ctypes.c_int32(window), ctypes.c_int32(n_neg), _dev(alias, torch.int64, "alias", n_neg == 0),
        ctypes.c_float(lr), ctypes.c_uint64(seed), ctypes.c_int32(mode),
        _dev(loss_sum, torch.float64, "loss_sum", True), _dev(pair_count, torch.int64, "pair_count", True),
        _dev(pairs_dump, torch.int32, "pairs_dump", True), _dev(negs_dump, torch.int32, "negs_dump", True),
        _stream()))


def gs_init_embeddings_bf16(w_in, w_out, seed: int):
    """Start values of gs_init_embeddings rounded to bfloat16; tables are torch.bfloat16."""
    ref = w_in if w_in is not None else w_out
    n, d = ref.shape
    _check(lib().gs_init_embeddings_bf16(_dev(w_in, torch.bfloat16, "w_in", True),
                                        _dev(w_out, torch.bfloat16, "w_out", True),
                                        ctypes.c_int64(n), ctypes.c_int32(d), ctypes.c_uint64(seed),
                                        _stream()))


def gs_sgns_step_bf16(w_in, w_out, walks, walk_id_base: int, window: int, n_neg: int, alias,
                     lr: float, seed: int, mode: int, loss_sum=None, pair_count=None,
                     pairs_dump=None, negs_dump=None):
    """gs_sgns_step on torch.bfloat16 tables (fp32 arithmetic, round-to-nearest write-back)."""
    n_nodes, dim = w_in.shape
    n_walks, walk_len = walks.shape
    _check(lib().gs_sgns_step_bf16(
        _dev(w_in, torch.bfloat16, "w_in"), _dev(w_out, torch.bfloat16, "w_out"),
        ctypes.c_int64(n_nodes), ctypes.c_int32(dim), _dev(walks, torch.int32, "walks", n_walks == 0),
        ctypes.c_int64(n_walks), ctypes.c_int64(walk_id_base), ctypes.c_int32(walk_len),
        ctypes.c_int32(window), ctypes.c_int32(n_neg), _dev(alias, torch.int64, "alias", n_neg == 0),
        ctypes.c_float(lr), ctypes.c_uint64(seed), ctypes.c_int32(mode),
        _dev(loss_sum, torch.float64, "loss_sum", True), _dev(pair_count, torch.int64, "pair_count", True),
        _dev(pairs_dump, torch.int32, "pairs_dump", True), _dev(negs_dump, torch.int32, "negs_dump", True),
        _stream()))


def gs_sgns_step_static(w_in, w_out, walks, walk_id_base: int, window: int, n_neg: int, alias,
                        lr: float, seed: int, loss_sum=None, pair_count=None):
    """Deterministic SGNS step that allocates nothing on the device (fixed 32 MiB scratch inside
    the library).  For callers that may not call cudaMalloc; small batches only - see gs.h."""
    n_nodes, dim = w_in.shape
    n_walks, walk_len = walks.shape
    _check(lib().gs_sgns_step_static(
        _dev(w_in, torch.float32, "w_in"), _dev(w_out, torch.float32, "w_out"),
        ctypes.c_int64(n_nodes), ctypes.c_int32(dim), _dev(walks, torch.int32, "walks", n_walks == 0),
        ctypes.c_int64(n_walks), ctypes.c_int64(walk_id_base), ctypes.c_int32(walk_len),
        ctypes.c_int32(window), ctypes.c_int32(n_neg), _dev(alias, torch.int64, "alias", n_neg == 0),
        ctypes.c_float(lr), ctypes.c_uint64(seed),
        _dev(loss_sum, torch.float64, "loss_sum", True), _dev(pair_count, torch.int64, "pair_count", True),
        _stream()))


def gs_sgns_step_momentum(w_in, w_out, m_in, m_out, last_in, last_out, walks, walk_id_base: int,
                          window: int, n_neg: int, alias, lr: float, momentum: float, iteration: int,
                          seed: int, loss_sum=None, pair_count=None):
    """Synchronous step with SGD momentum, rows updated lazily (see gs.h)."""
    n_nodes, dim = w_in.shape
    n_walks, walk_len = walks.shape
    _check(lib().gs_sgns_step_momentum(
        _dev(w_in, torch.float32, "w_in"), _dev(w_out, torch.float32, "w_out"),
        _dev(m_in, torch.float32, "m_in"), _dev(m_out, torch.float32, "m_out"),
        _dev(last_in, torch.int32, "last_in"), _dev(last_out, torch.int32, "last_out"),
        ctypes.c_int64(n_nodes), ctypes.c_int32(dim), _dev(walks, torch.int32, "walks", n_walks == 0),
        ctypes.c_int64(n_walks), ctypes.c_int64(walk_id_base), ctypes.c_int32(walk_len),
        ctypes.c_int32(window), ctypes.c_int32(n_neg), _dev(alias, torch.int64, "alias", n_neg == 0),
        ctypes.c_float(lr), ctypes.c_float(momentum), ctypes.c_int32(iteration), ctypes.c_uint64(seed),
        _dev(loss_sum, torch.float64, "loss_sum", True), _dev(pair_count, torch.int64, "pair_count", True),
        _stream()))


def gs_momentum_flush(w, m, last, lr: float, momentum: float, iteration: int):
    n_rows, dim = w.shape
    _check(lib().gs_momentum_flush(
        _dev(w, torch.float32, "w"), _dev(m, torch.float32, "m"), _dev(last, torch.int32, "last"),
        ctypes.c_int64(n_rows), ctypes.c_int32(dim), ctypes.c_float(lr), ctypes.c_float(momentum),
        ctypes.c_int32(iteration), _stream()))


def gs_sgns_step_adam(w_in, w_out, m_in, v_in, m_out, v_out, walks, walk_id_base: int, window: int,
                      n_neg: int, alias, lr: float, beta1: float, beta2: float, eps: float, step: int,
                      seed: int, pair_mode: int = 0, loss_sum=None, pair_count=None):
    """Synchronous step with Adam on the rows of the batch (see gs.h); step counts from 1."""
    n_nodes, dim = w_in.shape
    n_walks, walk_len = walks.shape
    _check(lib().gs_sgns_step_adam(
        _dev(w_in, torch.float32, "w_in"), _dev(w_out, torch.float32, "w_out"),
        _dev(m_in, torch.float32, "m_in"), _dev(v_in, torch.float32, "v_in"),
        _dev(m_out, torch.float32, "m_out"), _dev(v_out, torch.float32, "v_out"),
        ctypes.c_int64(n_nodes), ctypes.c_int32(dim), _dev(walks, torch.int32, "walks", n_walks == 0),
        ctypes.c_int64(n_walks), ctypes.c_int64(walk_id_base), ctypes.c_int32(walk_len),
        ctypes.c_int32(window), ctypes.c_int32(n_neg), _dev(alias, torch.int64, "alias", n_neg == 0),
        ctypes.c_float(lr), ctypes.c_float(beta1), ctypes.c_float(beta2), ctypes.c_float(eps),
        ctypes.c_int64(step), ctypes.c_uint64(seed), ctypes.c_int32(pair_mode),
        _dev(loss_sum, torch.float64, "loss_sum", True), _dev(pair_count, torch.int64, "pair_count", True),
        _stream()))


def gs_build_keep_thresholds(weights: np.ndarray, t: float) -> np.ndarray:
    """Host call.  Sub-sampling thresholds (uint32, 0xFFFFFFFF = always kept)."""
    w = np.ascontiguousarray(weights, dtype=np.float64)
    out = np.empty(len(w), dtype=np.uint32)
    _check(lib().gs_build_keep_thresholds(w.ctypes.data_as(ctypes.c_void_p), ctypes.c_int64(len(w)),
                                          ctypes.c_double(t), out.ctypes.data_as(ctypes.c_void_p)))
    return out


def gs_subsample_walks(walks, walk_id_base: int, keep_thr, seed: int, out=None, kept=None):
    """Drops walk entries by the thresholds (int32 CUDA tensor holding the uint32 bit patterns)
    and compacts each walk; out may be walks itself."""
    n_walks, walk_len = walks.shape
    if out is None:
        out = torch.empty_like(walks)
    _check(lib().gs_subsample_walks(
        _dev(walks, torch.int32, "walks", n_walks == 0), ctypes.c_int64(n_walks),
        ctypes.c_int64(walk_id_base), ctypes.c_int32(walk_len),
        _dev(keep_thr, torch.int32, "keep_thr", n_walks == 0),
        ctypes.c_int64(keep_thr.numel() if keep_thr is not None else 1), ctypes.c_uint64(seed),
        _dev(out, torch.int32, "out", n_walks == 0), _dev(kept, torch.int64, "kept", True), _stream()))
    return out


def gs_shuffled_starts(n_nodes: int, seed: int, epoch: int, walk_id_first: int, count: int, device,
                       out=None):
    """Start nodes of walk ids [first, first + count) under the keyed bijection of the epoch."""
    if out is None:
        out = torch.empty(count, dtype=torch.int32, device=device)
    _check(lib().gs_shuffled_starts(ctypes.c_int64(n_nodes), ctypes.c_uint64(seed),
                                    ctypes.c_uint32(epoch), ctypes.c_int64(walk_id_first),
                                    ctypes.c_int64(count), _dev(out, torch.int32, "out", count == 0),
                                    _stream()))
    return out


@dataclass
class EpochResult:
    loss_sum: float
    pairs: int
    steps: int
    cap_hits: int
    batches: int
    masked_negs: int
    ms_walk: float
    ms_sgns: float
    ms_total: float
    ms_prepare: float = 0.0
    refused_ids: int = 0


def gs_sgns_epoch(graph: Graph, alias, w_in, w_out, *, walks_per_node, walk_len, window, n_neg,
                  lr0, batch_walks, seed, mode, walk_kind=GS_WALK_UNIFORM,
                  lr_schedule=GS_LR_CONSTANT, p=1.0, q=1.0, max_rounds=1024, first_batch=0,
                  num_batches=0, keep_thr=None, shuffle_epoch=None, optimizer=GS_OPT_SGD, momentum=0.0,
                  beta2=0.999, eps=1e-8, iteration_base=0, m_in=None, m_out=None, v_in=None, v_out=None,
                  last_in=None, last_out=None) -> EpochResult:
    if w_in.dtype not in (torch.float32, torch.float16, torch.bfloat16) or w_out.dtype != w_in.dtype:
        raise TypeError("tables must both be float32, both float16 or both bfloat16")
    tdt = w_in.dtype
    cfg = SgnsConfig(dim=w_in.shape[1], walks_per_node=walks_per_node, walk_len=walk_len,
                     window=window, n_neg=n_neg, walk_kind=walk_kind, lr_schedule=lr_schedule,
                     mode=mode, max_rounds=max_rounds,
                     table_dtype={torch.float16: GS_TABLE_F16, torch.bfloat16: GS_TABLE_BF16}.get(tdt, GS_TABLE_F32),
                     p=p, q=q, lr0=lr0,
                     batch_walks=batch_walks, first_batch=first_batch, num_batches=num_batches,
                     seed=seed, d_keep_thr=_dev(keep_thr, torch.int32, "keep_thr", True).value,
                     shuffle_starts=0 if shuffle_epoch is None else 1,
                     epoch=0 if shuffle_epoch is None else shuffle_epoch,
                     optimizer=optimizer, momentum=momentum, beta2=beta2, eps=eps,
                     iteration_base=iteration_base,
                     d_m_in=_dev(m_in, torch.float32, "m_in", True).value,
                     d_m_out=_dev(m_out, torch.float32, "m_out", True).value,
                     d_v_in=_dev(v_in, torch.float32, "v_in", True).value,
                     d_v_out=_dev(v_out, torch.float32, "v_out", True).value,
                     d_last_in=_dev(last_in, torch.int32, "last_in", True).value,
                     d_last_out=_dev(last_out, torch.int32, "last_out", True).value)
    st = EpochStats()
    _check(lib().gs_sgns_epoch(graph._h, _dev(alias, torch.int64, "alias", n_neg == 0),
                               _dev(w_in, tdt, "w_in"), _dev(w_out, tdt, "w_out"),
                               ctypes.byref(cfg), ctypes.byref(st), _stream()))
    return EpochResult(st.loss_sum, st.pairs, st.steps, st.cap_hits, st.batches, st.masked_negs, st.ms_walk,
                       st.ms_sgns, st.ms_total, st.ms_prepare, st.refused_ids)


def gs_refused_ids(clear: bool = False) -> int:
    """Ids refused by the kernels of the current device so far (waits for the current stream)."""
    out = ctypes.c_uint64(0)
    _check(lib().gs_refused_ids(ctypes.byref(out), ctypes.c_int32(1 if clear else 0), _stream()))
    return out.value


def gs_stalled_kernels(clear: bool = False) -> int:
    """Blocks of the tensor-core attention kernels that gave up a wait (waits for the current stream).  While it is not
    zero, attention calls raise."""
    out = ctypes.c_uint64(0)
    _check(lib().gs_stalled_kernels(ctypes.byref(out), ctypes.c_int32(1 if clear else 0), _stream()))
    return out.value


def gs_stall_drill():
    """Queues a block whose wait runs out within about two seconds, to see what a caller does with the error."""
    _check(lib().gs_stall_drill(_stream()))


def gs_release_workspace():
    _check(lib().gs_release_workspace())


def gs_tune_node2vec_group(lanes: int):
    _check(lib().gs_tune_node2vec_group(ctypes.c_int32(lanes)))


# ---------------------------------------------------------------- sequence models over walks
# These calls are a few microseconds of work for small batches, so their marshalling is lean: plain integers
# against declared argument types, and the configuration packed in one step (the layout of AttentionConfig).
_TABLE_DTYPE = {torch.float32: GS_TABLE_F32, torch.float16: GS_TABLE_F16, torch.bfloat16: GS_TABLE_BF16}
_pack_config = struct.Struct("4iq4ifiQQ24q").pack
_raw_stream = torch._C._cuda_getCurrentRawStream
_NO_STRIDE = (0, 0, 0)


def _heads(t, dtype, device, shape, name):
    """Checks one [batch, position, head, head_dim] tensor; returns its first three strides."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.get_device() != device:
        raise TypeError(f"{name} must be a tensor of {dtype} on cuda:{device}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    st = t.stride()
    if st[3] != 1 and shape[3] > 1:
        raise ValueError(f"the last dimension of {name} must be contiguous")
    return st[:3]


def _lens(t, batch, device, name):
    if t is None:
        return 0
    if not (isinstance(t, torch.Tensor) and t.get_device() == device and t.dtype is torch.int32
            and t.shape == (batch,) and t.is_contiguous()):
        raise TypeError(f"{name} must be a contiguous int32 tensor of {batch} lengths on cuda:{device}")
    return t.data_ptr()


def _attention_shape(q, k, scale, window, q_lens, k_lens):
    """(device, leading fields of the configuration, shape of k and v)"""
    if not (isinstance(q, torch.Tensor) and q.is_cuda and q.dim() == 4 and q.dtype in _TABLE_DTYPE):
        raise TypeError("q must be a CUDA tensor [batch, position, head, head_dim] of float32, float16 or bfloat16")
    if not (isinstance(k, torch.Tensor) and k.dim() == 4):
        raise TypeError("k must be a tensor [batch, position, head, head_dim]")
    device = q.get_device()
    if device != torch._C._cuda_getDevice():
        raise ValueError(f"q is on {q.device}, which is not the current device")
    b, n, hq, d = q.shape
    _, m, hk, _ = k.shape
    if scale is None:
        scale = d ** -0.5 if d else 1.0
    return device, (_TABLE_DTYPE[q.dtype], d, hq, hk, b, n, m, window[0], window[1], scale, 0,
                    _lens(q_lens, b, device, "q_lens"), _lens(k_lens, b, device, "k_lens")), (b, m, hk, d)


def gs_attention_forward(q, k, v, scale=None, window=(-1, -1), q_lens=None, k_lens=None, out=None, lse=None):
    """Attention of q[batch, q_len, q_heads, head_dim] over k, v[batch, k_len, kv_heads, head_dim]
    (see gs.h for the visible keys).  Returns (out like q, lse float32[batch, q_heads, q_len])."""
    device, lead, kv = _attention_shape(q, k, scale, window, q_lens, k_lens)
    shape, dtype = q.shape, q.dtype
    rows = (shape[0], shape[2], shape[1])
    if out is None:
        out = torch.empty_like(q)
    if lse is None:
        lse = q.new_empty(rows, dtype=torch.float32)
    elif lse.shape != rows or lse.dtype is not torch.float32 or lse.get_device() != device or not lse.is_contiguous():
        raise ValueError(f"lse must be a contiguous float32 tensor of shape {rows} on cuda:{device}")
    cfg = _pack_config(*lead, *_heads(q, dtype, device, shape, "q"), *_heads(k, dtype, device, kv, "k"),
                       *_heads(v, dtype, device, kv, "v"), *_heads(out, dtype, device, shape, "out"),
                       *_NO_STRIDE, *_NO_STRIDE, *_NO_STRIDE, *_NO_STRIDE)
    _check(lib().gs_attention_forward(cfg, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(),
                                      _raw_stream(device)))
    return out, lse


@functools.lru_cache(maxsize=256)
def _backward_work(lead):
    """Floats of scratch for a configuration (its first fields; pointers and strides do not matter)."""
    return max(0, lib().gs_attention_backward_work(_pack_config(*lead, 0, 0, *(_NO_STRIDE * 8))))


def gs_attention_backward(dout, q, k, v, out, lse, scale=None, window=(-1, -1), q_lens=None, k_lens=None,
                          dq=None, dk=None, dv=None):
    """Gradients of gs_attention_forward: returns (dq, dk, dv), shaped like q, k, v.  out and lse are
    the forward call's results, dout the gradient of out."""
    device, lead, kv = _attention_shape(q, k, scale, window, q_lens, k_lens)
    shape, dtype = q.shape, q.dtype
    rows = (shape[0], shape[2], shape[1])
    if not isinstance(lse, torch.Tensor) or lse.shape != rows or lse.dtype is not torch.float32 \
            or lse.get_device() != device or not lse.is_contiguous():
        raise ValueError(f"lse must be a contiguous float32 tensor of shape {rows} on cuda:{device}")
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    cfg = _pack_config(*lead, *_heads(q, dtype, device, shape, "q"), *_heads(k, dtype, device, kv, "k"),
                       *_heads(v, dtype, device, kv, "v"), *_heads(out, dtype, device, shape, "out"),
                       *_heads(dout, dtype, device, shape, "dout"), *_heads(dq, dtype, device, shape, "dq"),
                       *_heads(dk, dtype, device, kv, "dk"), *_heads(dv, dtype, device, kv, "dv"))
    work = lse.new_empty(_backward_work(lead[:11]))
    _check(lib().gs_attention_backward(cfg, dout.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                                       lse.data_ptr(), work.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                                       _raw_stream(device)))
    return dq, dk, dv


def _tensor_list(tensors, device, name):
    """The host array of gs_tensor entries, as bytes."""
    words = []
    for t in tensors:
        code = _TABLE_DTYPE.get(t.dtype)
        if code is None or t.get_device() != device or not t.is_contiguous():
            raise TypeError(f"{name} must be contiguous float32, float16 or bfloat16 tensors on the current CUDA device")
        words += (t.data_ptr(), t.numel(), code)
    return struct.pack(f"{len(words)}Q", *words)


@functools.lru_cache(maxsize=64)
def _norm_work(n, device):
    return lib().gs_gradient_norm_work(n), torch.device("cuda", device)


def _norm_buffers(n, device):
    words, on = _norm_work(n, device)
    return torch.empty(words, dtype=torch.float64, device=on), torch.empty(1, dtype=torch.float32, device=on)


def gs_gradient_norm(grads):
    """Euclidean norm of all tensors of `grads` taken as one vector: float32[1] on the device."""
    device = torch._C._cuda_getDevice()
    entries = _tensor_list(grads, device, "grads")
    work, norm = _norm_buffers(len(grads), device)
    _check(lib().gs_gradient_norm(entries, len(grads), work.data_ptr(), norm.data_ptr(), _raw_stream(device)))
    return norm


def gs_clip_gradients(grads, max_norm: float, out=None):
    """Scales `grads` (into the tensors `out`, or in place) so that their joint norm is at most
    max_norm; returns the norm before clipping, float32[1] on the device (nothing waits for it)."""
    device = torch._C._cuda_getDevice()
    entries = _tensor_list(grads, device, "grads")
    targets = None
    if out is not None:
        if len(out) != len(grads):
            raise ValueError(f"{len(out)} outputs for {len(grads)} gradients")
        targets = _tensor_list(out, device, "out")
    work, norm = _norm_buffers(len(grads), device)
    _check(lib().gs_clip_gradients(entries, targets, len(grads), max_norm, work.data_ptr(), norm.data_ptr(),
                                   _raw_stream(device)))
    return norm


# ---------------------------------------------------------------- layers around attention
_pack_norm = struct.Struct("2i2qifQ8q").pack
_pack_recurrence = struct.Struct("2i2qQ12q").pack
_NO_STRIDE2 = (0, 0)


def _positions(t, dtype, device, shape, name):
    """Checks one [batch, position, column] tensor; returns its first two strides."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.get_device() != device:
        raise TypeError(f"{name} must be a tensor of {dtype} on cuda:{device}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    st = t.stride()
    if st[2] != 1 and shape[2] > 1:
        raise ValueError(f"the last dimension of {name} must be contiguous")
    return st[:2]


def _like(t):
    """A result beside t[batch, position, column]: its layout where that is dense, contiguous columns always (torch may put another
    dimension inmost where positions of t share memory)."""
    r = torch.empty_like(t)
    return r if r.dim() != 3 or r.stride(2) == 1 else t.new_empty(t.shape)


def _leading(t, name, dtypes):
    """Device and dtype code of the tensor that a call's other tensors are measured by."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dim() == 3 and t.dtype in dtypes):
        raise TypeError(f"{name} must be a CUDA tensor [batch, position, column] of {', '.join(str(d)[6:] for d in dtypes)}")
    device = t.get_device()
    if device != torch._C._cuda_getDevice():
        raise ValueError(f"{name} is on {t.device}, which is not the current device")
    return device


def _vector(t, dtype, device, columns, name):
    if t is None:
        return 0
    if not (isinstance(t, torch.Tensor) and t.get_device() == device and t.dtype is dtype and t.shape == (columns,)
            and t.is_contiguous()):
        raise TypeError(f"{name} must be a contiguous tensor of {columns} values of {dtype} on cuda:{device}")
    return t.data_ptr()


def _vector_dtype(weight, bias, dtype):
    """Type of weight and bias: float32 or the tensors' own, one for both."""
    given = weight if weight is not None else bias
    if given is None:
        return torch.float32
    if not isinstance(given, torch.Tensor) or (given.dtype is not torch.float32 and given.dtype is not dtype):
        raise TypeError(f"weight and bias must be tensors of float32 or {dtype}")
    return given.dtype


def _exactly(t, dtype, device, shape, name):
    """Checks a contiguous tensor of the library's own layout; returns its address."""
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == device and t.shape == shape
            and t.is_contiguous()):
        raise TypeError(f"{name} must be a contiguous tensor of {dtype} and shape {tuple(shape)} on cuda:{device}")
    return t.data_ptr()


def gs_layer_norm_forward(x, weight=None, bias=None, eps=1e-5, lens=None, checkpoint=False, y=None):
    """Layer norm of x[batch, length, columns] over its columns (see gs.h).  Returns (y like x, stats float32[batch, length, 2]),
    with checkpoint=True (y, stats, packed, scales): x in 8 bits, to be given to gs_layer_norm_backward in its place."""
    device = _leading(x, "x", _TABLE_DTYPE)
    shape, dtype = x.shape, x.dtype
    b, n, c = shape
    wt = _vector_dtype(weight, bias, dtype)
    y = _like(x) if y is None else y
    stats = x.new_empty((b, n, 2), dtype=torch.float32)
    packed = scales = None
    if checkpoint:
        packed = x.new_empty(shape, dtype=torch.int8)
        scales = x.new_empty((b, n, (c + 127) // 128), dtype=torch.float32)
    cfg = _pack_norm(_TABLE_DTYPE[dtype], _TABLE_DTYPE[wt], b, n, c, eps, _lens(lens, b, device, "lens"),
                     *_positions(x, dtype, device, shape, "x"), *_positions(y, dtype, device, shape, "y"), *_NO_STRIDE2, *_NO_STRIDE2)
    _check(lib().gs_layer_norm_forward(cfg, x.data_ptr(), _vector(weight, wt, device, c, "weight"),
                                       _vector(bias, wt, device, c, "bias"), y.data_ptr(), stats.data_ptr(),
                                       packed.data_ptr() if checkpoint else 0, scales.data_ptr() if checkpoint else 0,
                                       _raw_stream(device)))
    return (y, stats, packed, scales) if checkpoint else (y, stats)


@functools.lru_cache(maxsize=256)
def _norm_backward_work(dtype, rows, columns, device):
    """Floats of scratch, which follow the number of blocks."""
    return max(0, lib().gs_layer_norm_backward_work(_pack_norm(dtype, dtype, 1, rows, columns, 0.0, 0, *(_NO_STRIDE2 * 4))))


def gs_layer_norm_backward(dy, x, weight, bias, stats, lens=None, scales=None, dx=None, sums=True):
    """Gradients of gs_layer_norm_forward: returns (dx like dy, dweight, dbias), None for a weight or bias that is None, and for both
    with sums=False (frozen ones).  x: the forward call's, or its `packed` together with its `scales`."""
    device = _leading(dy, "dy", _TABLE_DTYPE)
    shape, dtype = dy.shape, dy.dtype
    b, n, c = shape
    wt = _vector_dtype(weight, bias, dtype)
    dx = _like(dy) if dx is None else dx
    if scales is None:
        at_x, strides, packed, at_scales = None, _positions(x, dtype, device, shape, "x"), 0, 0
        at_x = x.data_ptr()
    else:
        packed, strides, at_x = _exactly(x, torch.int8, device, shape, "x"), _NO_STRIDE2, 0
        at_scales = _exactly(scales, torch.float32, device, (b, n, (c + 127) // 128), "scales")
    at_stats = _exactly(stats, torch.float32, device, (b, n, 2), "stats")
    cfg = _pack_norm(_TABLE_DTYPE[dtype], _TABLE_DTYPE[wt], b, n, c, 0.0, _lens(lens, b, device, "lens"), *strides, *_NO_STRIDE2,
                     *_positions(dy, dtype, device, shape, "dy"), *_positions(dx, dtype, device, shape, "dx"))
    at_weight = _vector(weight, wt, device, c, "weight")
    _vector(bias, wt, device, c, "bias")
    dweight = torch.empty_like(weight) if sums and weight is not None else None
    dbias = torch.empty_like(bias) if sums and bias is not None else None
    work = None if dweight is None and dbias is None else stats.new_empty(_norm_backward_work(_TABLE_DTYPE[dtype], b * n, c, device))
    _check(lib().gs_layer_norm_backward(cfg, dy.data_ptr(), at_x, packed, at_scales, at_weight, at_stats, 0 if work is None else work.data_ptr(),
                                        dx.data_ptr(), 0 if dweight is None else dweight.data_ptr(),
                                        0 if dbias is None else dbias.data_ptr(), _raw_stream(device)))
    return dx, dweight, dbias


GS_RECURRENCE_SPAN = 128              # positions between two of the states that the forward call keeps


def _state(t, device, shape, name):
    return 0 if t is None else _exactly(t, torch.float32, device, shape, name)


@functools.lru_cache(maxsize=64)
def _recurrence_work(length, device):
    """Floats of scratch, which depend on the length (and the device) only."""
    return max(0, lib().gs_recurrence_work(_pack_recurrence(0, length, 1, 1, 0, *(_NO_STRIDE2 * 6))))


def gs_recurrence_forward(gate, x, h0=None, lens=None, keep=True, out=None, final=None):
    """Gated linear recurrence along the positions of x[batch, length, channels] (see gs.h) from the state h0 float32[batch, channels]
    (zeros if None).  Returns (out like x, final float32[batch, channels], states): states is what gs_recurrence_backward needs,
    None with keep=False.  final may be h0: sequences are continued by handing it to the next call."""
    device = _leading(x, "x", _TABLE_DTYPE)
    shape, dtype = x.shape, x.dtype
    b, n, c = shape
    out = _like(x) if out is None else out
    final = x.new_empty((b, c), dtype=torch.float32) if final is None else final
    states = x.new_empty((b, max(0, n - 1) // GS_RECURRENCE_SPAN, c), dtype=torch.float32) if keep else None
    cfg = _pack_recurrence(_TABLE_DTYPE[dtype], n, b, c, _lens(lens, b, device, "lens"),
                           *_positions(gate, dtype, device, shape, "gate"), *_positions(x, dtype, device, shape, "x"),
                           *_positions(out, dtype, device, shape, "out"), *(_NO_STRIDE2 * 3))
    work = final.new_empty(words) if (words := _recurrence_work(n, device)) else None
    _check(lib().gs_recurrence_forward(cfg, gate.data_ptr(), x.data_ptr(), _state(h0, device, (b, c), "h0"), out.data_ptr(),
                                       _state(final, device, (b, c), "final"), states.data_ptr() if keep else 0,
                                       0 if work is None else work.data_ptr(), _raw_stream(device)))
    return out, final, states


def gs_recurrence_backward(dout, gate, x, h0=None, states=None, dfinal=None, lens=None, dgate=None, dx=None):
    """Gradients of gs_recurrence_forward: returns (dgate, dx, dh0 float32[batch, channels]).  dout and dfinal are the gradients of
    out and final (None: zeros), states the forward call's."""
    device = _leading(x, "x", _TABLE_DTYPE)
    shape, dtype = x.shape, x.dtype
    b, n, c = shape
    dgate = _like(gate) if dgate is None else dgate
    dx = _like(x) if dx is None else dx
    dh0 = x.new_empty((b, c), dtype=torch.float32)
    kept = max(0, n - 1) // GS_RECURRENCE_SPAN
    cfg = _pack_recurrence(_TABLE_DTYPE[dtype], n, b, c, _lens(lens, b, device, "lens"),
                           *_positions(gate, dtype, device, shape, "gate"), *_positions(x, dtype, device, shape, "x"), *_NO_STRIDE2,
                           *(_NO_STRIDE2 if dout is None else _positions(dout, dtype, device, shape, "dout")),
                           *_positions(dgate, dtype, device, shape, "dgate"), *_positions(dx, dtype, device, shape, "dx"))
    work = dh0.new_empty(words) if (words := _recurrence_work(n, device)) else None
    at_states = _exactly(states, torch.float32, device, (b, kept, c), "states") if kept else 0
    _check(lib().gs_recurrence_backward(cfg, 0 if dout is None else dout.data_ptr(), _state(dfinal, device, (b, c), "dfinal"),
                                        gate.data_ptr(), x.data_ptr(), _state(h0, device, (b, c), "h0"), at_states,
                                        dgate.data_ptr(), dx.data_ptr(), dh0.data_ptr(), 0 if work is None else work.data_ptr(),
                                        _raw_stream(device)))
    return dgate, dx, dh0


def _rows(t, name):
    """(rows, columns, row stride) of a tensor whose leading dimensions are one run of rows."""
    if t.dim() == 0:
        raise ValueError(f"{name} must have at least one dimension")
    columns = t.shape[-1]
    rows = t.numel() // columns if columns else 0
    if t.is_contiguous():
        return rows, columns, columns
    if t.dim() == 2 and (t.stride(1) == 1 or columns == 1):
        return rows, columns, t.stride(0)
    raise ValueError(f"{name} must be contiguous, or have two dimensions and contiguous rows")


def gs_checkpoint_pack(x):
    """x[..., columns] in 8 bits (see gs.h): returns (packed int8 like x, scales float32[..., ceil(columns / 128)])."""
    if not (isinstance(x, torch.Tensor) and x.is_cuda and x.dtype in _TABLE_DTYPE):
        raise TypeError("x must be a CUDA tensor of float32, float16 or bfloat16")
    device = x.get_device()
    if device != torch._C._cuda_getDevice():
        raise ValueError(f"x is on {x.device}, which is not the current device")
    rows, columns, stride = _rows(x, "x")
    packed = x.new_empty(x.shape, dtype=torch.int8)
    scales = x.new_empty((*x.shape[:-1], (columns + 127) // 128), dtype=torch.float32)
    _check(lib().gs_checkpoint_pack(_TABLE_DTYPE[x.dtype], x.data_ptr(), rows, columns, stride, packed.data_ptr(),
                                    scales.data_ptr(), _raw_stream(device)))
    return packed, scales


def gs_checkpoint_unpack(packed, scales, dtype=torch.float32, out=None):
    """The values of gs_checkpoint_pack's result as a tensor of `dtype` (or in `out`)."""
    if not (isinstance(packed, torch.Tensor) and packed.is_cuda and packed.dtype is torch.int8 and packed.is_contiguous()
            and packed.dim() > 0):
        raise TypeError("packed must be a contiguous int8 CUDA tensor")
    device = packed.get_device()
    if device != torch._C._cuda_getDevice():
        raise ValueError(f"packed is on {packed.device}, which is not the current device")
    at_scales = _exactly(scales, torch.float32, device, (*packed.shape[:-1], (packed.shape[-1] + 127) // 128), "scales")
    if out is None:
        if dtype not in _TABLE_DTYPE:
            raise TypeError("dtype must be float32, float16 or bfloat16")
        out = packed.new_empty(packed.shape, dtype=dtype)
    elif not isinstance(out, torch.Tensor) or out.dtype not in _TABLE_DTYPE or out.get_device() != device:
        raise TypeError(f"out must be a tensor of float32, float16 or bfloat16 on cuda:{device}")
    elif out.shape != packed.shape:
        raise ValueError(f"out has shape {tuple(out.shape)}, expected {tuple(packed.shape)}")
    rows, columns, stride = _rows(out, "out")
    _check(lib().gs_checkpoint_unpack(_TABLE_DTYPE[out.dtype], packed.data_ptr(), at_scales, rows, columns, stride, out.data_ptr(),
                                      _raw_stream(device)))
    return out
