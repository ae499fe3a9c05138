"""Binding of libsdverify.so: same names as the C header, argument
marshalling only (in native code, csrc/native_calls.cpp; the plain ctypes
handle of the library is `lib`).  Tensors are torch CUDA tensors (device memory
and streams are all torch is used for); every step of the computation runs in
the library's kernels.  There is no CPU fallback: if the shared libraries
cannot be loaded, importing this module raises.
"""
from __future__ import annotations

import copy
import ctypes as C
import os
from typing import List, Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsdverify.so")
NATIVE_PATH = os.path.join(_HERE, "_sdnative.so")

SD_OK = 0
SD_ERR_INVALID_ARG = -1
SD_ERR_INVALID_TREE = -2
SD_ERR_UNSUPPORTED = -3
SD_ERR_WORKSPACE = -4
SD_ERR_CUDA = -5
SD_ERR_TIMEOUT = -6
SD_ERR_BOUNDS = -7

# kernel launches behind one call (kept in step with the kernels; used for launch accounting)
KERNELS_PER_ATTENTION = 1      # split-KV chunks merge inside the kernel (thread-block cluster)
ATTENTION_LAYERS_PER_LAUNCH = 32   # sd_verify_attention_layers: layers sharing one launch
KERNELS_PER_TAIL = 2               # sd_lmhead_accept_compact: LM-head tiles + fused tail kernel
KERNELS_PER_LMHEAD = 2         # tiles + cross-slab reduce
KERNELS_PER_SAMPLED_TAIL = 2       # sd_lmhead_accept_sampled_compact: LM-head tiles + one cluster kernel
KERNELS_PER_ROWS_CALL = 1          # each of the calls on rows of logits

SD_F32 = 0                     # sd_dtype
SD_BF16 = 1

EXPORTS = ["sd_version", "sd_status_string", "sd_workspace_bytes", "sd_tree_prepare",
           "sd_verify_attention", "sd_verify_attention_layers", "sd_lmhead_argmax", "sd_lmhead_argmax_static", "sd_accept_tree",
           "sd_compact_kv", "sd_lmhead_accept_compact", "sd_lmhead_stats", "sd_accept_tree_sampled", "sd_lmhead_accept_sampled_compact", "sd_accept_chain_sampled", "sd_lmhead_stats_logits", "sd_accept_tree_sampled_q",
           "sd_draft_feature_attention",
           "sd_top_logits", "sd_sample_logits", "sd_filter_logits", "sd_distill_loss", "sd_distill_grad",
           "sd_assign_blocks", "sd_prompt_plan_bytes", "sd_prompt_prepare", "sd_append_kv", "sd_prompt_workspace_bytes", "sd_prompt_attention"]


class sd_kv_layer(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("num_blocks", C.c_int32)]


class sd_batch(C.Structure):
    _fields_ = [("B", C.c_int32), ("T_max", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32),
                ("D", C.c_int32), ("block_size", C.c_int32), ("max_blocks_per_seq", C.c_int32),
                ("block_table", C.c_void_p), ("len", C.c_void_p), ("n_nodes", C.c_void_p),
                ("parents", C.c_void_p), ("anc_mask", C.c_void_p)]


class sd_sampling(C.Structure):
    _fields_ = [("inv_temp", C.c_void_p), ("top_k", C.c_void_p), ("top_p", C.c_void_p), ("min_p", C.c_void_p),
                ("n_used", C.c_void_p), ("per", C.c_int32)]


class sd_block_pool(C.Structure):
    _fields_ = [("free_blocks", C.c_void_p), ("n_free", C.c_void_p), ("num_blocks", C.c_int32)]


class sd_prompts(C.Structure):
    _fields_ = [("B", C.c_int32), ("N", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("D", C.c_int32), ("block_size", C.c_int32),
                ("max_blocks_per_seq", C.c_int32), ("num_blocks", C.c_int32), ("block_table", C.c_void_p), ("n_blocks", C.c_void_p),
                ("len", C.c_void_p), ("n_new", C.c_void_p), ("start", C.c_void_p), ("slot", C.c_void_p), ("position", C.c_void_p),
                ("plan", C.c_void_p)]


def _load(path: str = LIB_PATH) -> C.CDLL:
    if path == LIB_PATH and not (os.path.exists(LIB_PATH) and os.path.exists(NATIVE_PATH)):
        from . import build as _build          # needs nvcc; raises if it fails
        _build.build()
    lib = C.CDLL(path)
    lib.sd_version.restype = C.c_int
    lib.sd_status_string.restype = C.c_char_p
    lib.sd_status_string.argtypes = [C.c_int]
    lib.sd_workspace_bytes.restype = C.c_size_t
    lib.sd_workspace_bytes.argtypes = [C.c_void_p, C.c_int32, C.c_int32]
    lib.sd_tree_prepare.restype = C.c_int
    lib.sd_tree_prepare.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p]
    lib.sd_verify_attention.restype = C.c_int
    lib.sd_verify_attention.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                        C.c_float, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t,
                                        C.c_void_p, C.c_void_p]
    lib.sd_verify_attention_layers.restype = C.c_int
    lib.sd_verify_attention_layers.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p,
                                               C.c_void_p, C.c_float, C.c_void_p, C.c_void_p, C.c_void_p,
                                               C.c_size_t, C.c_void_p, C.c_void_p]
    lib.sd_lmhead_argmax.restype = C.c_int
    lib.sd_lmhead_argmax.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32,
                                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
    lib.sd_lmhead_argmax_static.restype = C.c_int
    lib.sd_lmhead_argmax_static.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32,
                                            C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.sd_accept_tree.restype = C.c_int
    lib.sd_accept_tree.argtypes = [C.c_void_p] * 9
    lib.sd_compact_kv.restype = C.c_int
    lib.sd_compact_kv.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p,
                                  C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.sd_lmhead_accept_compact.restype = C.c_int
    lib.sd_lmhead_accept_compact.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p,
                                             C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p,
                                             C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                             C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
    lib.sd_lmhead_stats.restype = C.c_int
    lib.sd_lmhead_stats.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_float,
                                    C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t,
                                    C.c_void_p, C.c_void_p]
    lib.sd_accept_tree_sampled.restype = C.c_int
    lib.sd_accept_tree_sampled.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_float,
                                           C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                           C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                           C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
    lib.sd_accept_chain_sampled.restype = C.c_int
    lib.sd_accept_tree_sampled_q.restype = C.c_int
    lib.sd_accept_tree_sampled_q.argtypes = [C.c_void_p, C.c_int32, C.c_float] + [C.c_void_p] * 12
    lib.sd_lmhead_stats_logits.restype = C.c_int
    lib.sd_lmhead_stats_logits.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_float,
                                           C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t,
                                           C.c_void_p, C.c_void_p]
    lib.sd_accept_chain_sampled.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_float,
                                            C.c_void_p, C.c_void_p,
                                            C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                            C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                            C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
    lib.sd_lmhead_accept_sampled_compact.restype = C.c_int
    lib.sd_lmhead_accept_sampled_compact.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_float,
                                                     C.c_void_p, C.c_void_p, C.c_void_p,
                                                     C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p,
                                                     C.c_void_p, C.c_void_p,
                                                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                                     C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
    lib.sd_draft_feature_attention.restype = C.c_int
    lib.sd_draft_feature_attention.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32,
                                               C.c_int32, C.c_int32, C.c_float, C.c_void_p, C.c_void_p]
    rows = [C.c_void_p, C.c_int32, C.c_int64, C.c_int32, C.c_int32]
    lib.sd_top_logits.restype = C.c_int
    lib.sd_top_logits.argtypes = rows + [C.c_int32, C.c_float] + [C.c_void_p] * 5
    lib.sd_sample_logits.restype = C.c_int
    lib.sd_sample_logits.argtypes = rows + [C.c_void_p, C.c_void_p, C.c_int32] + [C.c_void_p] * 6
    lib.sd_filter_logits.restype = C.c_int
    lib.sd_filter_logits.argtypes = rows + [C.c_void_p] * 6
    teacher = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_float, C.c_float, C.c_float]
    lib.sd_distill_loss.restype = C.c_int
    lib.sd_distill_loss.argtypes = rows + teacher + [C.c_void_p] * 5 + [C.c_int64, C.c_void_p, C.c_void_p]
    lib.sd_distill_grad.restype = C.c_int
    lib.sd_distill_grad.argtypes = rows + teacher + [C.c_void_p] * 3 + [C.c_int64, C.c_void_p, C.c_void_p]
    lib.sd_assign_blocks.restype = C.c_int
    lib.sd_assign_blocks.argtypes = [C.c_void_p, C.c_int32, C.c_int32] + [C.c_void_p] * 7
    lib.sd_prompt_prepare.restype = C.c_int
    lib.sd_prompt_prepare.argtypes = [C.c_void_p] * 3
    for sized in (lib.sd_prompt_plan_bytes, lib.sd_prompt_workspace_bytes):
        sized.restype = C.c_size_t
        sized.argtypes = [C.c_void_p]
    lib.sd_append_kv.restype = C.c_int
    lib.sd_append_kv.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]
    lib.sd_prompt_attention.restype = C.c_int
    lib.sd_prompt_attention.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_float, C.c_void_p, C.c_int64, C.c_void_p,
                                        C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
    return lib


lib = _load()
from . import _sdnative as _n      # noqa: E402  (linked to the library loaded above)


class SdError(RuntimeError):
    def __init__(self, code: int):
        self.code = code
        super().__init__(sd_status_string(code))


def sd_version() -> int:
    return int(lib.sd_version())


def sd_status_string(code: int) -> str:
    return lib.sd_status_string(int(code)).decode()


def _check(code: int) -> None:
    if code != SD_OK:
        raise SdError(code)


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    assert t.is_cuda and t.is_contiguous(), "device tensors must be contiguous CUDA tensors"
    return t.data_ptr()


_at = C.addressof          # address of a host structure or array


class Batch:
    """Owns the device arrays named by the C struct ``sd_batch``."""

    def __init__(self, B, T_max, Hq, Hkv, D, block_table, lens, n_nodes, parents,
                 block_size=64, device="cuda"):
        dev = torch.device(device)
        to = lambda a: torch.as_tensor(a, dtype=torch.int32).contiguous().to(dev)
        self.B, self.T_max, self.Hq, self.Hkv, self.D = int(B), int(T_max), int(Hq), int(Hkv), int(D)
        self.block_table = to(block_table).reshape(self.B, -1).contiguous()
        self.len = to(lens)
        self.n_nodes = to(n_nodes)
        self.parents = to(parents).reshape(self.B, self.T_max).contiguous()
        self.anc_mask = torch.zeros((self.B, self.T_max), dtype=torch.int64, device=dev)
        self.max_blocks = int(self.block_table.shape[1])
        self.c = sd_batch(self.B, self.T_max, self.Hq, self.Hkv, self.D, int(block_size), self.max_blocks,
                          self.block_table.data_ptr(), self.len.data_ptr(), self.n_nodes.data_ptr(),
                          self.parents.data_ptr(), self.anc_mask.data_ptr())

    @classmethod
    def of(cls, w, device="cuda") -> "Batch":
        """From any object carrying B, T_max, Hq, Hkv, D, block_table, len, n_nodes, parents."""
        return cls(w.B, w.T_max, w.Hq, w.Hkv, w.D, w.block_table, w.len, w.n_nodes, w.parents, device=device)

    def ref(self):
        return C.byref(self.c)


def kv_layer(k_cache: torch.Tensor, v_cache: torch.Tensor) -> sd_kv_layer:
    """Descriptor of one layer's paged cache.  The struct only carries addresses, so the returned
    object also holds on to the two tensors: a descriptor built from temporaries stays valid."""
    layer = sd_kv_layer(_ptr(k_cache), _ptr(v_cache), int(k_cache.shape[0]))
    layer._keep = (k_cache, v_cache)
    return layer


def new_status(device="cuda") -> torch.Tensor:
    return torch.zeros(1, dtype=torch.int32, device=device)


def sd_workspace_bytes(batch: Optional[Batch], M: int = 0, V: int = 0) -> int:
    return int(lib.sd_workspace_bytes(batch.ref() if batch is not None else None, int(M), int(V)))


def _lm_sizes(hidden, W):
    M, Hd = hidden.size(0), hidden.size(1)
    assert hidden.dim() == 2 and W.size(1) == Hd
    return M, Hd, W.size(0)


def sd_tree_prepare(batch: Batch, status: torch.Tensor, stream=None) -> None:
    _check(_n.sd_tree_prepare(_at(batch.c), status, stream))


def sd_verify_attention(batch: Batch, cache: sd_kv_layer, q, k_tree, v_tree, scale: float,
                        out, lse, workspace, status, stream=None) -> None:
    _check(_n.sd_verify_attention(_at(batch.c), _at(cache), q, k_tree, v_tree, scale, out, lse, workspace, workspace,
                                  status, stream))


class AttentionLayerSet:
    """Host arrays of per-layer pointers for ``sd_verify_attention_layers`` (built once, reused)."""

    def __init__(self, k_caches, v_caches, qs, k_trees, v_trees, outs, lses=None):
        L = len(k_caches)
        self.L = L
        self.caches = (sd_kv_layer * L)(*[kv_layer(k, v) for k, v in zip(k_caches, v_caches)])
        self.q = (C.c_void_p * L)(*[_ptr(t) for t in qs])
        self.kt = (C.c_void_p * L)(*[_ptr(t) for t in k_trees])
        self.vt = (C.c_void_p * L)(*[_ptr(t) for t in v_trees])
        self.out = (C.c_void_p * L)(*[_ptr(t) for t in outs])
        self.lse = (C.c_void_p * L)(*[_ptr(t) for t in lses]) if lses is not None else None
        self._keep = (list(k_caches), list(v_caches), list(qs), list(k_trees), list(v_trees), list(outs),
                      list(lses) if lses is not None else None)


def sd_verify_attention_layers(batch: Batch, layers: AttentionLayerSet, scale: float, workspace, status,
                               stream=None) -> None:
    _check(_n.sd_verify_attention_layers(_at(batch.c), _at(layers.caches), layers.L, _at(layers.q), _at(layers.kt),
                                         _at(layers.vt), scale, _at(layers.out), None if layers.lse is None else _at(layers.lse),
                                         workspace, workspace, status, stream))


def sd_lmhead_argmax(hidden, W, argmax, maxlogit, workspace, status, stream=None) -> None:
    M, Hd, V = _lm_sizes(hidden, W)
    _check(_n.sd_lmhead_argmax(hidden, W, M, Hd, V, argmax, maxlogit, workspace, workspace, status, stream))


def sd_lmhead_argmax_static(hidden, W, argmax, maxlogit, status, stream=None) -> None:
    """LM-head arg-max using the scratch table built into the library: for callers
    that may not allocate device memory.  At most 512 rows per call."""
    M, Hd, V = _lm_sizes(hidden, W)
    _check(_n.sd_lmhead_argmax_static(hidden, W, M, Hd, V, argmax, maxlogit, status, stream))


def sd_accept_tree(batch: Batch, draft_tok, target_argmax, n_acc, path, out_tok, new_len,
                   status, stream=None) -> None:
    _check(_n.sd_accept_tree(_at(batch.c), draft_tok, target_argmax, n_acc, path, out_tok, new_len, status, stream))


class LayerSet:
    """Host arrays of per-layer descriptors for ``sd_compact_kv`` (built once, reused)."""

    def __init__(self, k_caches: Sequence[torch.Tensor], v_caches: Sequence[torch.Tensor],
                 k_trees: Sequence[torch.Tensor], v_trees: Sequence[torch.Tensor]):
        L = len(k_caches)
        self.L = L
        self.layers = (sd_kv_layer * L)(*[kv_layer(k, v) for k, v in zip(k_caches, v_caches)])
        self.kt = (C.c_void_p * L)(*[_ptr(t) for t in k_trees])
        self.vt = (C.c_void_p * L)(*[_ptr(t) for t in v_trees])
        self._keep = (list(k_caches), list(v_caches), list(k_trees), list(v_trees))


def sd_compact_kv(batch: Batch, layers: LayerSet, n_acc, path, status, stream=None) -> None:
    _check(_n.sd_compact_kv(_at(batch.c), _at(layers.layers), layers.L, _at(layers.kt), _at(layers.vt), n_acc, path,
                            status, stream))


def sd_lmhead_accept_compact(batch: Batch, hidden, W, draft_tok, layers: LayerSet, argmax, maxlogit,
                             n_acc, path, out_tok, new_len, workspace, status, stream=None) -> None:
    """LM-head arg-max over the B * T_max rows of `hidden`, greedy acceptance and KV compaction in all
    layers; the three steps share one tail kernel."""
    M, Hd, V = _lm_sizes(hidden, W)
    assert M == batch.B * batch.T_max
    _check(_n.sd_lmhead_accept_compact(_at(batch.c), hidden, W, Hd, V, draft_tok, _at(layers.layers), layers.L,
                                       _at(layers.kt), _at(layers.vt), argmax, maxlogit, n_acc, path, out_tok,
                                       new_len, workspace, workspace, status, stream))


def group_stats_shape(M: int, V: int):
    """Shape (float32) of the optional per-group statistics table of sd_lmhead_stats."""
    return ((V + 31) // 32, M, 2)


def sd_lmhead_stats(hidden, W, inv_temp: float, argmax, maxlogit, lse, workspace, status, stream=None,
                    group_stats=None) -> None:
    """LM-head arg-max plus lse[r] = log sum_v exp(logit[r][v] * inv_temp); optionally the per-group
    (maximum, sum) table that lets sd_accept_tree_sampled skip its second pass over W."""
    M, Hd, V = _lm_sizes(hidden, W)
    _check(_n.sd_lmhead_stats(hidden, W, M, Hd, V, inv_temp, argmax, maxlogit, lse, group_stats, workspace, workspace,
                              status, stream))


def sd_accept_tree_sampled(batch: Batch, hidden, W, inv_temp: float, lse, draft_tok, u, w,
                           n_acc, path, out_tok, new_len, workspace, status, stream=None, group_stats=None) -> None:
    """Acceptance at a sampling temperature (uniforms u [B,T] and w [B] are inputs)."""
    M, Hd, V = _lm_sizes(hidden, W)
    assert M == batch.B * batch.T_max
    _check(_n.sd_accept_tree_sampled(_at(batch.c), hidden, W, Hd, V, inv_temp, lse, group_stats, draft_tok, u, w,
                                     n_acc, path, out_tok, new_len, workspace, workspace, status, stream))


def sd_lmhead_stats_logits(hidden, W, inv_temp: float, argmax, maxlogit, lse, logits, workspace, status,
                           stream=None) -> None:
    """sd_lmhead_stats that also keeps the raw logits [M,V] (device f32)."""
    M, Hd = hidden.shape
    V = W.shape[0]
    assert W.shape[1] == Hd and tuple(logits.shape) == (M, V) and logits.dtype == torch.float32 and logits.is_contiguous()
    _check(_n.sd_lmhead_stats_logits(hidden, W, M, Hd, V, inv_temp, argmax, maxlogit, lse, logits, workspace,
                                     workspace, status, stream))


def sd_accept_tree_sampled_q(batch: Batch, inv_temp: float, lse, logits, draft_tok, q_rows, u, w,
                             n_acc, path, out_tok, new_len, status, stream=None) -> None:
    """Acceptance at a sampling temperature for trees whose children were sampled from q_rows [B,T,V];
    lse [M] and logits [M,V] from sd_lmhead_stats_logits (device f32)."""
    M, V = logits.shape
    assert M == batch.B * batch.T_max and tuple(q_rows.shape) == (batch.B, batch.T_max, V)
    assert logits.dtype == torch.float32 and q_rows.dtype == torch.float32 and logits.is_contiguous() and q_rows.is_contiguous()
    _check(_n.sd_accept_tree_sampled_q(_at(batch.c), V, inv_temp, lse, logits, draft_tok, q_rows, u, w, n_acc, path,
                                       out_tok, new_len, status, stream))


def sd_accept_chain_sampled(batch: Batch, hidden, W, inv_temp: float, lse, draft_tok, q_tok, q_rows, u, w,
                            n_acc, path, out_tok, new_len, workspace, status, stream=None, logits=None) -> None:
    """Acceptance at a sampling temperature for chains drafted by sampling: q_tok [B,T] the draft's
    probability of every drafted token, q_rows [B,T,V] its distributions (device f32); logits: what
    sd_lmhead_stats_logits kept, or None (the stop rows then go through the LM head once more)."""
    M, Hd, V = _lm_sizes(hidden, W)
    assert M == batch.B * batch.T_max
    assert tuple(q_rows.shape) == (batch.B, batch.T_max, V) and q_rows.dtype == torch.float32 and q_rows.is_contiguous()
    _check(_n.sd_accept_chain_sampled(_at(batch.c), hidden, W, Hd, V, inv_temp, lse, logits, draft_tok, q_tok, q_rows,
                                      u, w, n_acc, path, out_tok, new_len, workspace, workspace, status, stream))


def sd_lmhead_accept_sampled_compact(batch: Batch, hidden, W, inv_temp: float, draft_tok, u, w, layers: LayerSet,
                                     lse, group_stats, n_acc, path, out_tok, new_len, workspace, status,
                                     stream=None) -> None:
    """LM-head statistics, acceptance at a sampling temperature and KV compaction in all layers: the
    LM-head tiles and one tail kernel."""
    M, Hd, V = _lm_sizes(hidden, W)
    assert M == batch.B * batch.T_max
    _check(_n.sd_lmhead_accept_sampled_compact(_at(batch.c), hidden, W, Hd, V, inv_temp, draft_tok, u, w,
                                               _at(layers.layers), layers.L, _at(layers.kt), _at(layers.vt), lse,
                                               group_stats, n_acc, path, out_tok, new_len, workspace, workspace,
                                               status, stream))


def sd_draft_feature_attention(qp, k, v, H: int, scale: float, out, stream=None) -> None:
    """Meta-query cross-attention core: qp [Q,D], k and v [S,L,D], out [S,Q,D]; D = H * 128."""
    Q, D = qp.shape
    S, L, _ = k.shape
    _check(_n.sd_draft_feature_attention(qp, k, v, S, L, Q, H, D, scale, out, stream))


# ------------------------------------------------------------------ rows of logits
_DTYPES = {torch.float32: SD_F32, torch.bfloat16: SD_BF16}


def _rows(t):
    """(address, dtype, row stride, rows, columns) of a matrix of logits; rows may lie further apart than they are long."""
    M, V = t.shape
    assert t.is_cuda and t.dtype in _DTYPES, "logits are float32 or bfloat16 CUDA tensors"
    assert t.get_device() == torch.cuda.current_device(), "logits lie on another device than the current one"
    ld = t.stride(0) if M > 1 else max(t.stride(0), V)
    assert (t.stride(1) == 1 or V == 1) and ld >= V, "a row's logits must be contiguous, rows must not overlap"
    return t.data_ptr(), _DTYPES[t.dtype], ld, M, V


def _shaped(t, shape, dtype=torch.float32):
    if t is not None:
        assert t.shape == shape and t.dtype == dtype, f"expected {dtype} {shape}, got {t.dtype} {tuple(t.shape)}"


def _raw_stream(stream) -> int:
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()) if stream is None else int(getattr(stream, "cuda_stream", stream))


def stream_of(stream) -> "torch.cuda.Stream":
    """The stream behind an argument, a torch stream or a handle (0: the default stream)."""
    raw = _raw_stream(stream)
    return torch.cuda.ExternalStream(raw) if raw else torch.cuda.default_stream()


class Sampling:
    """Owns the per-row arrays named by the C struct ``sd_sampling`` (each a sequence or tensor of M values, or None).  Arrays that are
    made here, on the current stream, are ready for calls on any other; a tensor that can be taken as it is stays the caller's."""

    def __init__(self, inv_temp=None, top_k=None, top_p=None, min_p=None, device="cuda"):
        self._made, self._event = [], None

        def to(a, t):
            if a is None:
                return None
            got = torch.as_tensor(a, dtype=t).contiguous().to(torch.device(device))
            if got is not a:
                self._made.append(got)
                self._event = self._event or (torch.cuda.Event() if torch.is_tensor(a) and a.is_cuda else None)
            return got
        self.inv_temp, self.top_p, self.min_p = to(inv_temp, torch.float32), to(top_p, torch.float32), to(min_p, torch.float32)
        self.top_k = to(top_k, torch.int32)
        have = [t for t in (self.inv_temp, self.top_k, self.top_p, self.min_p) if t is not None]
        assert all(t.dim() == 1 and t.shape == have[0].shape for t in have), "one value per row in each array"
        self.M = have[0].numel() if have else None
        self._streams = {_raw_stream(None)} if self._made and self._made[0].is_cuda else set()
        if self._event is not None:
            self._event.record()
        self.c = sd_sampling(_ptr(self.inv_temp), _ptr(self.top_k), _ptr(self.top_p), _ptr(self.min_p))

    def on(self, stream) -> int:
        """The struct's address for a call on `stream` (None: the current one)."""
        raw = _raw_stream(stream) if self._made else None
        if raw is not None and raw not in self._streams:
            self._streams.add(raw)
            other = stream_of(raw)
            with torch.cuda.stream(other):
                if self._event is not None and not torch.cuda.is_current_stream_capturing():       # (a capture begins behind a synchronisation)
                    other.wait_event(self._event)
            for t in self._made:
                t.record_stream(other)
        return _at(self.c)

    def for_nodes(self, batch: Batch) -> "Sampling":
        """The same for the B * T_max rows of a batch: rows that no node uses count as masked, and nothing is reported of them."""
        assert self.M is None or self.M == batch.B * batch.T_max, "one set of sampling parameters per row"
        of = copy.copy(self)
        of.batch = batch
        of.c = sd_sampling(self.c.inv_temp, self.c.top_k, self.c.top_p, self.c.min_p, _ptr(batch.n_nodes), batch.T_max)
        return of


def sd_top_logits(logits, inv_temp: float, values, index, lse, status, stream=None) -> None:
    """The K first entries of every row of logits [M,V] (values, index [M,K]) and lse [M] (or None) at inv_temp."""
    x, dtype, ld, M, V = _rows(logits)
    K = values.size(1)
    _shaped(values, (M, K))
    _shaped(index, (M, K), torch.int32)
    _shaped(lse, (M,))
    _check(_n.sd_top_logits(x, dtype, ld, M, V, K, inv_temp, values, index, lse, status, stream))


def sd_sample_logits(logits, how: Sampling, u, tokens, prob, probs, lse, status, stream=None) -> None:
    """N tokens per row drawn with the uniforms u [M,N]: tokens [M,N], their probabilities prob [M,N] (or None), the filtered
    distributions probs [M,V] (or None) and the log of the mass that stays, lse [M] (or None)."""
    x, dtype, ld, M, V = _rows(logits)
    N = u.size(1)
    assert how.M is None or how.M == M, "one set of sampling parameters per row"
    _shaped(u, (M, N))
    _shaped(tokens, (M, N), torch.int32)
    _shaped(prob, (M, N))
    _shaped(probs, (M, V))
    _shaped(lse, (M,))
    _check(_n.sd_sample_logits(x, dtype, ld, M, V, how.on(stream), u, N, tokens, prob, probs, lse, status, stream))


def sd_filter_logits(logits, how: Sampling, out, lse, kept, status, stream=None) -> None:
    """out [M,V] (f32; may be f32 logits themselves) = logits * inv_temp where the filters let them stay, minus infinity elsewhere; lse [M];
    kept [M] (or None).  sd_accept_tree_sampled_q and sd_accept_chain_sampled take out and lse with inv_temp = 1."""
    x, dtype, ld, M, V = _rows(logits)
    assert how.M is None or how.M == M, "one set of sampling parameters per row"
    _shaped(out, (M, V))
    _shaped(lse, (M,))
    _shaped(kept, (M,), torch.int32)
    _check(_n.sd_filter_logits(x, dtype, ld, M, V, how.on(stream), out, lse, kept, status, stream))


def _distill_args(logits, top_val, top_idx, top_lse, label, dloss, grad, stats):
    x, dtype, ld, M, V = _rows(logits)
    K = top_val.size(1)
    _shaped(top_val, (M, K))
    _shaped(top_idx, (M, K), torch.int32)
    _shaped(top_lse, (M,))
    _shaped(label, (M,), torch.int32)
    _shaped(dloss, (M,))
    _shaped(stats, (M, 4))
    g, g_ld = None, V
    if grad is not None:
        g, g_dtype, g_ld, g_M, g_V = _rows(grad)
        assert (g_dtype, g_M, g_V) == (dtype, M, V), "the gradient has the logits' type and shape"
    return x, dtype, ld, M, V, K, g, g_ld


def sd_distill_loss(logits, top_val, top_idx, top_lse, label, inv_temp: float, kl_weight: float, ce_weight: float, kl, ce, stats,
                    dloss, grad, status, stream=None) -> None:
    """KL from the target's first logits (top_val, top_idx [M,K], top_lse [M] or None: sd_top_logits) to the student's rows, kl [M], and
    cross-entropy with label [M] (or None), ce [M].  With grad (the logits' type and shape, or the logits themselves): the gradient of
    sum_r dloss[r] (kl_weight kl[r] + ce_weight ce[r]) too.  stats [M,4] (or None): for sd_distill_grad."""
    x, dtype, ld, M, V, K, g, g_ld = _distill_args(logits, top_val, top_idx, top_lse, label, dloss, grad, stats)
    _shaped(kl, (M,))
    _shaped(ce, (M,))
    _check(_n.sd_distill_loss(x, dtype, ld, M, V, top_val, top_idx, K, top_lse, label, inv_temp, kl_weight, ce_weight, kl, ce, stats,
                              dloss, g, g_ld, status, stream))


def sd_distill_grad(logits, top_val, top_idx, top_lse, label, inv_temp: float, kl_weight: float, ce_weight: float, stats, dloss, grad,
                    status, stream=None) -> None:
    """The gradient of sd_distill_loss in a call of its own, from the stats that it left."""
    x, dtype, ld, M, V, K, g, g_ld = _distill_args(logits, top_val, top_idx, top_lse, label, dloss, grad, stats)
    _check(_n.sd_distill_grad(x, dtype, ld, M, V, top_val, top_idx, K, top_lse, label, inv_temp, kl_weight, ce_weight, stats, dloss,
                              g, g_ld, status, stream))


# ------------------------------------------------------------------ packed new tokens
_here = torch._C._cuda_getDevice           # (torch.cuda.current_device() takes 0.4 us, a tenth of a small call)
_BF16 = (torch.bfloat16, torch.int16, torch.uint16)


def _ints(t, n, what, here=None):
    """A contiguous int32 tensor of shape n on the current device."""
    if t.dtype is not torch.int32 or t.shape != n or not t.is_contiguous() or t.get_device() != (_here() if here is None else here):
        raise AssertionError(f"{what}: expected a contiguous int32 tensor {n} on the current device, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t


def _heads(t, rows, heads, what, here):
    """(address, row stride) of bf16 rows of heads [rows, heads, 128]; rows may lie further apart (a view of a projection's output)."""
    if t.dtype not in _BF16 or t.shape != (rows, heads, 128) or t.get_device() != here:
        raise AssertionError(f"{what}: expected bf16 {(rows, heads, 128)} on the current device, got {t.dtype} {tuple(t.shape)} on {t.device}")
    ld, between, one = t.stride()
    if rows < 2:
        ld = heads * 128
    if one != 1 or (heads > 1 and between != 128) or ld < heads * 128:
        raise AssertionError(f"{what}: the heads of a row must be contiguous, rows must not overlap (strides {t.stride()})")
    return t.data_ptr(), ld


class _OnAnyStream:
    """The arrays that an object makes, on the current stream, are ready for calls on any other and outlive them."""

    def _makes(self, *tensors):
        self._made = [t for t in tensors if t is not None]
        self._streams = set()
        self._device = _here()                             # (where its arrays lie: _ints)
        if self._made:
            self._streams.add(torch._C._cuda_getCurrentRawStream(_here()))
            self._event = None
            if not torch.cuda.is_current_stream_capturing():                   # (nothing outside of a capture can wait for an event in it)
                self._event = torch.cuda.Event()
                self._event.record()

    def _ready(self, stream) -> None:
        """In front of a call on `stream` (None: the current one)."""
        here = _here()
        if here != self._device:
            raise AssertionError(f"arrays on device {self._device}, the current one is {here}")
        if self._made:
            raw = torch._C._cuda_getCurrentRawStream(here) if stream is None else _raw_stream(stream)
            if raw not in self._streams:
                self._streams.add(raw)
                other = stream_of(raw)
                with torch.cuda.stream(other):
                    if self._event is not None and not torch.cuda.is_current_stream_capturing():       # (a capture begins behind a synchronisation)
                        other.wait_event(self._event)
                for t in self._made:
                    t.record_stream(other)

    def on(self, stream) -> int:
        """The struct's address for a call on `stream`."""
        self._ready(stream)
        return _at(self.c)


class BlockPool(_OnAnyStream):
    """Owns the arrays named by the C struct ``sd_block_pool``: all blocks free, block 0 on top, or the caller's own stack."""

    def __init__(self, num_blocks: int, free_blocks: Optional[torch.Tensor] = None, n_free: Optional[torch.Tensor] = None, device="cuda"):
        self.num_blocks = int(num_blocks)
        own = free_blocks is None
        if own:
            free_blocks = torch.arange(self.num_blocks - 1, -1, -1, dtype=torch.int32, device=device)
            n_free = torch.full((1,), self.num_blocks, dtype=torch.int32, device=device)
        self.free_blocks = _ints(free_blocks, (self.num_blocks,), "free_blocks")
        self.n_free = _ints(n_free, (1,), "n_free")
        self.c = sd_block_pool(self.free_blocks.data_ptr(), self.n_free.data_ptr(), self.num_blocks)
        self._makes(*((self.free_blocks, self.n_free) if own else ()))


def sd_assign_blocks(pool: BlockPool, block_table, n_blocks, lens, n_new, granted, status, stream=None) -> None:
    """Makes the tables [B, max_blocks] cover lens + n_new tokens (each [B]): n_blocks [B] and the pool are brought up to date,
    granted [B] (or None) is 0 for requests that the pool did not suffice for."""
    B, W = block_table.shape
    here, n = _here(), (B,)
    _ints(block_table, (B, W), "block_table", here)
    _ints(n_blocks, n, "n_blocks", here)
    _ints(lens, n, "lens", here)
    _ints(n_new, n, "n_new", here)
    if granted is not None:
        _ints(granted, n, "granted", here)
    _check(_n.sd_assign_blocks(pool.on(stream), B, W, block_table, n_blocks, lens, n_new, granted, status, stream))


class Prompts(_OnAnyStream):
    """New tokens of B requests in N packed rows: owns the arrays named by the C struct ``sd_prompts``.  Tensors that are int32 on
    the device are taken as they are and may change between calls (sd_prompt_prepare then comes again); others are copied there."""

    def __init__(self, N, Hq, Hkv, D, block_table, lens, n_new, n_blocks=None, *, num_blocks, block_size=64, device="cuda"):
        dev, made = torch.device(device), []

        def to(a):
            if isinstance(a, torch.Tensor) and a.is_cuda and a.dtype is torch.int32 and not a.is_contiguous():
                raise AssertionError("int32 tensors on the device are taken as they are and have to be contiguous")
            got = torch.as_tensor(a, dtype=torch.int32).contiguous().to(dev)
            if got is not a:
                made.append(got)
            return got
        self.N, self.Hq, self.Hkv, self.D = int(N), int(Hq), int(Hkv), int(D)
        self.len, self.n_new = to(lens), to(n_new)
        self.B = int(self.len.numel())
        self.block_table = to(block_table)
        if self.block_table.dim() != 2 or self.block_table.shape[0] != self.B:
            raise AssertionError(f"block_table: expected [{self.B}, max_blocks], got {tuple(self.block_table.shape)}")
        self.n_blocks = None if n_blocks is None else to(n_blocks)
        self.max_blocks, self.num_blocks = int(self.block_table.shape[1]), int(num_blocks)
        for t in (self.len, self.n_new, self.n_blocks):
            if t is not None:
                _ints(t, (self.B,), "lens, n_new and n_blocks")
        rows = lambda n: torch.empty(max(n, 1), dtype=torch.int32, device=dev)[:n]
        self.c = sd_prompts(self.B, self.N, self.Hq, self.Hkv, self.D, int(block_size), self.max_blocks, self.num_blocks,
                            self.block_table.data_ptr(), _ptr(self.n_blocks), self.len.data_ptr(), self.n_new.data_ptr())
        self.plan = torch.empty(max(int(lib.sd_prompt_plan_bytes(self.ref())), 16), dtype=torch.uint8, device=dev)
        self.c.plan = self.plan.data_ptr()
        own = rows(self.B + 1), rows(self.N), rows(self.N)
        self.use(*own)
        self._makes(self.plan, *own, *made)

    def use(self, start, slot, position) -> "Prompts":
        """Puts what sd_prompt_prepare makes into the caller's arrays: start [B + 1], slot and position [N]."""
        self.start, self.slot, self.position = (_ints(t, (n,), "start, slot and position") for t, n in
                                                ((start, self.B + 1), (slot, self.N), (position, self.N)))
        at = lambda t, other: t.data_ptr() or other.data_ptr()                   # (an empty tensor has no address)
        self.c.start, self.c.slot, self.c.position = start.data_ptr(), at(slot, start), at(position, start)
        return self

    def ref(self):
        return C.byref(self.c)


def sd_prompt_plan_bytes(prompts: Prompts) -> int:
    return int(lib.sd_prompt_plan_bytes(prompts.ref()))


def sd_prompt_workspace_bytes(prompts: Prompts) -> int:
    return int(lib.sd_prompt_workspace_bytes(prompts.ref()))


def sd_prompt_prepare(prompts: Prompts, status, stream=None) -> None:
    """First rows, slots and positions of the packed tokens, and the plan of their attention; once for all layers of a step."""
    _check(_n.sd_prompt_prepare(prompts.on(stream), status, stream))


def sd_append_kv(prompts: Prompts, cache: sd_kv_layer, k, v, status, stream=None) -> None:
    """K and V of the packed tokens, [N, Hkv, 128] each (rows may be strided), into one layer's cache."""
    here = _here()
    k, ldk = _heads(k, prompts.N, prompts.Hkv, "k", here)
    v, ldv = _heads(v, prompts.N, prompts.Hkv, "v", here)
    _check(_n.sd_append_kv(prompts.on(stream), _at(cache), k, ldk, v, ldv, status, stream))


def sd_prompt_attention(prompts: Prompts, cache: sd_kv_layer, q, scale: float, out, lse, workspace, status, stream=None) -> None:
    """Causal attention of the packed tokens over one layer's cache, which holds their own K and V: q, out [N, Hq, 128] (rows may be
    strided), lse [N, Hq] f32 or None."""
    here = _here()
    q, ldq = _heads(q, prompts.N, prompts.Hq, "q", here)
    out, ldo = _heads(out, prompts.N, prompts.Hq, "out", here)
    _shaped(lse, (prompts.N, prompts.Hq))
    _check(_n.sd_prompt_attention(prompts.on(stream), _at(cache), q, ldq, scale, out, ldo, lse, workspace, workspace, status, stream))
