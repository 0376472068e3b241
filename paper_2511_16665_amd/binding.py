"""Thin ctypes binding of libtlt.so: same names as the C ABI, argument marshalling only.

torch is used for device memory and streams; every step of the path runs in the library's HIP
kernels.  There is no CPU fallback: loading fails loudly when the library has not been built
(`python -m paper_2511_16665_amd.build`).
"""
from __future__ import annotations

import ctypes as C
import dataclasses
import os
from typing import Optional

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtlt.so")

TLT_F32, TLT_BF16 = 0, 1
ERRORS = {0: "TLT_OK", -1: "TLT_EINVAL", -2: "TLT_ESHAPE", -3: "TLT_ENOPAGES", -4: "TLT_EHIP", -5: "TLT_ENOTIMPL",
          -6: "TLT_ESYNC"}

EXPORTS = [
    "tlt_strerror", "tlt_last_hip_error", "tlt_workspace_bytes", "tlt_create", "tlt_destroy", "tlt_draft_expand",
    "tlt_tree_finalize", "tlt_verify_forward", "tlt_accept", "tlt_kv_commit", "tlt_gemm", "tlt_set_attention_impl",
    "tlt_profile_begin", "tlt_profile_read", "tlt_mab_create", "tlt_mab_destroy", "tlt_mab_select", "tlt_mab_record",
    "tlt_mab_median_reward", "tlt_ngram_create", "tlt_ngram_destroy", "tlt_ngram_insert", "tlt_ngram_propose",
    "tlt_template_build", "tlt_draft_sample", "tlt_gemm_argmax", "tlt_gemm_glu", "tlt_gemm_parts", "tlt_draft_pool", "tlt_set_oproj_rounding", "tlt_device_status", "tlt_accept_sample_static", "tlt_attention", "tlt_attention_workspace_bytes",
    "tlt_graph_pool_create", "tlt_graph_pool_destroy", "tlt_graph_pool_step", "tlt_graph_pool_count", "tlt_mfma_stream", "tlt_prefill", "tlt_step_report",
    "tlt_kv8_write", "tlt_kv8_attention", "tlt_kv8_attention_workspace_bytes", "tlt_kv8_commit", "tlt_kv8_read",
    "tlt_pages_grow", "tlt_pages_release", "tlt_rope_freqs", "tlt_rope_write", "tlt_sample", "tlt_sample_filter", "tlt_sample_workspace_bytes",
]


class TltError(RuntimeError):
    def __init__(self, code, where, hip=0):
        self.code = code
        super().__init__(f"{where}: {ERRORS.get(code, code)}" + (f" (hipError {hip})" if hip else ""))


class ModelCfgC(C.Structure):
    _fields_ = [(k, C.c_int32) for k in ("n_layers", "hidden", "n_q_heads", "n_kv_heads", "head_dim", "mlp", "vocab")] + \
        [("rms_eps", C.c_float), ("rope_theta", C.c_float), ("dtype", C.c_int32), ("page_size", C.c_int32)]


class LayerWeightsC(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in ("attn_norm", "wqkv", "wo", "mlp_norm", "wg", "wu", "wd", "bqkv")]


class WeightsC(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("lm_head", C.c_void_p), ("final_norm", C.c_void_p),
                ("layers", C.POINTER(LayerWeightsC)), ("fc", C.c_void_p)]


class StrategyC(C.Structure):
    _fields_ = [("draft_depth", C.c_int32), ("topk", C.c_int32), ("tokens_to_verify", C.c_int32)]


class KVC(C.Structure):
    _fields_ = [("k_pool", C.c_void_p), ("v_pool", C.c_void_p), ("n_pages", C.c_int64), ("block_table", C.c_void_p),
                ("seq_len", C.c_void_p), ("max_pages", C.c_int32), ("seq_len_bound", C.c_int32)]


class KV8C(C.Structure):
    _fields_ = [("k_pool", C.c_void_p), ("v_pool", C.c_void_p), ("k_exp", C.c_void_p), ("v_exp", C.c_void_p), ("n_pages", C.c_int64),
                ("block_table", C.c_void_p), ("seq_len", C.c_void_p), ("max_pages", C.c_int32), ("seq_len_bound", C.c_int32)]


class PagesC(C.Structure):
    _fields_ = [("free_page", C.c_void_p), ("n_free", C.c_void_p), ("page_count", C.c_void_p), ("block_table", C.c_void_p), ("n_pages", C.c_int64),
                ("max_pages", C.c_int32), ("page_size", C.c_int32)]


class RopeC(C.Structure):
    _fields_ = [("freq", C.c_void_p), ("rot_dim", C.c_int32), ("layout", C.c_int32), ("amplitude", C.c_float)]


class FilterC(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in ("temperature", "top_k", "top_p", "min_p")]


class TreeC(C.Structure):
    _fields_ = [("token", C.c_void_p), ("parent", C.c_void_p), ("depth", C.c_void_p), ("anc_mask", C.c_void_p),
                ("score", C.c_void_p), ("n", C.c_int32)]


class StepArgsC(C.Structure):
    _fields_ = [("new_tokens", C.c_void_p), ("new_src", C.c_void_p), ("n_new", C.c_void_p), ("new_stride", C.c_int32),
                ("hidden", C.c_void_p), ("hidden_n", C.c_int32), ("draft_kv", C.POINTER(KVC)), ("tree", C.POINTER(TreeC)),
                ("kv", C.POINTER(KVC)), ("argmax", C.c_void_p), ("hidden_out", C.c_void_p), ("stride", C.c_int32),
                ("accept_len", C.c_void_p), ("path_idx", C.c_void_p), ("out_tokens", C.c_void_p), ("n_out", C.c_void_p)]


_lib = None


def load() -> C.CDLL:
    """Loads libtlt.so; raises if it is missing (no fallback path exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} not found: build it with `python -m paper_2511_16665_amd.build`")
    lib = C.CDLL(LIB_PATH)
    lib.tlt_strerror.restype = C.c_char_p
    lib.tlt_workspace_bytes.restype = C.c_size_t
    lib.tlt_workspace_bytes.argtypes = [C.POINTER(ModelCfgC)] + [C.c_int] * 5
    lib.tlt_create.argtypes = [C.POINTER(C.c_void_p), C.POINTER(ModelCfgC), C.POINTER(WeightsC), C.POINTER(WeightsC)] + \
        [C.c_int] * 5 + [C.c_void_p, C.c_size_t]
    lib.tlt_destroy.argtypes = [C.c_void_p]
    lib.tlt_last_hip_error.argtypes = [C.c_void_p]
    lib.tlt_draft_expand.argtypes = [C.c_void_p, C.c_void_p] + [C.c_int] * 5 + [C.c_void_p] * 3 + [C.c_int, C.c_void_p, C.c_int,
                                                                                         C.c_void_p, C.POINTER(KVC),
                                                                                         C.POINTER(TreeC)]
    lib.tlt_prefill.argtypes = [C.c_void_p, C.c_void_p] + [C.c_int] * 3 + [C.c_void_p, C.c_int, C.POINTER(KVC), C.POINTER(KVC)]
    lib.tlt_draft_pool.argtypes = [C.c_void_p, C.c_void_p] + [C.c_int] * 3 + [C.c_void_p] * 3
    lib.tlt_template_build.argtypes = [C.c_int] * 3 + [C.POINTER(C.c_int32)] * 4
    lib.tlt_draft_sample.argtypes = [C.c_void_p, C.c_void_p] + [C.c_int] * 4 + [C.c_float] + [C.c_void_p] * 3 + \
        [C.c_int, C.c_void_p, C.c_int, C.c_void_p, C.POINTER(KVC), C.c_void_p, C.POINTER(TreeC), C.c_void_p]
    lib.tlt_tree_finalize.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.POINTER(TreeC)]
    lib.tlt_graph_pool_create.argtypes = [C.c_void_p, C.POINTER(C.c_int32), C.c_int, C.c_int, C.POINTER(C.c_void_p)]
    lib.tlt_graph_pool_destroy.argtypes = [C.c_void_p]
    lib.tlt_graph_pool_step.argtypes = [C.c_void_p, C.c_void_p] + [C.c_int] * 4 + [C.POINTER(StepArgsC)]
    lib.tlt_graph_pool_count.argtypes = [C.c_void_p, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
    lib.tlt_verify_forward.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.POINTER(TreeC), C.POINTER(KVC)] + [C.c_void_p] * 4
    lib.tlt_accept.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_float, C.POINTER(TreeC)] + [C.c_void_p] * 5 + \
        [C.c_int] + [C.c_void_p] * 4
    lib.tlt_accept_sample_static.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_float, C.POINTER(TreeC)] + [C.c_void_p] * 4 + \
        [C.c_int] + [C.c_void_p] * 5
    lib.tlt_kv_commit.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.POINTER(KVC), C.c_void_p, C.c_void_p, C.c_int]
    lib.tlt_gemm.argtypes = [C.c_void_p] + [C.c_int] * 5 + [C.c_void_p] * 3
    lib.tlt_gemm_glu.argtypes = [C.c_void_p] + [C.c_int] * 3 + [C.c_void_p] * 4
    lib.tlt_gemm_parts.argtypes = [C.c_void_p] + [C.c_int] * 3 + [C.c_void_p] * 3 + [C.c_size_t, C.POINTER(C.c_int)]
    lib.tlt_gemm_argmax.argtypes = [C.c_void_p] + [C.c_int] * 3 + [C.c_void_p] * 3 + [C.c_size_t, C.c_void_p]
    lib.tlt_mfma_stream.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int]
    lib.tlt_set_attention_impl.argtypes = [C.c_void_p, C.c_int]
    lib.tlt_attention_workspace_bytes.restype = C.c_size_t
    lib.tlt_attention_workspace_bytes.argtypes = [C.c_int] * 6
    lib.tlt_attention.argtypes = [C.c_void_p] + [C.c_int] * 7 + [C.c_void_p, C.c_void_p, C.POINTER(KVC), C.c_void_p, C.c_void_p,
                                                               C.c_size_t, C.c_int]
    lib.tlt_kv8_write.argtypes = [C.c_void_p] + [C.c_int] * 7 + [C.c_float] + [C.c_void_p] * 3 + [C.POINTER(KV8C), C.c_void_p, C.c_int64]
    lib.tlt_kv8_attention_workspace_bytes.restype = C.c_size_t
    lib.tlt_kv8_attention_workspace_bytes.argtypes = [C.c_int] * 6
    lib.tlt_pages_grow.argtypes = [C.c_void_p, C.c_int, C.POINTER(PagesC)] + [C.c_void_p] * 3 + [C.c_int] + [C.c_void_p] * 5
    lib.tlt_pages_release.argtypes = [C.c_void_p, C.c_int, C.POINTER(PagesC), C.c_void_p]
    lib.tlt_rope_freqs.argtypes = [C.c_int] * 2 + [C.c_double] * 5 + [C.c_void_p, C.POINTER(C.c_float)]
    lib.tlt_rope_write.argtypes = [C.c_void_p] + [C.c_int] * 6 + [C.POINTER(RopeC), C.c_void_p, C.c_int64] + [C.c_void_p] * 3 + \
        [C.POINTER(KVC), C.POINTER(KV8C), C.c_void_p, C.c_int64, C.c_void_p, C.c_int64]
    lib.tlt_sample_workspace_bytes.restype = C.c_size_t
    lib.tlt_sample_workspace_bytes.argtypes = [C.c_int] * 2
    lib.tlt_sample.argtypes = [C.c_void_p] + [C.c_int] * 4 + [C.c_void_p, C.c_int64, C.POINTER(FilterC)] + [C.c_void_p] * 5 + [C.c_size_t]
    lib.tlt_sample_filter.argtypes = [C.c_void_p] + [C.c_int] * 4 + [C.c_void_p, C.c_int64, C.POINTER(FilterC), C.c_void_p, C.c_int64] + [C.c_void_p] * 2 + [C.c_size_t]
    lib.tlt_kv8_attention.argtypes = [C.c_void_p] + [C.c_int] * 7 + [C.c_void_p, C.c_int64, C.c_void_p, C.POINTER(KV8C), C.c_void_p, C.c_void_p,
                                                                   C.c_size_t, C.c_int]
    lib.tlt_kv8_commit.argtypes = [C.c_void_p] + [C.c_int] * 5 + [C.POINTER(KV8C), C.c_void_p, C.c_void_p, C.c_int]
    lib.tlt_kv8_read.argtypes = [C.c_void_p] + [C.c_int] * 7 + [C.POINTER(KV8C)] + [C.c_void_p] * 4
    lib.tlt_set_oproj_rounding.argtypes = [C.c_void_p, C.c_int]
    lib.tlt_device_status.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(C.c_uint32)]
    lib.tlt_step_report.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.POINTER(C.c_uint32)]
    lib.tlt_profile_begin.argtypes = [C.c_void_p, C.c_int]
    lib.tlt_profile_read.argtypes = [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_int64), C.POINTER(C.c_double),
                                     C.POINTER(C.c_double)]
    lib.tlt_mab_create.argtypes = [C.POINTER(StrategyC), C.c_int, C.POINTER(C.c_int32), C.c_int, C.c_double, C.c_int, C.c_int,
                                   C.POINTER(C.c_void_p)]
    lib.tlt_mab_destroy.argtypes = [C.c_void_p]
    lib.tlt_mab_destroy.restype = None
    lib.tlt_mab_select.argtypes = [C.c_void_p, C.c_int, C.c_uint32, C.c_uint32, C.POINTER(C.c_int32)]
    lib.tlt_mab_record.argtypes = [C.c_void_p, C.c_int, C.c_double, C.POINTER(C.c_int32), C.c_int, C.POINTER(C.c_double),
                                   C.POINTER(C.c_double)]
    lib.tlt_mab_median_reward.argtypes = [C.c_void_p, C.c_int, C.POINTER(C.c_double), C.POINTER(C.c_int32)]
    lib.tlt_ngram_create.argtypes = [C.c_int, C.POINTER(C.c_void_p)]
    lib.tlt_ngram_destroy.argtypes = [C.c_void_p]
    lib.tlt_ngram_destroy.restype = None
    lib.tlt_ngram_insert.argtypes = [C.c_void_p, C.c_int64, C.POINTER(C.c_int32), C.c_int]
    lib.tlt_ngram_propose.argtypes = [C.c_void_p, C.c_int64, C.POINTER(C.c_int32), C.c_int, C.c_int, C.c_int, C.c_int,
                                      C.POINTER(C.c_int32), C.POINTER(C.c_int32), C.POINTER(C.c_float)]
    _lib = lib
    return lib


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device tensors must be contiguous CUDA/HIP tensors"
    return C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def torch_dtype(dtype_code: int):
    return torch.float32 if dtype_code == TLT_F32 else torch.bfloat16


@dataclasses.dataclass
class KV:
    """Paged KV cache of one model: pools [L, n_pages, Hkv, page, d], block_table [B, max_pages] int32,
    seq_len [B] int32 (device), seq_len_bound = host-known upper bound of seq_len."""
    k_pool: torch.Tensor
    v_pool: torch.Tensor
    block_table: torch.Tensor
    seq_len: torch.Tensor
    seq_len_bound: int

    def c(self) -> KVC:
        assert self.block_table.dtype == torch.int32 and self.seq_len.dtype == torch.int32
        return KVC(_ptr(self.k_pool), _ptr(self.v_pool), self.k_pool.shape[1], _ptr(self.block_table), _ptr(self.seq_len),
                   self.block_table.shape[1], int(self.seq_len_bound))


@dataclasses.dataclass
class Tree:
    """Token tree, device tensors [B, n]: token/parent/depth int32, anc_mask int64 (bit pattern), score fp32."""
    token: torch.Tensor
    parent: torch.Tensor
    depth: torch.Tensor
    anc_mask: torch.Tensor
    score: torch.Tensor

    @staticmethod
    def empty(B: int, n: int, device="cuda") -> "Tree":
        i32 = lambda: torch.zeros((B, n), dtype=torch.int32, device=device)
        return Tree(i32(), i32(), i32(), torch.zeros((B, n), dtype=torch.int64, device=device),
                    torch.zeros((B, n), dtype=torch.float32, device=device))

    @property
    def n(self) -> int:
        return self.token.shape[1]

    def c(self) -> TreeC:
        return TreeC(_ptr(self.token), _ptr(self.parent), _ptr(self.depth), _ptr(self.anc_mask), _ptr(self.score), self.n)


def _weights_c(w: dict, n_layers: int, fc=None, keep=None):
    layers = (LayerWeightsC * n_layers)()
    src = w["layers"] if "layers" in w else [w["layer"]]
    for i in range(n_layers):
        for k, _ in LayerWeightsC._fields_:
            if k in src[i]:                 # (bqkv is optional: a missing entry stays NULL)
                setattr(layers[i], k, src[i][k].data_ptr())
    keep.append(layers)
    return layers


class Context:
    """tlt_create / tlt_destroy plus the step's calls as methods with the C names."""

    def __init__(self, cfg, dtype_code: int, target: dict, draft: Optional[dict], max_batch: int, max_n: int,
                 max_depth: int, max_topk: int, max_ctx: int):
        lib = load()
        self.lib = lib
        self.cfg = cfg
        self.dtype_code = dtype_code
        self.ccfg = ModelCfgC(cfg.n_layers, cfg.hidden, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, cfg.mlp, cfg.vocab,
                              cfg.rms_eps, cfg.rope_theta, dtype_code, cfg.page_size)
        nbytes = lib.tlt_workspace_bytes(C.byref(self.ccfg), max_batch, max_n, max_depth, max_topk, max_ctx)
        if nbytes == 0:
            raise TltError(-1, "tlt_workspace_bytes")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        self._keep = [target, draft]
        tl = _weights_c(target, cfg.n_layers, keep=self._keep)
        tw = WeightsC(target["embed"].data_ptr(), target["lm_head"].data_ptr(), target["final_norm"].data_ptr(), tl, None)
        dw_ref = None
        if draft is not None:
            dl = _weights_c(draft, 1, keep=self._keep)
            dw = WeightsC(target["embed"].data_ptr(), target["lm_head"].data_ptr(), target["final_norm"].data_ptr(), dl,
                          draft["fc"].data_ptr())
            dw_ref = C.byref(dw)
        self.handle = C.c_void_p()
        rc = lib.tlt_create(C.byref(self.handle), C.byref(self.ccfg), C.byref(tw), dw_ref, max_batch, max_n, max_depth,
                            max_topk, max_ctx, _ptr(self.workspace), nbytes)
        if rc:
            raise TltError(rc, "tlt_create")

    def close(self):
        if self.handle:
            torch.cuda.synchronize()
            self.lib.tlt_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc, where):
        if rc:
            raise TltError(rc, where, self.lib.tlt_last_hip_error(self.handle))

    def draft_expand(self, B, depth, topk, n_verify, new_tokens, new_src, n_new, hidden, root_tokens, draft_kv: KV,
                     out_tree: Optional[Tree], mode=0):
        new_stride = 0 if new_tokens is None else new_tokens.shape[1]
        hidden_n = 0 if hidden is None else hidden.shape[1]
        kvc = draft_kv.c()
        tree_ref = None
        if out_tree is not None:
            tc = out_tree.c()
            tree_ref = C.byref(tc)
        self._check(self.lib.tlt_draft_expand(self.handle, _stream(), B, depth, topk, n_verify, mode, _ptr(new_tokens),
                                              _ptr(new_src), _ptr(n_new), new_stride, _ptr(hidden), hidden_n,
                                              _ptr(root_tokens), C.byref(kvc), tree_ref), "tlt_draft_expand")

    def prefill(self, B, n_tokens, chunk, tokens, kv: KV, draft_kv: KV) -> bool:
        """tokens [B, > n_tokens] int32 (device).  False: this context takes such prompts chunk by chunk only (nothing was done)."""
        kvc, dkvc = kv.c(), draft_kv.c()
        rc = self.lib.tlt_prefill(self.handle, _stream(), B, n_tokens, chunk, _ptr(tokens), tokens.shape[1], C.byref(kvc),
                                  C.byref(dkvc))
        if rc == -5:   # TLT_ENOTIMPL
            return False
        self._check(rc, "tlt_prefill")
        return True

    def draft_pool(self, B, depth, topk):
        """(token, parent, score) device tensors [B, topk + (depth-1)*topk^2] of the last expansion's pool."""
        n = topk + (depth - 1) * topk * topk
        token, parent = (torch.empty((B, n), dtype=torch.int32, device="cuda") for _ in range(2))
        score = torch.empty((B, n), dtype=torch.float32, device="cuda")
        self._check(self.lib.tlt_draft_pool(self.handle, _stream(), B, depth, topk, _ptr(token), _ptr(parent), _ptr(score)),
                    "tlt_draft_pool")
        return token, parent, score

    def draft_sample(self, B, depth, topk, n_verify, temperature, new_tokens, new_src, n_new, hidden, root_tokens,
                     draft_kv: KV, u_draw, out_tree: Tree, out_draft_q):
        new_stride = 0 if new_tokens is None else new_tokens.shape[1]
        hidden_n = 0 if hidden is None else hidden.shape[1]
        kvc, tc = draft_kv.c(), out_tree.c()
        self._check(self.lib.tlt_draft_sample(self.handle, _stream(), B, depth, topk, n_verify, temperature,
                                              _ptr(new_tokens), _ptr(new_src), _ptr(n_new), new_stride, _ptr(hidden),
                                              hidden_n, _ptr(root_tokens), C.byref(kvc), _ptr(u_draw), C.byref(tc),
                                              _ptr(out_draft_q)), "tlt_draft_sample")

    def tree_finalize(self, B, tree: Tree):
        tc = tree.c()
        self._check(self.lib.tlt_tree_finalize(self.handle, _stream(), B, C.byref(tc)), "tlt_tree_finalize")

    def verify_forward(self, B, tree: Tree, kv: KV, out_logits=None, out_argmax=None, out_hidden=None, out_lse=None):
        tc, kvc = tree.c(), kv.c()
        self._check(self.lib.tlt_verify_forward(self.handle, _stream(), B, C.byref(tc), C.byref(kvc), _ptr(out_logits),
                                                _ptr(out_argmax), _ptr(out_lse), _ptr(out_hidden)), "tlt_verify_forward")

    def accept(self, B, mode, temperature, tree: Tree, target_logits, target_argmax, draft_q, u_accept, u_final, stride,
               accept_len, path_idx, out_tokens, n_out):
        tc = tree.c()
        self._check(self.lib.tlt_accept(self.handle, _stream(), B, mode, temperature, C.byref(tc), _ptr(target_logits),
                                        _ptr(target_argmax), _ptr(draft_q), _ptr(u_accept), _ptr(u_final), stride,
                                        _ptr(accept_len), _ptr(path_idx), _ptr(out_tokens), _ptr(n_out)), "tlt_accept")

    def kv_commit(self, B, kv: KV, accept_len, path_idx, stride):
        kvc = kv.c()
        self._check(self.lib.tlt_kv_commit(self.handle, _stream(), B, C.byref(kvc), _ptr(accept_len), _ptr(path_idx), stride),
                    "tlt_kv_commit")

    def set_attention_impl(self, impl: int):
        self._check(self.lib.tlt_set_attention_impl(self.handle, impl), "tlt_set_attention_impl")

    def device_status(self, check=True):
        """Synchronises the current stream and returns the device-side status bits (cleared by the call);
        with check=True a raised bit becomes a TltError (TLT_ESHAPE / TLT_ESYNC)."""
        flags = C.c_uint32()
        rc = self.lib.tlt_device_status(self.handle, _stream(), C.byref(flags))
        if check:
            self._check(rc, "tlt_device_status")
        return flags.value

    def step_report(self, words: torch.Tensor, pinned: torch.Tensor) -> np.ndarray:
        """Synchronises the current stream and returns a copy of the int32 device tensor `words` (1-D), by way of `pinned` (pinned host
        int32, one element more); raises like device_status."""
        assert words.dtype == pinned.dtype == torch.int32 and pinned.is_pinned() and pinned.numel() > words.numel()
        flags = C.c_uint32()
        self._check(self.lib.tlt_step_report(self.handle, _stream(), _ptr(words), words.numel(), C.c_void_p(pinned.data_ptr()),
                                             C.byref(flags)), "tlt_step_report")
        return pinned.numpy()[: words.numel()].copy()

    def set_oproj_rounding(self, round_to_model_dtype: bool):
        self._check(self.lib.tlt_set_oproj_rounding(self.handle, int(round_to_model_dtype)), "tlt_set_oproj_rounding")

    def profile_begin(self, enable=True):
        """enable: True/1 = start afresh, 2 = resume without dropping records, False/0 = pause."""
        self._check(self.lib.tlt_profile_begin(self.handle, int(enable)), "tlt_profile_begin")

    def profile_read(self):
        ms, n, fl, by = (C.c_double * 6)(), (C.c_int64 * 6)(), (C.c_double * 6)(), (C.c_double * 6)()
        self._check(self.lib.tlt_profile_read(self.handle, ms, n, fl, by), "tlt_profile_read")
        names = ("gemm", "attention", "kv_commit", "other", "gemm_draft", "attention_draft")
        return {k: {"ms": ms[i], "launches": n[i], "flops": fl[i], "bytes": by[i]} for i, k in enumerate(names)}


def accept_sample_static(B, vocab, temperature, tree: Tree, target_logits, draft_q, u_accept, u_final, stride, accept_len,
                         path_idx, out_tokens, n_out, status=None):
    """tlt_accept_sample_static: sampling acceptance on the library's static scratch; returns the library's code."""
    tc = tree.c()
    return load().tlt_accept_sample_static(_stream(), B, vocab, temperature, C.byref(tc), _ptr(target_logits), _ptr(draft_q),
                                           _ptr(u_accept), _ptr(u_final), stride, _ptr(accept_len), _ptr(path_idx),
                                           _ptr(out_tokens), _ptr(n_out), _ptr(status))


def template_build(topk: int, depth: int, n_verify: int):
    """Static tree template of sampled drafting: (parent, rank, depth) int32 arrays (host side)."""
    lib = load()
    par, rank, dep = (np.zeros(n_verify, dtype=np.int32) for _ in range(3))
    n = C.c_int32(0)
    p = lambda a: a.ctypes.data_as(C.POINTER(C.c_int32))
    rc = lib.tlt_template_build(topk, depth, n_verify, p(par), p(rank), p(dep), C.byref(n))
    if rc:
        raise TltError(rc, "tlt_template_build")
    return par[: n.value].copy(), rank[: n.value].copy(), dep[: n.value].copy()


class Mab:
    """tlt_mab_*: the strategy selector (host only).  strategies: (Draft_Depth, topK, Tokens_to_Verify) tuples."""

    def __init__(self, strategies, thresholds, epsilon, window, sd_threshold=32):
        arr = (StrategyC * len(strategies))(*[StrategyC(*map(int, s)) for s in strategies])
        thr = (C.c_int32 * len(thresholds))(*map(int, thresholds))
        self.h = C.c_void_p()
        rc = load().tlt_mab_create(arr, len(strategies), thr, len(thresholds), float(epsilon), int(window),
                                   int(sd_threshold), C.byref(self.h))
        if rc:
            raise TltError(rc, "tlt_mab_create")

    def select(self, batch_size, u1, u2):
        """Strategy index, or None while speculation is switched off for this batch size."""
        out = C.c_int32()
        rc = load().tlt_mab_select(self.h, int(batch_size), int(u1), int(u2), C.byref(out))
        if rc:
            raise TltError(rc, "tlt_mab_select")
        return None if out.value < 0 else out.value

    def record(self, strategy, elapsed_time, accept_lens, batch_size):
        a, r = C.c_double(), C.c_double()
        lens = (C.c_int32 * len(accept_lens))(*map(int, accept_lens))
        rc = load().tlt_mab_record(self.h, int(strategy), float(elapsed_time), lens, int(batch_size), C.byref(a), C.byref(r))
        if rc:
            raise TltError(rc, "tlt_mab_record")
        return a.value, r.value

    def median_reward(self, strategy):
        m, n = C.c_double(), C.c_int32()
        rc = load().tlt_mab_median_reward(self.h, int(strategy), C.byref(m), C.byref(n))
        if rc:
            raise TltError(rc, "tlt_mab_median_reward")
        return m.value, n.value

    def close(self):
        if self.h:
            load().tlt_mab_destroy(self.h)
            self.h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class NGram:
    """tlt_ngram_*: the model-free drafter (host only)."""

    def __init__(self, order):
        self.h = C.c_void_p()
        rc = load().tlt_ngram_create(int(order), C.byref(self.h))
        if rc:
            raise TltError(rc, "tlt_ngram_create")

    def insert(self, prompt_id, tokens):
        arr = np.ascontiguousarray(tokens, dtype=np.int32)
        rc = load().tlt_ngram_insert(self.h, int(prompt_id), arr.ctypes.data_as(C.POINTER(C.c_int32)), len(arr))
        if rc:
            raise TltError(rc, "tlt_ngram_insert")

    def propose(self, prompt_id, context, depth, topk, n_nodes):
        """(token [n], parent [n], score [n]) numpy arrays of the proposed tree."""
        ctx = np.ascontiguousarray(context, dtype=np.int32)
        token, parent = np.empty(n_nodes, np.int32), np.empty(n_nodes, np.int32)
        score = np.empty(n_nodes, np.float32)
        rc = load().tlt_ngram_propose(self.h, int(prompt_id), ctx.ctypes.data_as(C.POINTER(C.c_int32)), len(ctx), int(depth),
                                      int(topk), int(n_nodes), token.ctypes.data_as(C.POINTER(C.c_int32)),
                                      parent.ctypes.data_as(C.POINTER(C.c_int32)), score.ctypes.data_as(C.POINTER(C.c_float)))
        if rc:
            raise TltError(rc, "tlt_ngram_propose")
        return token, parent, score

    def close(self):
        if self.h:
            load().tlt_ngram_destroy(self.h)
            self.h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def gemm(dtype_code, out_mode, A, W, Cout):
    """tlt_gemm: Cout[M, N] (op)= A[M, K] . W[N, K]^T on device tensors."""
    M, K = A.shape
    N = W.shape[0]
    rc = load().tlt_gemm(_stream(), dtype_code, out_mode, M, N, K, _ptr(A), _ptr(W), _ptr(Cout))
    if rc:
        raise TltError(rc, "tlt_gemm")


def attention_workspace(B, n, n_q_heads, n_kv_heads, head_dim, max_ctx) -> torch.Tensor:
    nbytes = load().tlt_attention_workspace_bytes(B, n, n_q_heads, n_kv_heads, head_dim, max_ctx)
    if nbytes == 0:
        raise TltError(-1, "tlt_attention_workspace_bytes")
    return torch.empty(nbytes, dtype=torch.uint8, device="cuda")


def attention(dtype_code, n_q_heads, page_size, qkv, anc_mask, kv: KV, out, ws, impl=-1):
    """tlt_attention on one layer's pools [n_pages, Hkv, page, d]; qkv [B, n, (Hq+2Hkv)*d]; returns the code."""
    B, n = qkv.shape[0], qkv.shape[1]
    n_kv, d = kv.k_pool.shape[-3], kv.k_pool.shape[-1]
    kvc = KVC(_ptr(kv.k_pool), _ptr(kv.v_pool), kv.k_pool.shape[-4], _ptr(kv.block_table), _ptr(kv.seq_len),
              kv.block_table.shape[1], int(kv.seq_len_bound))
    return load().tlt_attention(_stream(), dtype_code, B, n, n_q_heads, n_kv, d, page_size, _ptr(qkv), _ptr(anc_mask),
                                C.byref(kvc), _ptr(out), _ptr(ws), ws.numel(), impl)


class KV8:
    """8-bit paged KV cache of one model (tlt_kv8): codes [L, n_pages, Hkv, page, d] and exponent bytes [L, n_pages, Hkv, page] of keys and
    values (one byte per element: uint8, or float8_e4m3fn for the codes); the other fields as in KV.  Fields may be set one by one where their shapes
    stay, and together by replace(); they are checked against each other first, and one that does not fit leaves the cache as it was.  The tensors'
    addresses are taken at every call, their shapes when they are set: one that has been resized in place is set again."""
    _TENSORS = ("k_pool", "v_pool", "k_exp", "v_exp", "block_table", "seq_len")

    def __init__(self, k_pool: torch.Tensor, v_pool: torch.Tensor, k_exp: torch.Tensor, v_exp: torch.Tensor, block_table: torch.Tensor,
                 seq_len: torch.Tensor, seq_len_bound: int):
        self.replace(k_pool=k_pool, v_pool=v_pool, k_exp=k_exp, v_exp=v_exp, block_table=block_table, seq_len=seq_len, seq_len_bound=seq_len_bound)

    def __setattr__(self, name, value):
        if name in self._TENSORS:
            self.replace(**{name: value})
        else:
            object.__setattr__(self, name, value)

    def replace(self, **fields):
        """Sets several fields together: a batch of another size (block_table, seq_len, seq_len_bound), pools of more pages (all four)."""
        unknown = set(fields) - {*self._TENSORS, "seq_len_bound"}
        if unknown:
            raise TypeError(f"KV8 has no field {sorted(unknown)}")
        new = {**self.__dict__, **fields}
        new["seq_len_bound"] = int(new["seq_len_bound"])
        self._check(**{name: new[name] for name in self._TENSORS})
        # (layers, pages, kv heads, page size, head_dim), sequences, entries of the table per sequence
        new["dims"], new["table_dims"] = tuple(new["k_pool"].shape), tuple(new["block_table"].shape)
        self.__dict__.update(new)

    @staticmethod
    def _check(k_pool, v_pool, k_exp, v_exp, block_table, seq_len):
        assert k_pool.dim() == 5 and v_pool.shape == k_pool.shape and k_exp.shape == v_exp.shape == k_pool.shape[:4], "pools' shapes"
        assert all(t.element_size() == 1 for t in (k_pool, v_pool, k_exp, v_exp)), "pools hold bytes"
        assert block_table.dtype == seq_len.dtype == torch.int32 and block_table.dim() == 2
        assert seq_len.shape == block_table.shape[:1]
        assert all(t.is_cuda and t.is_contiguous() and t.device == k_pool.device for t in (k_pool, v_pool, k_exp, v_exp, block_table, seq_len)), \
            "device tensors must be contiguous CUDA/HIP tensors"

    @staticmethod
    def empty(n_layers, n_pages, n_kv_heads, page_size, head_dim, block_table, seq_len, seq_len_bound) -> "KV8":
        """Pools of zeros; block_table [B, max_pages] and seq_len [B]: int32 device tensors."""
        pool = lambda *s: torch.zeros((n_layers, n_pages, n_kv_heads, page_size, *s), dtype=torch.uint8, device=block_table.device)
        return KV8(pool(head_dim), pool(head_dim), pool().fill_(127), pool().fill_(127), block_table, seq_len, seq_len_bound)

    def c(self, layer: int = 0) -> KV8C:
        """The C handle of the layers from `layer` on."""
        L, n_pages, n_kv, page, d = self.dims
        if not 0 <= layer < L:
            raise IndexError(f"layer {layer} of {L}")
        rows = layer * n_pages * n_kv * page
        return KV8C(self.k_pool.data_ptr() + rows * d, self.v_pool.data_ptr() + rows * d, self.k_exp.data_ptr() + rows, self.v_exp.data_ptr() + rows, n_pages,
                    self.block_table.data_ptr(), self.seq_len.data_ptr(), self.table_dims[1], self.seq_len_bound)


def _stream_of(kv: KV8):
    """The current stream of the cache's device, which has to be the current one."""
    device = kv.k_pool.get_device()
    assert device == torch.cuda.current_device(), "the cache lies on another device than the current one"
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)   # (a tenth of what current_stream()'s object costs, 2.8 us)
    return raw(device) if raw is not None else torch.cuda.current_stream(device).cuda_stream


def _addr(t: Optional[torch.Tensor], kv: KV8, shape, dtype):
    """The address of a contiguous tensor beside the cache, of this shape and type (a type, or the bytes of an element); None stays None."""
    if t is None:
        return None
    assert t.shape == shape and (t.dtype is dtype or t.element_size() == dtype) and t.is_contiguous() and t.get_device() == kv.k_pool.get_device(), \
        f"a contiguous tensor {tuple(shape)} of {dtype} on the cache's device"
    return t.data_ptr()


def _rows(t: torch.Tensor, kv: KV8, shape, dtype):
    """(address, elements between rows) of rows [B, n, width] that may lie in wider ones."""
    assert t.shape == shape and t.dtype is dtype and t.get_device() == kv.k_pool.get_device(), f"rows {tuple(shape)} of {dtype} on the cache's device"
    B, n, width = shape
    step = t.stride(1) if n > 1 else (t.stride(0) if B > 1 else width)   # (a dimension of one element may have any stride)
    assert t.stride(2) == 1 and (B == 1 or t.stride(0) == n * step), "rows must be evenly spaced"
    return t.data_ptr(), step


def kv8_write(dtype_code, n_q_heads, rope_theta, qkv, bias, depth, kv: KV8, layer, q_out):
    """tlt_kv8_write: qkv [B, n, (Hq+2Hkv)*d], bias [(Hq+2Hkv)*d] or None, depth [B, n] int32 or None (a chain), q_out [B, n, Hq*d] (contiguous, or
    the first Hq*d columns of wider rows: qkv[..., :Hq*d] itself)."""
    _, _, n_kv, page, d = kv.dims
    B, n, width = kv.table_dims[0], qkv.shape[1], (n_q_heads + 2 * n_kv) * d
    dt = torch_dtype(dtype_code)
    q, step = _rows(q_out, kv, (B, n, n_q_heads * d), dt)
    rc = load().tlt_kv8_write(_stream_of(kv), dtype_code, B, n, n_q_heads, n_kv, d, page, rope_theta, _addr(qkv, kv, (B, n, width), dt),
                              _addr(bias, kv, (width,), dt), _addr(depth, kv, (B, n), torch.int32), kv.c(layer), q, step)
    if rc:
        raise TltError(rc, "tlt_kv8_write")


def kv8_attention_workspace(B, n, n_q_heads, n_kv_heads, head_dim, max_ctx) -> torch.Tensor:
    nbytes = load().tlt_kv8_attention_workspace_bytes(B, n, n_q_heads, n_kv_heads, head_dim, max_ctx)
    if nbytes == 0:
        raise TltError(-1, "tlt_kv8_attention_workspace_bytes")
    return torch.empty(nbytes, dtype=torch.uint8, device="cuda")


def kv8_attention(dtype_code, n_q_heads, q, anc_mask, kv: KV8, layer, out, ws, impl=-1):
    """tlt_kv8_attention: q [B, n, Hq*d] (rows as kv8_write's q_out), anc_mask [B, n] int64 or None (a chain), out [B, n, Hq*d]."""
    _, _, n_kv, page, d = kv.dims
    B, n = kv.table_dims[0], q.shape[1]
    shape, dt = (B, n, n_q_heads * d), torch_dtype(dtype_code)
    qp, step = _rows(q, kv, shape, dt)
    assert ws.is_contiguous() and ws.get_device() == kv.k_pool.get_device()
    rc = load().tlt_kv8_attention(_stream_of(kv), dtype_code, B, n, n_q_heads, n_kv, d, page, qp, step, _addr(anc_mask, kv, (B, n), 8), kv.c(layer),
                                  _addr(out, kv, shape, dt), ws.data_ptr(), ws.numel() * ws.element_size(), impl)
    if rc:
        raise TltError(rc, "tlt_kv8_attention")


def kv8_commit(kv: KV8, accept_len, path_idx):
    """tlt_kv8_commit over all layers: accept_len [B], path_idx [B, stride] int32.  kv.seq_len_bound is left to the caller, as in kv_commit."""
    L, _, n_kv, page, d = kv.dims
    B, stride = kv.table_dims[0], path_idx.shape[1]
    rc = load().tlt_kv8_commit(_stream_of(kv), B, L, n_kv, d, page, kv.c(), _addr(accept_len, kv, (B,), torch.int32), _addr(path_idx, kv, (B, stride), torch.int32),
                               stride)
    if rc:
        raise TltError(rc, "tlt_kv8_commit")


def kv8_read(dtype_code, kv: KV8, first, count, out_k, out_v):
    """tlt_kv8_read over all layers: first [B] int32, count [B] int32 or None, out_k / out_v [L, B, n, Hkv, d] of dtype_code's type."""
    L, _, n_kv, page, d = kv.dims
    B, n, dt = kv.table_dims[0], out_k.shape[2], torch_dtype(dtype_code)
    shape = (L, B, n, n_kv, d)
    rc = load().tlt_kv8_read(_stream_of(kv), dtype_code, L, B, n, n_kv, d, page, kv.c(), _addr(first, kv, (B,), torch.int32), _addr(count, kv, (B,), torch.int32),
                             _addr(out_k, kv, shape, dt), _addr(out_v, kv, shape, dt))
    if rc:
        raise TltError(rc, "tlt_kv8_read")


# ---- pages, rotary positions, sampling: what a step of a caller with a forward of its own needs around the attention calls
# (Small calls are bound by the host, so checks are few and cheap: a launch costs 2.6 us, a tensor's check 0.3.)

_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _here(device: int) -> int:
    """The current stream of `device`, which has to be the current one."""
    assert device == _current_device(), "the tensors lie on another device than the current one"
    return _raw_stream(device) if _raw_stream is not None else torch.cuda.current_stream(device).cuda_stream


def _at(t: Optional[torch.Tensor], device: int, count: int, dtype, name: str):
    """The address of a contiguous device tensor of so many elements of this type; None stays None."""
    if t is None:
        return None
    assert t.dtype is dtype and t.numel() == count and t.is_contiguous() and t.get_device() == device, f"{name}: a contiguous {dtype} tensor of {count} on the device of the others"
    return t.data_ptr()


def _row_step(t: torch.Tensor, device: int, rows: int, width: int, dtype, name: str) -> int:
    """Elements between the rows of a tensor [..., width] whose leading dimensions are rows, evenly spaced; checks them."""
    assert t.dtype is dtype and t.get_device() == device and t.size(-1) == width and t.numel() == rows * width, f"{name}: {rows} rows of {width} {dtype} on the device of the others"
    if t.is_contiguous():
        return width
    assert width == 1 or t.stride(-1) == 1, f"{name}: elements of a row lie side by side"
    step, expect = width, None
    for size, stride in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:          # (a dimension of one element may have any stride)
            continue
        if expect is None:
            step = stride
        else:
            assert stride == expect, f"{name}: rows must be evenly spaced"
        expect = stride * size
    assert step >= width, f"{name}: rows may not overlap"
    return step


class Pages:
    """The pages of a paged cache (tlt_pages): free_page [n_pages], n_free [1], page_count [B], block_table [B, max_pages], int32 device tensors; block_table is the one
    that the cache's handle (KV, KV8) holds.  The tensors are checked here and kept; their addresses are taken at every call."""

    def __init__(self, free_page: torch.Tensor, n_free: torch.Tensor, page_count: torch.Tensor, block_table: torch.Tensor, page_size: int):
        dev = block_table.get_device()
        assert dev >= 0 and block_table.dim() == 2, "block_table: a device tensor [B, max_pages]"
        B, max_pages = block_table.shape
        for name, x, count in (("free_page", free_page, free_page.numel()), ("n_free", n_free, 1), ("page_count", page_count, B), ("block_table", block_table, B * max_pages)):
            _at(x, dev, count, torch.int32, name)
        self._tensors, self._sizes, self.device, self.batch = (free_page, n_free, page_count, block_table), (free_page.numel(), max_pages, int(page_size)), dev, B

    free_page, n_free, page_count, block_table = (property(lambda self, i=i: self._tensors[i]) for i in range(4))
    page_size = property(lambda self: self._sizes[2])

    @staticmethod
    def empty(B, n_pages, max_pages, page_size, device="cuda") -> "Pages":
        """All pages free, the lowest taken first; no sequence holds any."""
        i32 = dict(dtype=torch.int32, device=device)
        return Pages(torch.arange(n_pages - 1, -1, -1, **i32), torch.full((1,), n_pages, **i32), torch.zeros((B,), **i32), torch.full((B, max_pages), -1, **i32), page_size)

    def c(self) -> PagesC:
        free, n_free, count, table = self._tensors
        return PagesC(free.data_ptr(), n_free.data_ptr(), count.data_ptr(), table.data_ptr(), *self._sizes)


def pages_grow(pages: Pages, seq_len, n_new, depth, row_start, row_seq, position, slot, granted):
    """tlt_pages_grow: seq_len, n_new [B] int32; depth [rows] int32 or None; outputs (each may be None) row_start [B + 1], row_seq, position [rows] and granted [B] int32,
    slot [rows] int64, all row tensors of one size."""
    dev, B, i32, rows = pages.device, pages.batch, torch.int32, 0
    for t in (slot, position, row_seq, depth):
        if t is not None:
            rows = t.numel()
            break
    rc = load().tlt_pages_grow(_here(dev), B, pages.c(), _at(seq_len, dev, B, i32, "seq_len"), _at(n_new, dev, B, i32, "n_new"), _at(depth, dev, rows, i32, "depth"), rows,
                               _at(row_start, dev, B + 1, i32, "row_start"), _at(row_seq, dev, rows, i32, "row_seq"), _at(position, dev, rows, i32, "position"),
                               _at(slot, dev, rows, torch.int64, "slot"), _at(granted, dev, B, i32, "granted"))
    if rc:
        raise TltError(rc, "tlt_pages_grow")


def pages_release(pages: Pages, keep_len):
    """tlt_pages_release: keep_len [B] int32, or None: everything."""
    dev, B = pages.device, pages.batch
    rc = load().tlt_pages_release(_here(dev), B, pages.c(), _at(keep_len, dev, B, torch.int32, "keep_len"))
    if rc:
        raise TltError(rc, "tlt_pages_release")


ROPE_SCALING = {"plain": 0, "linear": 1, "base": 2, "ramp": 3, "bands": 4}


def rope_freqs(scaling: str, rot_dim: int, theta: float, factor: float = 1.0, original_len: float = 0.0, low: float = 1.0, high: float = 32.0):
    """tlt_rope_freqs: (frequencies [rot_dim / 2] float64 on the host, amplitude)."""
    freq, amplitude = np.empty(max(rot_dim // 2, 1), np.float64), C.c_float()
    rc = load().tlt_rope_freqs(ROPE_SCALING[scaling], rot_dim, theta, factor, original_len, low, high, freq.ctypes.data, C.byref(amplitude))
    if rc:
        raise TltError(rc, "tlt_rope_freqs")
    return freq, amplitude.value


class Rope:
    """tlt_rope: freq [rot_dim / 2] float64 device tensor (radians per position, as rope_freqs gives them), layout of the pairs, amplitude."""

    def __init__(self, freq: torch.Tensor, interleaved: bool = False, amplitude: float = 1.0):
        assert freq.dtype is torch.float64 and freq.dim() == 1 and freq.is_contiguous() and freq.get_device() >= 0, "freq: a contiguous float64 device tensor"
        self._freq, self._rest, self.device = freq, (2 * freq.numel(), int(bool(interleaved)), float(amplitude)), freq.get_device()

    freq = property(lambda self: self._freq)
    interleaved = property(lambda self: bool(self._rest[1]))
    amplitude = property(lambda self: self._rest[2])

    def c(self) -> RopeC:
        return RopeC(self._freq.data_ptr(), *self._rest)


def rope_write(dtype_code, n_q_heads, n_kv_heads, head_dim, rope: Rope, qkv, bias, position, slot, kv, layer, q_out, kv_out=None):
    """tlt_rope_write: qkv rows [..., (Hq+2Hkv)*d], evenly spaced; bias [(Hq+2Hkv)*d] or None; position [rows] int32, slot [rows] int64 (None without a cache); kv a KV (pools
    [layers, pages, Hkv, page, d] of dtype_code's type, or one layer's), a KV8 or None, `layer` of it; q_out rows [..., Hq*d] and kv_out rows [..., 2*Hkv*d], each or None."""
    dev, dt, d = rope.device, torch_dtype(dtype_code), head_dim
    width, rows = (n_q_heads + 2 * n_kv_heads) * d, position.numel()
    step = _row_step(qkv, dev, rows, width, dt, "qkv")
    q, q_step = (None, 0) if q_out is None else (q_out.data_ptr(), _row_step(q_out, dev, rows, n_q_heads * d, dt, "q_out"))
    o, o_step = (None, 0) if kv_out is None else (kv_out.data_ptr(), _row_step(kv_out, dev, rows, 2 * n_kv_heads * d, dt, "kv_out"))
    kvc, kv8c, page = None, None, 1
    if isinstance(kv, KV8):
        _, _, heads, page, pool_d = kv.dims
        assert heads == n_kv_heads and pool_d == d and kv.k_pool.get_device() == dev, "the cache's shape and device"
        kv8c = kv.c(layer)
    elif kv is not None:
        k, v = kv.k_pool, kv.v_pool
        shape = k.shape
        layers, (n_pages, heads, page, pool_d) = (shape[0] if len(shape) == 5 else 1), shape[-4:]
        assert len(shape) in (4, 5) and v.shape == shape and heads == n_kv_heads and pool_d == d, "the cache's shape"
        assert k.dtype is dt and v.dtype is dt and k.is_contiguous() and v.is_contiguous() and k.get_device() == dev and v.get_device() == dev, \
            "contiguous pools of the model's type on the device of the others"
        if not 0 <= layer < layers:
            raise IndexError(f"layer {layer} of {layers}")
        at = layer * n_pages * heads * page * d * (4 if dtype_code == TLT_F32 else 2)
        kvc = KVC(k.data_ptr() + at, v.data_ptr() + at, n_pages, None, None, 0, 0)
    rc = load().tlt_rope_write(_here(dev), dtype_code, rows, n_q_heads, n_kv_heads, d, page, rope.c(), qkv.data_ptr(), step, _at(bias, dev, width, dt, "bias"),
                               _at(position, dev, rows, torch.int32, "position"), _at(slot, dev, rows, torch.int64, "slot"), kvc, kv8c, q, q_step, o, o_step)
    if rc:
        raise TltError(rc, "tlt_rope_write")


class SampleFilter:
    """tlt_filter: what each sequence asks for, device tensors [B] or None: temperature, top_p, min_p float32, top_k int32.  Checked here and kept; addresses are taken at every call."""

    def __init__(self, temperature=None, top_k=None, top_p=None, min_p=None):
        tensors, self.device, self.batch = (temperature, top_k, top_p, min_p), None, None
        for name, t, dt in zip(("temperature", "top_k", "top_p", "min_p"), tensors, (torch.float32, torch.int32, torch.float32, torch.float32)):
            if t is not None:
                assert t.dim() == 1 and t.get_device() >= 0, f"{name}: a device tensor [B]"
                if self.batch is None:
                    self.device, self.batch = t.get_device(), t.numel()
                _at(t, self.device, self.batch, dt, name)
        self._tensors = tensors

    temperature, top_k, top_p, min_p = (property(lambda self, i=i: self._tensors[i]) for i in range(4))

    def c(self, B, device) -> FilterC:
        assert self.batch is None or (self.batch == B and self.device == device), f"settings of {B} sequences on the device of the others"
        a, b, c, d = self._tensors
        return FilterC(a.data_ptr() if a is not None else None, b.data_ptr() if b is not None else None, c.data_ptr() if c is not None else None, d.data_ptr() if d is not None else None)


def sample_workspace(rows, vocab) -> torch.Tensor:
    nbytes = load().tlt_sample_workspace_bytes(rows, vocab)
    if nbytes == 0:
        raise TltError(-1, "tlt_sample_workspace_bytes")
    return torch.empty(nbytes, dtype=torch.uint8, device="cuda")


def _logit_rows(logits, dtype_code):
    """(device, rows, rows per sequence, sequences, vocab, elements between rows) of logits [B, V] or [B, n, V]."""
    shape = logits.shape
    assert len(shape) in (2, 3), "logits [B, V] or [B, n, V]"
    B, V, n = shape[0], shape[-1], shape[1] if len(shape) == 3 else 1
    dev = logits.get_device()
    return dev, B * n, n, B, V, _row_step(logits, dev, B * n, V, torch_dtype(dtype_code), "logits")


def sample(dtype_code, logits, asked: SampleFilter, u, token, logprob, kept, ws):
    """tlt_sample: logits [B, V] or [B, n, V] of dtype_code's type (rows evenly spaced, so a slice of wider rows will do), u like logits without V, int32 or uint32;
    token and kept (may be None) int32 of u's size, logprob (may be None) float32 [..., 2]."""
    dev, rows, n, B, V, step = _logit_rows(logits, dtype_code)
    assert ws.is_contiguous() and ws.get_device() == dev, "the workspace"
    rc = load().tlt_sample(_here(dev), dtype_code, rows, n, V, logits.data_ptr(), step, asked.c(B, dev), _at(u, dev, rows, torch.uint32 if u.dtype is torch.uint32 else torch.int32, "u"),
                           _at(token, dev, rows, torch.int32, "token"), _at(logprob, dev, 2 * rows, torch.float32, "logprob"), _at(kept, dev, rows, torch.int32, "kept"),
                           ws.data_ptr(), ws.numel() * ws.element_size())
    if rc:
        raise TltError(rc, "tlt_sample")


def sample_filter(dtype_code, logits, asked: SampleFilter, out, kept, ws):
    """tlt_sample_filter: out like logits (may be logits itself), kept (may be None) int32 of logits' size without V."""
    dev, rows, n, B, V, step = _logit_rows(logits, dtype_code)
    assert out.shape == logits.shape and ws.is_contiguous() and ws.get_device() == dev, "out like logits, and the workspace"
    rc = load().tlt_sample_filter(_here(dev), dtype_code, rows, n, V, logits.data_ptr(), step, asked.c(B, dev), out.data_ptr(),
                                  _row_step(out, dev, rows, V, torch_dtype(dtype_code), "out"), _at(kept, dev, rows, torch.int32, "kept"), ws.data_ptr(), ws.numel() * ws.element_size())
    if rc:
        raise TltError(rc, "tlt_sample_filter")


def gemm_argmax(A, W, ws, out):
    """out[m] = argmax_n (A W^T)[m, n] for bf16 device tensors A [M, K], W [N, K]; returns the library's code."""
    M, K = A.shape
    N = W.shape[0]
    return load().tlt_gemm_argmax(_stream(), M, N, K, _ptr(A), _ptr(W), _ptr(ws), ws.numel() * ws.element_size(), _ptr(out))


def gemm_glu(A, Wg, Wu, act):
    """act = silu(A Wg^T) * (A Wu^T) for bf16 device tensors A [M, K], Wg/Wu [N, K], act [M, N]; returns the code."""
    M, K = A.shape
    return load().tlt_gemm_glu(_stream(), M, Wg.shape[0], K, _ptr(A), _ptr(Wg), _ptr(Wu), _ptr(act))


def gemm_parts(A, W, parts):
    """tlt_gemm_parts: A [M, K], W [N, K] bf16, parts a flat fp32 device tensor; returns the slices [n_parts, M, N] written to it."""
    M, K = A.shape
    N = W.shape[0]
    n = C.c_int()
    rc = load().tlt_gemm_parts(_stream(), M, N, K, _ptr(A), _ptr(W), _ptr(parts), parts.numel() * 4, C.byref(n))
    if rc:
        raise TltError(rc, "tlt_gemm_parts")
    return parts[:n.value * M * N].view(n.value, M, N)


def mfma_stream(frags, out, iters):
    """tlt_mfma_stream: `iters` rounds of a wave tile's 64 MFMAs on the register fragments read from `frags` (bf16
    device tensor of 16384 values), every lane's accumulator sum to `out` (fp32 device tensor of 65536); returns the code."""
    assert frags.numel() * frags.element_size() == 32768 and out.numel() == 65536 and out.element_size() == 4
    return load().tlt_mfma_stream(_stream(), _ptr(frags), _ptr(out), int(iters))


class GraphPool:
    """tlt_graph_pool_*: the library's HIP-graph pool (greedy step per batch bucket, drafter and target graphs
    apart).  The caller's tensors must stay alive and in place for as long as their graphs are replayed."""

    def __init__(self, ctx: "Context", buckets, seq_len_bound: int):
        self.ctx = ctx
        self.lib = ctx.lib
        arr = (C.c_int32 * len(buckets))(*buckets)
        self.handle = C.c_void_p()
        rc = self.lib.tlt_graph_pool_create(ctx.handle, arr, len(buckets), int(seq_len_bound), C.byref(self.handle))
        if rc:
            raise TltError(rc, "tlt_graph_pool_create", self.lib.tlt_last_hip_error(ctx.handle))

    def step(self, B, depth, topk, n_verify, new_tokens, new_src, n_new, hidden, draft_kv: "KV", tree: "Tree", kv: "KV",
             argmax, hidden_out, stride, accept_len, path_idx, out_tokens, n_out):
        dkv_c, kv_c, tree_c = draft_kv.c(), kv.c(), tree.c()
        a = StepArgsC(_ptr(new_tokens), _ptr(new_src), _ptr(n_new), new_tokens.shape[1], _ptr(hidden), hidden.shape[1],
                      C.pointer(dkv_c), C.pointer(tree_c), C.pointer(kv_c), _ptr(argmax), _ptr(hidden_out), stride,
                      _ptr(accept_len), _ptr(path_idx), _ptr(out_tokens), _ptr(n_out))
        rc = self.lib.tlt_graph_pool_step(self.handle, _stream(), B, depth, topk, n_verify, C.byref(a))
        if rc:
            raise TltError(rc, "tlt_graph_pool_step", self.lib.tlt_last_hip_error(self.ctx.handle))

    def count(self):
        nd, nt = C.c_int32(), C.c_int32()
        rc = self.lib.tlt_graph_pool_count(self.handle, C.byref(nd), C.byref(nt))
        if rc:
            raise TltError(rc, "tlt_graph_pool_count")
        return nd.value, nt.value

    def close(self):
        if self.handle:
            torch.cuda.synchronize()
            self.lib.tlt_graph_pool_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
