"""Thin ctypes binding of libanpd.so: argument marshalling only.

Every step of the verification path runs inside the library's HIP kernels.
PyTorch appears here only as the allocator of device memory and the owner of
the stream.  There is no CPU fallback: if the library is missing, importing
``lib()`` raises.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os
from typing import Dict, List, Optional, Sequence, Tuple

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libanpd.so")

OK, E_INVAL, E_RANGE, E_CAPACITY, E_NOMEM, E_HIP, E_UNIMPLEMENTED = 0, -1, -2, -3, -4, -5, -6
F32, BF16, INT8 = 0, 1, 8
VERIFY, APPEND = 0, 1
GEMM_AUTO, GEMM_DOT, GEMM_MFMA, GEMM_MFMA_STREAM, GEMM_MFMA_LAUNCHES = 0, 1, 2, 3, 4
MAX_WINDOW = 32
TREE_MAX_ROWS = 64

_PER_LAYER = ("attn_norm", "wq", "wk", "wv", "wo", "ffn_norm", "w_gate", "w_up", "w_down")

# every symbol include/anpd.h declares
EXPORTS = (
    "anpd_last_error",
    "anpd_ngram_create", "anpd_ngram_destroy", "anpd_ngram_reset", "anpd_ngram_update",
    "anpd_ngram_length", "anpd_ngram_query", "anpd_ngram_propose", "anpd_ngram_propose_tree",
    "anpd_model_workspace_bytes", "anpd_model_create", "anpd_model_destroy",
    "anpd_kv_pool_bytes", "anpd_kv_create", "anpd_kv_destroy", "anpd_kv_length", "anpd_kv_truncate",
    "anpd_kv_set_page_order", "anpd_kv_num_pages", "anpd_kv_write", "anpd_kv_read",
    "anpd_verify", "anpd_verify_tree", "anpd_verify_batch", "anpd_prefill_workspace_bytes", "anpd_prefill", "anpd_linear_workspace_bytes", "anpd_linear",
    "anpd_model_profile", "anpd_model_profile_read", "anpd_packed_bytes", "anpd_pack_weights",
    "anpd_model_trace", "anpd_model_set_barrier_spin_limit", "anpd_linear_static",
    "anpd_cache_pool_bytes", "anpd_cache_create", "anpd_attention_workspace_bytes", "anpd_attention",
    "anpd_key_mass_workspace_bytes", "anpd_key_mass", "anpd_kv_evict",
    "anpd_kv_observe_workspace_bytes", "anpd_kv_observe",
    "anpd_kv_store", "anpd_kv_load", "anpd_tree_attention_workspace_bytes", "anpd_tree_attention", "anpd_kv_commit",
    "anpd_sample_workspace_bytes", "anpd_sample", "anpd_verify_sample",
)
PROF_CATEGORIES = ("gemm_qkv", "gemm_o", "gemm_gate_up", "gemm_down", "gemm_lm_head", "attn", "other", "step")


class AnpdError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__("anpd error %d: %s" % (code, msg))
        self.code = code


class ModelCfg(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_heads", C.c_int32),
                ("head_dim", C.c_int32), ("d_ffn", C.c_int32), ("vocab", C.c_int32),
                ("rms_eps", C.c_float), ("rope_base", C.c_float), ("dtype", C.c_int32),
                ("page_tokens", C.c_int32), ("max_window", C.c_int32), ("max_positions", C.c_int32),
                ("gemm_path", C.c_int32), ("n_kv_heads", C.c_int32)]


class CacheCfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "n_heads", "head_dim", "n_kv_heads", "dtype", "page_tokens")]


class AttnRules(C.Structure):
    _fields_ = [("scale", C.c_float), ("cap", C.c_float), ("window", C.c_int32), ("prefix", C.c_int32),
                ("slopes", C.c_void_p), ("first_key", C.c_void_p)]


class SampleRules(C.Structure):
    _fields_ = [("temperature", C.c_float), ("top_k", C.c_int32), ("top_p", C.c_float), ("min_p", C.c_float)] + \
               [(n, C.c_void_p) for n in ("temperatures", "top_ks", "top_ps", "min_ps")]


class Weights(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("final_norm", C.c_void_p), ("lm_head", C.c_void_p)] + \
               [(n, C.POINTER(C.c_void_p)) for n in _PER_LAYER]


_lib = None


def lib():
    """Load libanpd.so (built by ``build.build()``); fail loudly if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError("libanpd.so is not built: run `python -m paper_2404_08698_amd.build` "
                          "(there is no fallback path)")
    # PyTorch ships its own copy of the HIP runtime.  Load it first, so that this library binds to the
    # runtime the device memory comes from: with the order reversed the process ends up with two runtimes,
    # and the second one finds no device.
    try:
        import torch  # noqa: F401
    except ImportError:
        pass
    L = C.CDLL(LIB_PATH)
    i32p, vp = C.POINTER(C.c_int32), C.c_void_p
    L.anpd_last_error.restype = C.c_char_p
    L.anpd_last_error.argtypes = []
    L.anpd_ngram_create.restype = C.c_int32
    L.anpd_ngram_create.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.POINTER(vp)]
    L.anpd_ngram_destroy.restype = None
    L.anpd_ngram_destroy.argtypes = [vp]
    L.anpd_ngram_reset.restype = C.c_int32
    L.anpd_ngram_reset.argtypes = [vp]
    L.anpd_ngram_update.restype = C.c_int32
    L.anpd_ngram_update.argtypes = [vp, i32p, C.c_int64]
    L.anpd_ngram_length.restype = C.c_int64
    L.anpd_ngram_length.argtypes = [vp]
    L.anpd_ngram_query.restype = C.c_int32
    L.anpd_ngram_query.argtypes = [vp, i32p, C.c_int32, i32p, i32p]
    L.anpd_ngram_propose.restype = C.c_int32
    L.anpd_ngram_propose.argtypes = [vp, C.c_int32, i32p, i32p]
    L.anpd_ngram_propose_tree.restype = C.c_int32
    L.anpd_ngram_propose_tree.argtypes = [vp, C.c_int32, C.c_int32, C.c_int32, i32p, i32p, i32p]
    L.anpd_model_workspace_bytes.restype = C.c_size_t
    L.anpd_model_workspace_bytes.argtypes = [C.POINTER(ModelCfg)]
    L.anpd_model_create.restype = C.c_int32
    L.anpd_model_create.argtypes = [C.POINTER(ModelCfg), C.POINTER(Weights), vp, C.c_size_t, vp, C.POINTER(vp)]
    L.anpd_model_destroy.restype = None
    L.anpd_model_destroy.argtypes = [vp]
    L.anpd_kv_pool_bytes.restype = C.c_size_t
    L.anpd_kv_pool_bytes.argtypes = [vp, C.c_int32]
    L.anpd_kv_create.restype = C.c_int32
    L.anpd_kv_create.argtypes = [vp, vp, C.c_size_t, C.c_int32, C.POINTER(vp)]
    L.anpd_kv_destroy.restype = None
    L.anpd_kv_destroy.argtypes = [vp]
    L.anpd_kv_length.restype = C.c_int32
    L.anpd_kv_length.argtypes = [vp]
    L.anpd_kv_truncate.restype = C.c_int32
    L.anpd_kv_truncate.argtypes = [vp, C.c_int32, vp]
    L.anpd_kv_set_page_order.restype = C.c_int32
    L.anpd_kv_set_page_order.argtypes = [vp, i32p, C.c_int32]
    L.anpd_kv_num_pages.restype = C.c_int32
    L.anpd_kv_num_pages.argtypes = [vp]
    L.anpd_kv_write.restype = C.c_int32
    L.anpd_kv_write.argtypes = [vp, C.c_int32, C.c_int32, C.c_int32, vp, vp, vp]
    L.anpd_kv_read.restype = C.c_int32
    L.anpd_kv_read.argtypes = [vp, C.c_int32, C.c_int32, C.c_int32, vp, vp, vp]
    L.anpd_verify.restype = C.c_int32
    L.anpd_verify.argtypes = [vp, vp, i32p, C.c_int32, C.c_int32, i32p, i32p, i32p, vp, vp]
    L.anpd_verify_tree.restype = C.c_int32
    L.anpd_verify_tree.argtypes = [vp, vp, i32p, i32p, C.c_int32, i32p, i32p, i32p, i32p, vp, vp]
    L.anpd_verify_batch.restype = C.c_int32
    L.anpd_verify_batch.argtypes = [vp, C.POINTER(vp), C.c_int32, C.POINTER(i32p), i32p, C.c_int32, i32p, i32p, vp, vp]
    L.anpd_prefill_workspace_bytes.restype = C.c_size_t
    L.anpd_prefill_workspace_bytes.argtypes = [vp, C.c_int32]
    L.anpd_prefill.restype = C.c_int32
    L.anpd_prefill.argtypes = [vp, vp, i32p, C.c_int32, i32p, vp, vp, C.c_size_t, vp]
    L.anpd_linear_workspace_bytes.restype = C.c_size_t
    L.anpd_linear_workspace_bytes.argtypes = [C.c_int32, C.c_int32]
    L.anpd_linear.restype = C.c_int32
    L.anpd_linear.argtypes = [vp, vp, vp, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, vp, C.c_size_t, vp]
    L.anpd_linear_static.restype = C.c_int32
    L.anpd_linear_static.argtypes = [vp, vp, vp, C.c_int32, C.c_int32, C.c_int32, vp]
    L.anpd_packed_bytes.restype = C.c_size_t
    L.anpd_packed_bytes.argtypes = [C.c_int32, C.c_int32]
    L.anpd_pack_weights.restype = C.c_int32
    L.anpd_pack_weights.argtypes = [vp, C.c_int32, C.c_int32, vp, C.c_size_t, vp]
    L.anpd_model_trace.restype = C.c_int32
    L.anpd_model_trace.argtypes = [vp, vp, C.c_size_t]
    L.anpd_model_set_barrier_spin_limit.restype = C.c_int32
    L.anpd_model_set_barrier_spin_limit.argtypes = [vp, C.c_int32]
    L.anpd_model_profile.restype = C.c_int32
    L.anpd_model_profile.argtypes = [vp, C.c_int32]
    L.anpd_model_profile_read.restype = C.c_int32
    L.anpd_model_profile_read.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_int64), C.POINTER(C.c_int64)]
    seqs = [vp, C.c_int32, vp, vp]
    L.anpd_cache_pool_bytes.restype = C.c_size_t
    L.anpd_cache_pool_bytes.argtypes = [C.POINTER(CacheCfg), C.c_int32]
    L.anpd_cache_create.restype = C.c_int32
    L.anpd_cache_create.argtypes = [C.POINTER(CacheCfg), vp, C.c_size_t, C.c_int32, C.POINTER(vp)]
    L.anpd_attention_workspace_bytes.restype = C.c_size_t
    L.anpd_attention_workspace_bytes.argtypes = seqs + [vp]
    L.anpd_attention.restype = C.c_int32
    L.anpd_attention.argtypes = seqs + [C.c_int32, vp, C.c_int64, C.c_int32, vp, vp, C.c_int64, vp, vp, C.c_size_t, vp]
    L.anpd_key_mass_workspace_bytes.restype = C.c_size_t
    L.anpd_key_mass_workspace_bytes.argtypes = seqs + [vp]
    L.anpd_key_mass.restype = C.c_int32
    L.anpd_key_mass.argtypes = seqs + [C.c_int32, vp, C.c_int64, C.c_int32, vp, vp, vp, C.c_int64, vp, C.c_size_t, vp]
    L.anpd_kv_evict.restype = C.c_int32
    L.anpd_kv_evict.argtypes = [vp, vp, vp, C.c_int64, C.c_int32, C.c_int32, C.c_int32, C.c_float, vp, vp, C.c_int64, vp]
    L.anpd_kv_observe_workspace_bytes.restype = C.c_size_t
    L.anpd_kv_observe_workspace_bytes.argtypes = [vp, C.c_int32]
    L.anpd_kv_observe.restype = C.c_int32
    L.anpd_kv_observe.argtypes = [vp, vp, C.c_int64, C.c_int32, vp, C.c_size_t]
    rows = seqs + [C.c_int32, vp, C.c_int64, vp, C.c_int64, C.c_int32, vp]
    L.anpd_kv_store.restype = C.c_int32
    L.anpd_kv_store.argtypes = rows
    L.anpd_kv_load.restype = C.c_int32
    L.anpd_kv_load.argtypes = rows
    L.anpd_tree_attention_workspace_bytes.restype = C.c_size_t
    L.anpd_tree_attention_workspace_bytes.argtypes = seqs + [vp]
    L.anpd_tree_attention.restype = C.c_int32
    L.anpd_tree_attention.argtypes = seqs + [C.c_int32, vp, C.c_int64, C.c_int32, vp, vp, vp, C.c_int64, vp, vp, C.c_size_t, vp]
    L.anpd_kv_commit.restype = C.c_int32
    L.anpd_kv_commit.argtypes = [vp, i32p, C.c_int32, vp]
    L.anpd_sample_workspace_bytes.restype = C.c_size_t
    L.anpd_sample_workspace_bytes.argtypes = [C.c_int32, C.c_int32]
    L.anpd_sample.restype = C.c_int32
    L.anpd_sample.argtypes = [vp, C.c_int64, C.c_int32, C.c_int32, C.c_int32, vp, vp, vp, vp, vp, C.c_size_t, vp]
    L.anpd_verify_sample.restype = C.c_int32
    L.anpd_verify_sample.argtypes = [vp, vp, i32p, C.c_int32, vp, vp, i32p, i32p, i32p, vp, vp, C.c_size_t, vp]
    _lib = L
    return L


def _alive() -> bool:
    """False once the interpreter is shutting down (module globals are being cleared)."""
    import sys
    return _lib is not None and lib is not None and not sys.is_finalizing()


def _check(rc: int) -> int:
    if rc < 0:
        raise AnpdError(rc, lib().anpd_last_error().decode("utf-8", "replace"))
    return rc


def _ints(seq: Sequence[int]):
    return (C.c_int32 * max(1, len(seq)))(*[int(t) for t in seq])


# --------------------------------------------------------------- host table

class NgramTable:
    """anpd_ngram_*: the adaptive multi-level N-gram drafter (host)."""

    def __init__(self, n_min: int, n_max: int, vocab: int):
        h = C.c_void_p()
        _check(lib().anpd_ngram_create(n_min, n_max, vocab, C.byref(h)))
        self._h = h

    def close(self):
        try:
            if getattr(self, "_h", None) and _alive():
                lib().anpd_ngram_destroy(self._h)
        except TypeError:   # interpreter shutdown: this module's globals are already gone
            pass
        self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def reset(self) -> None:
        _check(lib().anpd_ngram_reset(self._h))

    def update(self, tokens: Sequence[int]) -> int:
        return _check(lib().anpd_ngram_update(self._h, _ints(tokens), len(tokens)))

    def __len__(self) -> int:
        return int(lib().anpd_ngram_length(self._h))

    def query(self, tail: Sequence[int]) -> Tuple[Optional[int], int]:
        tok, lvl = C.c_int32(-1), C.c_int32(0)
        hit = _check(lib().anpd_ngram_query(self._h, _ints(tail), len(tail), C.byref(tok), C.byref(lvl)))
        return (tok.value, lvl.value) if hit else (None, 0)

    def propose(self, max_k: int) -> Tuple[List[int], List[int]]:
        toks, lvls = (C.c_int32 * max(1, max_k))(), (C.c_int32 * max(1, max_k))()
        n = _check(lib().anpd_ngram_propose(self._h, max_k, toks, lvls))
        return list(toks[:n]), list(lvls[:n])


# ------------------------------------------------------------- device side

def _propose_tree(self, max_k: int, n_cand: int, max_drafts: int):
    """anpd_ngram_propose_tree: (tokens, parents, levels) of the drafts; draft i is window row i + 1."""
    n = max(1, max_drafts)
    toks, pars, lvls = (C.c_int32 * n)(), (C.c_int32 * n)(), (C.c_int32 * n)()
    k = _check(lib().anpd_ngram_propose_tree(self._h, max_k, n_cand, max_drafts, toks, pars, lvls))
    return list(toks[:k]), list(pars[:k]), list(lvls[:k])


NgramTable.propose_tree = _propose_tree


def _stream_ptr(stream) -> int:
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


class Model:
    """anpd_model_*: borrows torch CUDA weight tensors, owns a workspace tensor."""

    def __init__(self, shape, weights: Dict[str, object], max_window: int = 8, max_positions: int = 1024,
                 page_tokens: int = 16, gemm_path: int = GEMM_AUTO, stream=None):
        import torch
        self.shape = shape
        self.vocab = shape.vocab
        self.weights = weights  # keep the tensors alive
        want = torch.bfloat16 if shape.dtype == "bf16" else torch.float32
        cfg = ModelCfg(shape.n_layers, shape.d_model, shape.n_heads, shape.head_dim, shape.d_ffn, shape.vocab,
                       shape.rms_eps, shape.rope_base, BF16 if shape.dtype == "bf16" else F32, page_tokens,
                       max_window, max_positions, gemm_path, int(getattr(shape, "n_kv_heads", 0) or 0))
        self.cfg = cfg

        def ptr(t):
            if not (t.is_cuda and t.is_contiguous() and t.dtype == want):
                raise ValueError("weights must be contiguous CUDA tensors of the model dtype")
            return t.data_ptr()

        ws = Weights()
        for name in ("embed", "final_norm", "lm_head"):
            setattr(ws, name, ptr(weights[name]))
        self._arrays = []
        for name in _PER_LAYER:
            arr = (C.c_void_p * shape.n_layers)(*[ptr(t) for t in weights[name]])
            self._arrays.append(arr)
            setattr(ws, name, C.cast(arr, C.POINTER(C.c_void_p)))
        nbytes = lib().anpd_model_workspace_bytes(C.byref(cfg))
        if nbytes == 0:
            _check(E_INVAL)
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=weights["embed"].device)
        h = C.c_void_p()
        _check(lib().anpd_model_create(C.byref(cfg), C.byref(ws), self.workspace.data_ptr(), nbytes,
                                       _stream_ptr(stream), C.byref(h)))
        self._h = h
        self.device = weights["embed"].device
        self.max_window = max_window

    def close(self):
        try:
            if getattr(self, "_h", None) and _alive():
                lib().anpd_model_destroy(self._h)
        except TypeError:   # interpreter shutdown: this module's globals are already gone
            pass
        self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def trace(self, enable: bool):
        """Barrier timestamps of the one-kernel step: returns an int64 CUDA tensor [grid][1024] (or None)."""
        import torch
        if not enable:
            _check(lib().anpd_model_trace(self._h, None, 0))
            self._trace = None
            return None
        grid = _check(lib().anpd_model_trace(self._h, None, 0))
        if grid == 0:
            return None
        self._trace = torch.zeros(grid, 1024, dtype=torch.int64, device=self.device)
        _check(lib().anpd_model_trace(self._h, self._trace.data_ptr(), self._trace.numel() * 8))
        return self._trace

    def set_barrier_spin_limit(self, spins: int) -> None:
        """Test hook: polls before a grid-barrier wait of the one-kernel step gives up (0 = default)."""
        _check(lib().anpd_model_set_barrier_spin_limit(self._h, spins))

    def profile(self, enable: bool) -> None:
        _check(lib().anpd_model_profile(self._h, 1 if enable else 0))

    def profile_read(self) -> Dict[str, object]:
        n = len(PROF_CATEGORIES)
        ms, cnt, steps = (C.c_double * n)(), (C.c_int64 * n)(), C.c_int64(0)
        _check(lib().anpd_model_profile_read(self._h, ms, cnt, C.byref(steps)))
        return {"steps": steps.value, "ms": dict(zip(PROF_CATEGORIES, list(ms))),
                "intervals": dict(zip(PROF_CATEGORIES, list(cnt)))}


def _settled(nbytes: int, device):
    """Memory that calls on any stream are going to use: what its last owner may still do with it, on the current stream, is
    waited for."""
    import torch
    t = torch.empty(nbytes, dtype=torch.uint8, device=device)
    torch.cuda.current_stream(t.device).synchronize()
    return t


class KVCache:
    """anpd_kv_*: one sequence's paged KV cache in a torch-allocated pool."""

    def __init__(self, model: Model, max_tokens: int):
        import torch
        self.model = model
        nbytes = lib().anpd_kv_pool_bytes(model._h, max_tokens)
        if nbytes == 0:
            _check(E_INVAL)
        self.pool = _settled(nbytes, model.device)
        h = C.c_void_p()
        _check(lib().anpd_kv_create(model._h, self.pool.data_ptr(), nbytes, max_tokens, C.byref(h)))
        self._h = h
        self.max_tokens = max_tokens
        self.n_layers = model.shape.n_layers
        self.n_kv_heads = int(getattr(model.shape, "n_kv_heads", 0) or model.shape.n_heads)

    def close(self):
        try:
            if getattr(self, "_h", None) and _alive():
                lib().anpd_kv_destroy(self._h)
        except TypeError:   # interpreter shutdown: this module's globals are already gone
            pass
        self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def length(self) -> int:
        return _check(lib().anpd_kv_length(self._h))

    @property
    def num_pages(self) -> int:
        return _check(lib().anpd_kv_num_pages(self._h))

    def truncate(self, new_len: int, stream=None) -> None:
        _check(lib().anpd_kv_truncate(self._h, new_len, _stream_ptr(stream)))

    def set_page_order(self, perm: Sequence[int]) -> None:
        _check(lib().anpd_kv_set_page_order(self._h, _ints(perm), len(perm)))

    def write(self, layer: int, pos0: int, k, v, stream=None) -> None:
        """k, v: CUDA float32 [n][n_kv_heads * head_dim]."""
        import torch
        n = k.shape[0] if k.dim() else 0
        for t in (k, v):
            if not (t.device == self.pool.device and t.dtype == torch.float32 and t.is_contiguous()
                    and t.dim() >= 2 and t.shape[0] == n and t.numel() == n * self.n_kv_heads * self.model.shape.head_dim):
                raise ValueError("k and v: contiguous float32 [positions][n_kv_heads * head_dim] on the cache's device")
        _check(lib().anpd_kv_write(self._h, layer, pos0, n, k.data_ptr(), v.data_ptr(), _stream_ptr(stream)))

    def read(self, layer: int, pos0: int, n: int, stream=None):
        import torch
        d = self.n_kv_heads * self.model.shape.head_dim
        k, v = (_empty((n, d), torch.float32, self.pool.device, stream) for _ in range(2))
        _check(lib().anpd_kv_read(self._h, layer, pos0, n, k.data_ptr(), v.data_ptr(), _stream_ptr(stream)))
        return k, v

    def commit(self, rows: Sequence[int], stream=None) -> None:
        """anpd_kv_commit: the rows of a tree that were accepted (a path from the root) move together behind the committed positions."""
        if any(not -1 << 31 <= r < 1 << 31 for r in rows):     # (the array would take their last 32 bits)
            raise ValueError("rows of a tree")
        _check(lib().anpd_kv_commit(self._h, _ints(rows), len(rows), _stream_of(self.pool.device, stream)))

    def observe(self, mass, rows: int = 32) -> None:
        """anpd_kv_observe: prompts into this cache add the weights of their last rows to mass, CUDA float32
        [n_layers][n_kv_heads][positions that they may reach], contiguous (None: no longer)."""
        import torch
        if mass is None:
            _check(lib().anpd_kv_observe(self._h, None, 0, 0, None, 0))
            self._observed = None
            return
        if not (mass.is_cuda and mass.device == self.pool.device and mass.dtype == torch.float32 and mass.dim() == 3 and mass.is_contiguous()
                and tuple(mass.shape[:2]) == (self.n_layers, self.n_kv_heads)):
            raise ValueError("mass: contiguous float32 [n_layers][n_kv_heads][positions] on the cache's device")
        nbytes = lib().anpd_kv_observe_workspace_bytes(self._h, rows)
        if nbytes == 0:
            _check(E_INVAL)
        ws = _settled(nbytes, mass.device)      # (prompts bring streams of their own)
        _check(lib().anpd_kv_observe(self._h, mass.data_ptr(), mass.shape[2], rows, ws.data_ptr(), nbytes))
        self._observed = (mass, ws)     # kept alive


def verify(model: Model, kv: KVCache, window: Sequence[int], mode: int = VERIFY, want_predicts: bool = False,
           out_logits=None, stream=None):
    """anpd_verify.  Returns (accepted, next) or (accepted, next, predicts)."""
    n = len(window)
    acc, nxt = C.c_int32(0), C.c_int32(0)
    preds = (C.c_int32 * max(1, n))() if want_predicts else None
    lp = 0
    if out_logits is not None:
        import torch
        assert out_logits.is_cuda and out_logits.dtype == torch.float32 and out_logits.is_contiguous()
        assert out_logits.numel() >= n * model.vocab
        lp = out_logits.data_ptr()
    _check(lib().anpd_verify(model._h, kv._h, _ints(window), n, mode, C.byref(acc), C.byref(nxt), preds, lp,
                             _stream_ptr(stream)))
    if want_predicts:
        return acc.value, nxt.value, list(preds[:n])
    return acc.value, nxt.value


def verify_tree(model: Model, kv: KVCache, window: Sequence[int], parent: Sequence[int], want_predicts: bool = False,
                out_logits=None, stream=None):
    """anpd_verify_tree.  Returns (accepted depth, next token, path rows) or with the per-row predictions appended."""
    n = len(window)
    assert len(parent) == n
    acc, nxt = C.c_int32(0), C.c_int32(0)
    path = (C.c_int32 * (n + 1))()
    preds = (C.c_int32 * max(1, n))() if want_predicts else None
    lp = 0
    if out_logits is not None:
        import torch
        assert out_logits.is_cuda and out_logits.dtype == torch.float32 and out_logits.is_contiguous()
        assert out_logits.numel() >= n * model.vocab
        lp = out_logits.data_ptr()
    _check(lib().anpd_verify_tree(model._h, kv._h, _ints(window), _ints(parent), n, C.byref(acc), C.byref(nxt), path, preds, lp,
                                  _stream_ptr(stream)))
    if want_predicts:
        return acc.value, nxt.value, list(path[:acc.value + 1]), list(preds[:n])
    return acc.value, nxt.value, list(path[:acc.value + 1])


def verify_batch(model: Model, kvs: Sequence[KVCache], windows: Sequence[Sequence[int]], mode: int = VERIFY,
                 out_logits=None, stream=None):
    """anpd_verify_batch: one step for several sequences.  Returns [(accepted, next)] per sequence."""
    n = len(kvs)
    assert len(windows) == n
    handles = (C.c_void_p * max(1, n))(*[kv._h for kv in kvs])
    rows = [_ints(w) for w in windows]
    wins = (C.POINTER(C.c_int32) * max(1, n))(*[C.cast(r, C.POINTER(C.c_int32)) for r in rows])
    counts = _ints([len(w) for w in windows])
    acc, nxt = (C.c_int32 * max(1, n))(), (C.c_int32 * max(1, n))()
    lp = 0
    if out_logits is not None:
        import torch
        assert out_logits.is_cuda and out_logits.dtype == torch.float32 and out_logits.is_contiguous()
        assert out_logits.numel() >= sum(len(w) for w in windows) * model.vocab
        lp = out_logits.data_ptr()
    _check(lib().anpd_verify_batch(model._h, handles, n, wins, counts, mode, acc, nxt, lp, _stream_ptr(stream)))
    return [(acc[i], nxt[i]) for i in range(n)]


def pack_weights(W, stream=None):
    """anpd_pack_weights: bf16 CUDA [N][K] -> fragment-order buffer (uint8 tensor)."""
    import torch
    N, K = W.shape
    assert W.is_cuda and W.dtype == torch.bfloat16 and W.is_contiguous()
    nb = lib().anpd_packed_bytes(N, K)
    if nb == 0:
        _check(E_INVAL)
    out = torch.empty(nb, dtype=torch.uint8, device=W.device)
    _check(lib().anpd_pack_weights(W.data_ptr(), N, K, out.data_ptr(), nb, _stream_ptr(stream)))
    return out


def linear(X, W, path: int, stream=None, packed=None, Y=None, workspace=None):
    """anpd_linear: Y = X @ W.T.  X: CUDA float32 [M][K]; W: CUDA [N][K] float32 or bfloat16.
    For the MFMA paths the weights are repacked first unless ``packed`` (from pack_weights) is given."""
    import torch
    M, K = X.shape
    N = W.shape[0]
    assert X.is_cuda and X.dtype == torch.float32 and X.is_contiguous() and W.is_contiguous() and W.shape[1] == K
    dtype = BF16 if W.dtype == torch.bfloat16 else F32
    if Y is None:
        Y = torch.empty(M, N, dtype=torch.float32, device=X.device)
    nb = lib().anpd_linear_workspace_bytes(M, K)
    ws = workspace if workspace is not None else torch.empty(max(nb, 256), dtype=torch.uint8, device=X.device)
    wptr = W.data_ptr()
    if path in (GEMM_MFMA, GEMM_MFMA_STREAM):
        if dtype != BF16:
            _check(lib().anpd_linear(X.data_ptr(), wptr, Y.data_ptr(), M, N, K, dtype, path, ws.data_ptr(), nb,
                                     _stream_ptr(stream)))
        if packed is None:
            packed = pack_weights(W, stream)
        wptr = packed.data_ptr()
    _check(lib().anpd_linear(X.data_ptr(), wptr, Y.data_ptr(), M, N, K, dtype, path, ws.data_ptr(), nb,
                             _stream_ptr(stream)))
    return Y


def linear_static(X, packed, N: int, Y, stream=None):
    """anpd_linear_static: Y = X @ W.T on the matrix cores with the library's built-in scratch; allocates
    nothing (the caller passes the output).  ``packed``: W as written by pack_weights."""
    M, K = X.shape
    _check(lib().anpd_linear_static(X.data_ptr(), packed.data_ptr(), Y.data_ptr(), M, N, K, _stream_ptr(stream)))
    return Y


# ------------------------------------------------------ operators on caches

class LayerCache(KVCache):
    """anpd_cache_create: a paged cache without a model, for programs whose layers are their own.  All of KVCache's
    methods; verify and prefill do not take it.  dtype "int8": keys and values as 8-bit codes with a scale for every position and
    head, which are quantised as they are written."""

    def __init__(self, n_layers: int, n_heads: int, head_dim: int, max_tokens: int, n_kv_heads: int = 0, dtype: str = "bf16",
                 page_tokens: int = 16, device="cuda"):
        import torch
        from types import SimpleNamespace
        types = {"bf16": BF16, "f32": F32, "int8": INT8}
        if dtype not in types:
            raise ValueError("dtype must be 'bf16', 'f32' or 'int8'")
        cfg = CacheCfg(n_layers, n_heads, head_dim, n_kv_heads, types[dtype], page_tokens)
        nbytes = lib().anpd_cache_pool_bytes(C.byref(cfg), max_tokens)
        if nbytes == 0:
            _check(E_INVAL)
        self.pool = _settled(nbytes, device)
        # (what KVCache asks of its model)
        self.model = SimpleNamespace(shape=SimpleNamespace(n_layers=n_layers, n_heads=n_heads, head_dim=head_dim, n_kv_heads=n_kv_heads or n_heads, dtype=dtype),
                                     device=self.pool.device)
        h = C.c_void_p()
        with torch.cuda.device(self.pool.device):
            _check(lib().anpd_cache_create(C.byref(cfg), self.pool.data_ptr(), nbytes, max_tokens, C.byref(h)))
        self._h = h
        self.max_tokens = max_tokens
        self.n_layers = n_layers
        self.n_kv_heads = n_kv_heads or n_heads


class AttentionRules:
    """anpd_attn_rules: the rules of the scores for attention() and key_mass(); keeps its tensors alive."""

    def __init__(self, scale: float = 0.0, cap: float = 0.0, window: int = 0, prefix: int = 0, slopes=None, first_key=None):
        import torch
        for t, dtype in ((slopes, torch.float32), (first_key, torch.int32)):
            if t is not None and not (t.is_cuda and t.dtype == dtype and t.is_contiguous()):
                raise ValueError("slopes: contiguous CUDA float32, first_key: contiguous CUDA int32")
        if not (0 <= window < 1 << 31 and 0 <= prefix < 1 << 31):     # (the struct would take their last 32 bits)
            raise ValueError("window and prefix must be in 0..2^31 - 1")
        self.slopes, self.first_key = slopes, first_key
        self.struct = AttnRules(scale, cap, window, prefix, None if slopes is None else slopes.data_ptr(),
                                None if first_key is None else first_key.data_ptr())
        self.ref = C.addressof(self.struct)


def _sequences(kvs, q, n_rows, pos0, rules):
    """(shape of the caches, n_seq, handles, rows, positions or None) for the calls on several caches."""
    import torch
    if isinstance(kvs, KVCache):
        kvs = (kvs,)
    n = len(kvs)
    if n == 0:
        raise ValueError("no cache")
    first = kvs[0]
    shape = first.model.shape
    if q.dim() != 2 or q.stride(1) != 1 or q.shape[1] != shape.n_heads * shape.head_dim or q.device != first.pool.device or q.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("rows must be a 2-d float32 or bfloat16 tensor on the caches' device, n_heads * head_dim wide")
    rows = q.shape[0]
    handles = (C.c_void_p * n)(*[kv._h.value for kv in kvs])
    if n_rows is None:      # the same number of each sequence
        if rows % n:
            raise ValueError("n_rows is needed: %d rows do not divide among %d sequences" % (rows, n))
        counts = (C.c_int32 * n)(*([rows // n] * n))
    else:
        if len(n_rows) != n or sum(n_rows) != rows or min(n_rows) < 0:
            raise ValueError("n_rows does not add up to the rows")
        counts = (C.c_int32 * n)(*n_rows)
    if pos0 is not None:
        if len(pos0) != n or max(pos0) >= 1 << 31 or min(pos0) < 0:
            raise ValueError("pos0: one position per sequence")
        pos0 = (C.c_int32 * n)(*pos0)
    if rules is not None:
        t = rules.slopes
        if t is not None and (t.numel() < shape.n_heads or t.device != q.device):
            raise ValueError("slopes: one per head, on the caches' device")
        t = rules.first_key
        if t is not None and (t.numel() < rows or t.device != q.device):
            raise ValueError("first_key: one per row, on the caches' device")
    return shape, n, handles, counts, pos0


def _pitch(t) -> int:
    """Elements between rows (of a single row, or none: its width)."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _stream_of(device, stream) -> int:
    """The stream of a call: the given one, or the device's current one."""
    if stream is not None:
        return stream.cuda_stream
    import torch
    return torch._C._cuda_getCurrentRawStream(device.index)


def _empty(shape, dtype, device, stream):
    """An output or workspace of a call on `stream` (None: the current one), from that stream's memory: what its last owner
    still does with it is done before."""
    import torch
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _with_workspace(fn, bytes_of, seqs, ref, head, tail, workspace, device, stream) -> None:
    """fn(*seqs, *head, workspace, its bytes, stream): most calls need no workspace, so how much is only asked for
    where none was given and the call says so."""
    st = _stream_of(device, stream)
    if workspace is not None:
        _check(fn(*seqs, *head, *tail, workspace.data_ptr(), workspace.numel() * workspace.element_size(), st))
        return
    rc = fn(*seqs, *head, *tail, None, 0, st)
    if rc == E_INVAL:
        nbytes = bytes_of(*seqs, ref)
        if nbytes:
            import torch
            ws = _empty(nbytes, torch.uint8, device, stream)
            rc = fn(*seqs, *head, *tail, ws.data_ptr(), nbytes, st)
        else:
            rc = fn(*seqs, *head, *tail, None, 0, st)   # (for its message)
    _check(rc)


def _workspace_bytes(fn, kvs, n_rows, pos0, rules) -> int:
    kvs = (kvs,) if isinstance(kvs, KVCache) else kvs
    return int(fn((C.c_void_p * len(kvs))(*[kv._h.value for kv in kvs]), len(kvs), _ints(n_rows), None if pos0 is None else _ints(pos0), None if rules is None else rules.ref))


def attention_workspace_bytes(kvs, n_rows: Sequence[int], pos0: Optional[Sequence[int]] = None, rules: Optional[AttentionRules] = None) -> int:
    """anpd_attention_workspace_bytes (0: none is needed)."""
    return _workspace_bytes(lib().anpd_attention_workspace_bytes, kvs, n_rows, pos0, rules)


def tree_attention_workspace_bytes(kvs, n_rows: Sequence[int], pos0: Optional[Sequence[int]] = None, rules: Optional[AttentionRules] = None) -> int:
    """anpd_tree_attention_workspace_bytes (0: none is needed)."""
    return _workspace_bytes(lib().anpd_tree_attention_workspace_bytes, kvs, n_rows, pos0, rules)


def attention(kvs, layer: int, q, n_rows: Optional[Sequence[int]] = None, pos0: Optional[Sequence[int]] = None,
              rules: Optional[AttentionRules] = None, out=None, lse=None, want_lse: bool = False, workspace=None, stream=None):
    """anpd_attention: new rows of one cache or of a list of caches over what is cached.  q: CUDA float32 or bfloat16
    [rows of all sequences][n_heads * head_dim].  Returns out, or (out, lse) where lse was given or asked for."""
    L = lib()
    return _attend(L.anpd_attention, L.anpd_attention_workspace_bytes, kvs, layer, q, (), n_rows, pos0, rules, out, lse, want_lse, workspace, stream)


def tree_attention(kvs, layer: int, q, parent, n_rows: Optional[Sequence[int]] = None, pos0: Optional[Sequence[int]] = None,
                   rules: Optional[AttentionRules] = None, out=None, lse=None, want_lse: bool = False, workspace=None, stream=None):
    """anpd_tree_attention: as attention(), where the new rows of every sequence are a tree of drafts.  parent: CUDA int32, for every
    row the row of its sequence that it continues, -1 for the root."""
    import torch
    if not (parent.device == q.device and parent.dtype == torch.int32 and parent.is_contiguous() and parent.dim() == 1 and parent.shape[0] == q.shape[0]):
        raise ValueError("parent: contiguous int32, one per row, on the caches' device")
    L = lib()
    return _attend(L.anpd_tree_attention, L.anpd_tree_attention_workspace_bytes, kvs, layer, q, (parent.data_ptr(),), n_rows, pos0, rules, out, lse, want_lse,
                   workspace, stream)


def _attend(fn, bytes_of, kvs, layer, q, tree, n_rows, pos0, rules, out, lse, want_lse, workspace, stream):
    import torch
    shape, n, handles, counts, at = _sequences(kvs, q, n_rows, pos0, rules)
    rows = q.shape[0]
    if out is None:
        out = _empty(q.shape, q.dtype, q.device, stream)
    elif not (out.device == q.device and out.dtype == q.dtype and out.shape == q.shape and out.stride(1) == 1):
        raise ValueError("out must be like the rows")
    if lse is not None:
        if not (lse.device == q.device and lse.dtype == torch.float32 and lse.is_contiguous() and tuple(lse.shape) == (rows, shape.n_heads)):
            raise ValueError("lse: contiguous float32 [rows][n_heads]")
    elif want_lse:
        lse = _empty((rows, shape.n_heads), torch.float32, q.device, stream)
    ref = None if rules is None else rules.ref
    _with_workspace(fn, bytes_of, (handles, n, counts, at), ref, (layer, q.data_ptr(), _pitch(q), F32 if q.dtype == torch.float32 else BF16, *tree, ref),
                    (out.data_ptr(), _pitch(out), None if lse is None else lse.data_ptr()), workspace, q.device, stream)
    return out if lse is None else (out, lse)


def key_mass(kvs, layer: int, q, lse, mass, n_rows: Optional[Sequence[int]] = None, pos0: Optional[Sequence[int]] = None,
             rules: Optional[AttentionRules] = None, workspace=None, stream=None):
    """anpd_key_mass: adds the rows' weights to mass and returns it.  mass: CUDA float32 [n_kv_heads][>= keys] for one
    cache, [sequences][n_kv_heads][>= keys] for several; rows apart as they like, keys side by side."""
    import torch
    shape, n, handles, counts, at = _sequences(kvs, q, n_rows, pos0, rules)
    each = mass if mass.dim() == 3 else mass[None]
    kv_heads = (kvs if isinstance(kvs, KVCache) else kvs[0]).n_kv_heads
    if not (mass.dtype == torch.float32 and mass.device == q.device and each.dim() == 3 and each.shape[0] == n and each.shape[1] == kv_heads and each.stride(2) == 1):
        raise ValueError("mass: float32 [sequences][n_kv_heads][keys] on the caches' device")
    if not (lse.device == q.device and lse.dtype == torch.float32 and lse.is_contiguous() and tuple(lse.shape) == (q.shape[0], shape.n_heads)):
        raise ValueError("lse: contiguous float32 [rows][n_heads]")
    ld = each.stride(1) if kv_heads > 1 else each.shape[2]
    if ld < each.shape[2] or any(c and c + (kv.length if at is None else at[i]) > each.shape[2]
                                 for i, (c, kv) in enumerate(zip(counts, (kvs,) if isinstance(kvs, KVCache) else kvs))):
        raise ValueError("mass has fewer columns than there are keys")
    step, base = each.stride(0) * 4, each.data_ptr()
    ptrs = (C.c_void_p * n)(*[base + i * step for i in range(n)])
    L, ref = lib(), None if rules is None else rules.ref
    _with_workspace(L.anpd_key_mass, L.anpd_key_mass_workspace_bytes, (handles, n, counts, at), ref,
                    (layer, q.data_ptr(), _pitch(q), F32 if q.dtype == torch.float32 else BF16, ref),
                    (lse.data_ptr(), ptrs, ld), workspace, q.device, stream)
    return mass


def evict(src: KVCache, mass, keep: int, first: int = 0, last: int = 0, into: Optional[KVCache] = None, rope_base: float = 0.0, stream=None):
    """anpd_kv_evict: `keep` positions of src stay, per layer and key / value head those with the largest mass, the
    first and last ones in any case; into: the cache that they move into (src itself if absent).  mass: CUDA float32
    [n_layers][n_kv_heads][>= length].  Returns (positions [n_layers][n_kv_heads][keep] int32, their mass)."""
    import torch
    if not (mass.is_cuda and mass.device == src.pool.device and mass.dtype == torch.float32 and mass.dim() == 3 and mass.stride(2) == 1):
        raise ValueError("mass: float32 [n_layers][n_kv_heads][positions] on the cache's device")
    layers, kv_heads = src.n_layers, src.n_kv_heads
    # elements between rows: of heads, of layers where there is one head, of a single row its length
    ld = mass.stride(1) if kv_heads > 1 else mass.stride(0) if layers > 1 else mass.shape[2]
    if mass.shape[:2] != (layers, kv_heads) or mass.shape[2] < src.length or (layers > 1 and mass.stride(0) != kv_heads * ld):
        raise ValueError("mass: one row of at least the cache's length per layer and key / value head, equally far apart")
    kept = _empty((layers, kv_heads, max(0, keep)), torch.int32, mass.device, stream)
    out = _empty((layers, kv_heads, max(0, keep)), torch.float32, mass.device, stream)
    dst = src if into is None else into
    _check(lib().anpd_kv_evict(src._h, dst._h, mass.data_ptr(), ld, keep, first, last, rope_base, kept.data_ptr(), out.data_ptr(), max(0, keep),
                               _stream_of(mass.device, stream)))
    return kept, out


def _span_of(kvs, n_rows, pos0):
    """(caches, n_seq, handles, rows, positions or None) of store() and load()."""
    if isinstance(kvs, KVCache):
        kvs = (kvs,)
    n = len(kvs)
    if n == 0 or len(n_rows) != n or min(n_rows) < 0 or max(n_rows) >= 1 << 31:
        raise ValueError("n_rows: one number per cache")
    if pos0 is not None and (len(pos0) != n or max(pos0) >= 1 << 31 or min(pos0) < 0):
        raise ValueError("pos0: one position per sequence")
    return kvs, n, (C.c_void_p * n)(*[kv._h for kv in kvs]), (C.c_int32 * n)(*n_rows), None if pos0 is None else (C.c_int32 * n)(*pos0)


def _check_rows(t, rows: int, kv, dtype) -> None:
    if not (t.device == kv.pool.device and t.dtype == dtype and t.dim() == 2 and tuple(t.shape) == (rows, kv.n_kv_heads * kv.model.shape.head_dim)
            and (t.stride(1) == 1 or rows == 0)):
        raise ValueError("k and v: float32 or bfloat16 [rows][n_kv_heads * head_dim] on the caches' device, alike")


def store(kvs, layer: int, k, v, n_rows: Optional[Sequence[int]] = None, pos0: Optional[Sequence[int]] = None, stream=None) -> None:
    """anpd_kv_store: new rows' keys and values into one cache or a list of caches, rounded to their type or quantised.  k, v: CUDA
    float32 or bfloat16 [rows of all sequences][n_kv_heads * head_dim]."""
    import torch
    if n_rows is None:      # the same number of each sequence
        n = 1 if isinstance(kvs, KVCache) else len(kvs)
        if n == 0 or k.shape[0] % n:
            raise ValueError("n_rows is needed: %d rows do not divide among %d sequences" % (k.shape[0], n))
        n_rows = [k.shape[0] // n] * n
    kvs, n, handles, counts, at = _span_of(kvs, n_rows, pos0)
    if k.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("k and v must be float32 or bfloat16")
    rows = sum(n_rows)
    for t in (k, v):
        _check_rows(t, rows, kvs[0], k.dtype)
    _check(lib().anpd_kv_store(handles, n, counts, at, layer, k.data_ptr(), _pitch(k), v.data_ptr(), _pitch(v), F32 if k.dtype == torch.float32 else BF16,
                               _stream_of(kvs[0].pool.device, stream)))


def load(kvs, layer: int, n_rows: Sequence[int], pos0: Optional[Sequence[int]] = None, dtype=None, k=None, v=None, stream=None):
    """anpd_kv_load: (k, v) of n_rows positions of each cache from its committed length (or pos0) on, in dtype (float32 if absent), into
    k and v where given."""
    import torch
    kvs, n, handles, counts, at = _span_of(kvs, n_rows, pos0)
    if dtype is None:
        dtype = torch.float32 if k is None else k.dtype
    if dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("dtype must be float32 or bfloat16")
    rows, first = sum(n_rows), kvs[0]
    shape = (rows, first.n_kv_heads * first.model.shape.head_dim)
    k, v = (_empty(shape, dtype, first.pool.device, stream) if t is None else t for t in (k, v))
    for t in (k, v):
        _check_rows(t, rows, first, dtype)
    _check(lib().anpd_kv_load(handles, n, counts, at, layer, k.data_ptr(), _pitch(k), v.data_ptr(), _pitch(v), F32 if dtype == torch.float32 else BF16,
                              _stream_of(first.pool.device, stream)))
    return k, v


# --------------------------------------------------------- drawing of tokens

class SamplingRules:
    """anpd_sample_rules: which tokens may be drawn.  A number for all rows, or a CUDA tensor with one for each (float32, top_k int32); keeps
    its tensors alive."""

    def __init__(self, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
        import torch
        self.struct, self.tensors = SampleRules(1.0, 0, 1.0, 0.0), {}
        for name, value in (("temperature", temperature), ("top_k", top_k), ("top_p", top_p), ("min_p", min_p)):
            if isinstance(value, torch.Tensor):
                if not (value.is_cuda and value.is_contiguous() and value.dim() == 1 and value.dtype == (torch.int32 if name == "top_k" else torch.float32)):
                    raise ValueError("%s: contiguous CUDA %s, one per row" % (name, "int32" if name == "top_k" else "float32"))
                self.tensors[name] = value
                setattr(self.struct, name + "s", value.data_ptr())
            elif name == "top_k" and not 0 <= value < 1 << 31:      # (the struct would take its last 32 bits)
                raise ValueError("top_k must be in 0..2^31 - 1")
            else:
                setattr(self.struct, name, value)
        self.ref = C.addressof(self.struct)

    def check(self, rows: int, device) -> None:
        for name, t in self.tensors.items():
            if t.numel() < rows or t.device != device:
                raise ValueError("%s: one per row, on the logits' device" % name)


def sample_workspace_bytes(rows: int, vocab: int) -> int:
    """anpd_sample_workspace_bytes (0: none is needed)."""
    return int(lib().anpd_sample_workspace_bytes(rows, vocab))


def _sample_workspace(workspace, rows: int, vocab: int, device, stream):
    """(kept alive, pointer, bytes) of the given workspace, or of one from the call's stream's memory."""
    if workspace is None:
        nbytes = sample_workspace_bytes(rows, vocab) if vocab > 8192 else 0
        if nbytes == 0:
            return None, None, 0
        import torch
        workspace = _empty(nbytes, torch.uint8, device, stream)
    elif workspace.device != device or not workspace.is_contiguous():
        raise ValueError("workspace: contiguous, on the logits' device")
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def sample(logits, uniform, rules: Optional[SamplingRules] = None, tokens=None, logprob=None, want_logprob: bool = False, workspace=None, stream=None):
    """anpd_sample: a token for each row of logits (CUDA float32 or bfloat16 [rows][vocab]) by random numbers in [0, 1) (float32 [rows]).
    Returns int32 tokens, or (tokens, logprob) where logprob was given or asked for."""
    import torch
    if logits.dim() != 2 or not logits.is_cuda or logits.dtype not in (torch.float32, torch.bfloat16) or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError("logits must be a 2-d CUDA float32 or bfloat16 tensor, tokens side by side")
    rows, device = logits.shape[0], logits.device
    if not (uniform.device == device and uniform.dtype == torch.float32 and uniform.is_contiguous() and tuple(uniform.shape) == (rows,)):
        raise ValueError("uniform: contiguous float32, one per row, on the logits' device")
    if rules is not None:
        rules.check(rows, device)
    if tokens is None:
        tokens = _empty((rows,), torch.int32, device, stream)
    elif not (tokens.device == device and tokens.dtype == torch.int32 and tokens.is_contiguous() and tuple(tokens.shape) == (rows,)):
        raise ValueError("tokens: contiguous int32, one per row")
    if logprob is not None:
        if not (logprob.device == device and logprob.dtype == torch.float32 and logprob.is_contiguous() and tuple(logprob.shape) == (rows,)):
            raise ValueError("logprob: contiguous float32, one per row")
    elif want_logprob:
        logprob = _empty((rows,), torch.float32, device, stream)
    _keep, at, nbytes = _sample_workspace(workspace, rows, logits.shape[1], device, stream)
    _check(lib().anpd_sample(logits.data_ptr(), _pitch(logits), F32 if logits.dtype == torch.float32 else BF16, rows, logits.shape[1],
                             None if rules is None else rules.ref, uniform.data_ptr(), tokens.data_ptr(), None if logprob is None else logprob.data_ptr(),
                             at, nbytes, _stream_of(device, stream)))
    return tokens if logprob is None else (tokens, logprob)


def verify_sample(model: Model, kv: KVCache, window: Sequence[int], uniform, rules: Optional[SamplingRules] = None, out_logits=None, workspace=None,
                  stream=None):
    """anpd_verify_sample: a verification step that draws its tokens.  uniform: CUDA float32, one per window row.  Returns
    (accepted, next, tokens drawn after every row)."""
    import torch
    n = len(window)
    device = kv.pool.device
    if not (uniform.device == device and uniform.dtype == torch.float32 and uniform.is_contiguous() and tuple(uniform.shape) == (n,)):
        raise ValueError("uniform: contiguous float32, one per window row, on the cache's device")
    if rules is not None:
        rules.check(n, device)
    if out_logits is None:
        out_logits = _empty((n, model.vocab), torch.float32, device, stream)
    elif not (out_logits.device == device and out_logits.dtype == torch.float32 and out_logits.is_contiguous() and out_logits.numel() >= n * model.vocab):
        raise ValueError("out_logits: contiguous float32 [window rows][vocab] on the cache's device")
    _keep, at, nbytes = _sample_workspace(workspace, n, model.vocab, device, stream)
    acc, nxt, drawn = C.c_int32(0), C.c_int32(0), (C.c_int32 * max(1, n))()
    _check(lib().anpd_verify_sample(model._h, kv._h, _ints(window), n, None if rules is None else rules.ref, uniform.data_ptr(), C.byref(acc), C.byref(nxt), drawn,
                                    out_logits.data_ptr(), at, nbytes, _stream_of(device, stream)))
    return acc.value, nxt.value, list(drawn[:n])


# ------------------------------------------------------------ decode loops

def prefill_workspace_bytes(model: Model, n_tokens: int) -> int:
    """anpd_prefill_workspace_bytes (0 for models that process the prompt in windows)."""
    return int(lib().anpd_prefill_workspace_bytes(model._h, n_tokens))


def prefill(model: Model, kv: KVCache, prompt: Sequence[int], stream=None, out_logits=None, workspace=None) -> int:
    """anpd_prefill: LLM(prompt) of Algorithm 1, all rows in one pass; returns the greedy token
    after the prompt.  ``out_logits``: CUDA float32 [vocab] for the last row's logits.
    ``workspace``: a CUDA uint8 tensor to reuse (allocated here if absent)."""
    import torch
    n = len(prompt)
    nb = prefill_workspace_bytes(model, n) if n >= 1 else 0
    ws = workspace
    if ws is None or ws.numel() < nb:
        ws = _empty(max(nb, 256), torch.uint8, kv.pool.device, stream)
    lp = 0
    if out_logits is not None:
        assert out_logits.is_cuda and out_logits.dtype == torch.float32 and out_logits.is_contiguous()
        assert out_logits.numel() >= model.vocab
        lp = out_logits.data_ptr()
    nxt = C.c_int32(0)
    _check(lib().anpd_prefill(model._h, kv._h, _ints(prompt), n, C.byref(nxt), lp, ws.data_ptr(), ws.numel(),
                              _stream_ptr(stream)))
    return nxt.value


def prefill_windows(model: Model, kv: KVCache, prompt: Sequence[int], stream=None) -> int:
    """The prompt appended through the verification step in windows of max_window rows (what
    anpd_prefill replaces on the matrix-core path); returns the greedy token after it."""
    nxt = -1
    for lo in range(0, len(prompt), model.max_window):
        _, nxt = verify(model, kv, prompt[lo:lo + model.max_window], APPEND, stream=stream)
    return nxt


def greedy_generate(model: Model, kv: KVCache, prompt: Sequence[int], n_tokens: int, stream=None) -> List[int]:
    """Plain autoregressive decoding: windows of one row."""
    c = prefill(model, kv, prompt, stream)
    out: List[int] = []
    while len(out) < n_tokens:
        out.append(c)
        _, c = verify(model, kv, [c], VERIFY, stream=stream)
    return out


def adaptive_draft_length(levels: Sequence[int], k_max: int) -> int:
    """Draft length chosen from the level that answered the first draft: 2^(level - 2), capped
    (level 2 -> 1 draft, 3 -> 2, 4 -> 4, 5 -> 8, 6 -> 16); no answer -> no drafts."""
    if not levels:
        return 0
    return max(1, min(k_max, 1 << (levels[0] - 2)))


def anpd_generate_multi(model: Model, kv: KVCache, table: NgramTable, prompt: Sequence[int], K: int, n_cand: int,
                        n_tokens: int, stream=None) -> Dict[str, object]:
    """Algorithm 1 with multi-candidate verification: every step drafts up to n_cand candidate
    continuations (NgramTable.propose_tree), scores them in one forward (verify_tree) and keeps the
    longest accepted one."""
    table.reset()
    table.update(prompt)
    c = prefill(model, kv, prompt, stream)
    out: List[int] = []
    steps = proposed = accepted = rows = 0
    while len(out) < n_tokens:
        table.update([c])
        out.append(c)
        toks, pars, _ = table.propose_tree(K, n_cand, model.max_window - 1)
        a, nxt, path = verify_tree(model, kv, [c] + toks, [-1] + pars, stream=stream)
        kept = [toks[r - 1] for r in path[1:]]
        if kept:
            table.update(kept)
            out.extend(kept)
        steps += 1
        proposed += len(toks)
        rows += 1 + len(toks)
        accepted += a
        c = nxt
    return {"tokens": out[:n_tokens], "n_steps": steps, "proposed": proposed, "accepted": accepted, "rows": rows}


def anpd_generate(model: Model, kv: KVCache, table: NgramTable, prompt: Sequence[int], K: int, n_tokens: int,
                  stream=None, drafter=None, adaptive: bool = False, sampling: Optional[SamplingRules] = None, generator=None) -> Dict[str, object]:
    """Algorithm 1: commit, draft K tokens from the table, verify, accept the
    matching prefix, continue from the LLM's own token.  ``adaptive`` cuts the
    drafts of a step to adaptive_draft_length().  ``sampling``: tokens are drawn by these rules (numbers, not tensors per row) instead of
    taken greedily, with random numbers from ``generator`` (torch, of the model's device; absent: its default one)."""
    import torch
    if sampling is not None and sampling.tensors:
        raise ValueError("sampling: the same rules for all rows")
    side = contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)
    uniform = lambda n: torch.rand(n, generator=generator, dtype=torch.float32, device=kv.pool.device)  # noqa: E731
    table.reset()
    table.update(prompt)
    if sampling is None:
        c = prefill(model, kv, prompt, stream)
    else:
        with side:
            logits = torch.empty(max(1, model.max_window), model.vocab, dtype=torch.float32, device=kv.pool.device)
            prefill(model, kv, prompt, stream, out_logits=logits[0])
            c = int(sample(logits[:1], uniform(1), sampling, stream=stream))
    out: List[int] = []
    steps = proposed = accepted = 0
    while len(out) < n_tokens:
        table.update([c])
        out.append(c)
        if drafter is not None:
            drafts = drafter(len(out), K)
        else:
            drafts, levels = table.propose(K)
            if adaptive:
                drafts = drafts[:adaptive_draft_length(levels, K)]
        if sampling is None:
            a, nxt = verify(model, kv, [c] + drafts, VERIFY, stream=stream)
        else:
            with side:
                a, nxt, _ = verify_sample(model, kv, [c] + drafts, uniform(1 + len(drafts)), sampling,
                                          out_logits=logits, stream=stream)
        if a:
            table.update(drafts[:a])
            out.extend(drafts[:a])
        steps += 1
        proposed += len(drafts)
        accepted += a
        c = nxt
    return {"tokens": out[:n_tokens], "n_steps": steps, "proposed": proposed, "accepted": accepted}
