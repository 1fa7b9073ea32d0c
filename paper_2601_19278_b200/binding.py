"""Thin ctypes binding of ``libdart.so`` (the C ABI declared in ``include/dart.h``).

Argument marshalling only: torch provides device memory and streams, every step of the
drafting path runs in the library's CUDA kernels.  There is no fallback: if the shared
library is missing or fails to load, importing callers get an exception.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import Dict, Optional

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# DART_LIB: load another build of the same library instead (the tests run once against the -DDART_DEBUG build)
LIB_PATH = os.environ.get("DART_LIB") or os.path.join(_HERE, "libdart.so")

DART_OK = 0
DART_ERR_INVALID_ARG = -1
DART_ERR_UNSUPPORTED_ARCH = -2
DART_ERR_CUDA = -3
DART_ERR_CAPACITY = -4
DART_ERR_TIMEOUT = -5
DART_ERR_INTERNAL = -6

EXPORTS = [
    "dart_draft_init", "dart_draft_step", "dart_build_tree", "dart_draft_destroy", "dart_last_device_status",
    "dart_last_cuda_error", "dart_status_string", "dart_workspace_bytes", "dart_ngram_bytes", "dart_train_attention_fwd", "dart_step_launch_count", "dart_draft_prefill", "dart_tree_verify_inputs",
    "dart_set_profile_events", "dart_topk_rows_noalloc", "dart_selftest_bounded_wait", "dart_draft_step_host",
    "dart_kv8_attention", "dart_kv8_attention_workspace_bytes", "dart_kv8_append", "dart_kv8_append_owned", "dart_kv8_fork", "dart_kv8_reserve", "dart_kv8_release",
    "dart_kv8_compact", "dart_kv8_pages_workspace_bytes", "dart_selftest_kv8_wait", "dart_selftest_kv8_window_wait",
    "dart_kv8_attention_plan", "dart_kv8_attention_window", "dart_kv8_attention_window_workspace_bytes", "dart_kv8_attention_window_plan",
    "dart_kv8_trim", "dart_rope_frequencies", "dart_qk_norm_rope", "dart_token_logprobs", "dart_token_logprobs_workspace_bytes",
]


class DartConfig(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("hidden", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
        ("head_dim", C.c_int32), ("mlp_inter", C.c_int32), ("vocab", C.c_int32), ("feat_in", C.c_int32),
        ("max_batch", C.c_int32), ("max_prefix", C.c_int32), ("K", C.c_int32), ("topk", C.c_int32),
        ("beam", C.c_int32), ("tree_budget", C.c_int32), ("ngram_order", C.c_int32),
        ("rope_theta", C.c_float), ("rms_eps", C.c_float), ("w_ng", C.c_float), ("logit_decay", C.c_float),
        ("level_exp", C.c_float), ("eps_logit", C.c_float), ("eps_ng", C.c_float), ("temperature", C.c_float),
        ("philox_seed", C.c_uint64), ("ngram_layout", C.c_int32), ("reserved0", C.c_int32),
    ]


NGRAM_HASH, NGRAM_TRIE = 0, 1


class DartTrainAttnIn(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("prompt_len", C.c_int32), ("draft_len", C.c_int32), ("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p),
                ("seq_lens_host", C.c_void_p), ("out", C.c_void_p), ("status", C.c_void_p)]


WEIGHT_NAMES = ["w_fc", "embed", "mask_vec", "norm_g", "norm_e", "w_q", "w_k", "w_v", "w_o", "norm_post",
                "w_gate", "w_up", "w_down", "norm_final", "w_lm"]


class DartWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in WEIGHT_NAMES]


class DartNgramHost(C.Structure):
    _fields_ = [("n_rows", C.c_int64), ("order", C.c_void_p), ("ctx0", C.c_void_p), ("ctx1", C.c_void_p),
                ("next", C.c_void_p), ("score", C.c_void_p)]


class DartStepIn(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_fresh", C.c_int32), ("feats", C.c_void_p), ("tokens", C.c_void_p),
                ("seq_lens", C.c_void_p), ("seq_lens_host", C.c_void_p), ("k_cache", C.c_void_p),
                ("v_cache", C.c_void_p), ("step_counter", C.c_uint64), ("fresh_counts_host", C.c_void_p)]


class DartPrefillIn(C.Structure):
    _fields_ = [("batch", C.c_int32), ("feats", C.c_void_p), ("tokens", C.c_void_p), ("seq_lens_host", C.c_void_p),
                ("new_rows_host", C.c_void_p), ("k_cache", C.c_void_p), ("v_cache", C.c_void_p)]


class DartVerifyIn(C.Structure):
    _fields_ = [("batch", C.c_int32), ("max_levels", C.c_int32), ("parents", C.c_void_p), ("depth", C.c_void_p),
                ("n_nodes", C.c_void_p), ("root_pos", C.c_void_p)]


class DartVerifyOut(C.Structure):
    _fields_ = [("position_ids", C.c_void_p), ("retrieve", C.c_void_p), ("n_leaves", C.c_void_p)]


class DartStepOut(C.Structure):
    _fields_ = [("topk_ids", C.c_void_p), ("topk_slogit", C.c_void_p), ("logits", C.c_void_p)]


class DartTreeIn(C.Structure):
    _fields_ = [("batch", C.c_int32), ("first_row", C.c_int32), ("n_levels", C.c_int32), ("topk_ids", C.c_void_p),
                ("topk_slogit", C.c_void_p), ("ctx_tail", C.c_void_p), ("first_rows_host", C.c_void_p)]


class DartTreeOut(C.Structure):
    _fields_ = [("tokens", C.c_void_p), ("parents", C.c_void_p), ("depth", C.c_void_p), ("mask", C.c_void_p),
                ("n_nodes", C.c_void_p), ("scores", C.c_void_p)]


class DartHostIo(C.Structure):
    _fields_ = [("in_host", C.c_void_p), ("in_dev", C.c_void_p), ("in_bytes", C.c_size_t),
                ("out_dev", C.c_void_p), ("out_host", C.c_void_p), ("out_bytes", C.c_size_t)]


KV8_E4M3, KV8_INT8 = 0, 1


class DartKv8Cache(C.Structure):
    _fields_ = [("format", C.c_int32), ("n_layers", C.c_int32), ("n_pages", C.c_int32), ("n_kv_heads", C.c_int32),
                ("page_tokens", C.c_int32), ("head_dim", C.c_int32), ("k_pages", C.c_void_p), ("v_pages", C.c_void_p),
                ("k_scale", C.c_void_p), ("v_scale", C.c_void_p)]


class DartKv8AttnIn(C.Structure):
    _fields_ = [("layer", C.c_int32), ("batch", C.c_int32), ("rows", C.c_int32), ("n_q_heads", C.c_int32), ("max_seqs", C.c_int32),
                ("max_pages", C.c_int32), ("max_len", C.c_int32), ("q", C.c_void_p), ("k_new", C.c_void_p), ("v_new", C.c_void_p),
                ("q_stride", C.c_int64), ("new_stride", C.c_int64), ("slots", C.c_void_p), ("seq_lens", C.c_void_p),
                ("page_table", C.c_void_p), ("n_rows", C.c_void_p), ("mask", C.c_void_p), ("out", C.c_void_p), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_size_t), ("status", C.c_void_p)]


class DartKv8AppendIn(C.Structure):
    _fields_ = [("first_layer", C.c_int32), ("n_layers", C.c_int32), ("batch", C.c_int32), ("rows", C.c_int32), ("max_append", C.c_int32),
                ("max_seqs", C.c_int32), ("max_pages", C.c_int32), ("k_new", C.c_void_p), ("v_new", C.c_void_p), ("row_stride", C.c_int64),
                ("layer_stride", C.c_int64), ("slots", C.c_void_p), ("seq_lens", C.c_void_p), ("page_table", C.c_void_p),
                ("n_append", C.c_void_p), ("row_index", C.c_void_p), ("status", C.c_void_p)]


class DartKv8Plan(C.Structure):
    _fields_ = [("many_rows", C.c_int32), ("row_tiles", C.c_int32), ("paired", C.c_int32), ("keys_per_part", C.c_int32), ("max_parts", C.c_int32)]


class DartKv8Pages(C.Structure):
    _fields_ = [("n_pages", C.c_int32), ("page_tokens", C.c_int32), ("max_seqs", C.c_int32), ("max_pages", C.c_int32),
                ("page_table", C.c_void_p), ("seq_lens", C.c_void_p), ("ref_count", C.c_void_p)]


class DartKv8Window(C.Structure):
    _fields_ = [("window", C.c_int32), ("sinks", C.c_int32), ("positions", C.c_void_p)]


DART_BF16, DART_FP16, DART_FP32 = 0, 1, 2
KV8_GIVEN_BACK = -2


class DartQkRopeIn(C.Structure):
    _fields_ = [("batch", C.c_int32), ("rows", C.c_int32), ("n_q_heads", C.c_int32), ("n_k_heads", C.c_int32), ("head_dim", C.c_int32),
                ("rotary_dim", C.c_int32), ("interleaved", C.c_int32), ("dtype", C.c_int32), ("max_seqs", C.c_int32), ("eps", C.c_float),
                ("q", C.c_void_p), ("k", C.c_void_p), ("q_out", C.c_void_p), ("k_out", C.c_void_p), ("q_stride", C.c_int64),
                ("k_stride", C.c_int64), ("q_out_stride", C.c_int64), ("k_out_stride", C.c_int64), ("q_norm", C.c_void_p),
                ("k_norm", C.c_void_p), ("freqs", C.c_void_p), ("positions", C.c_void_p), ("seq_lens", C.c_void_p), ("slots", C.c_void_p),
                ("n_rows", C.c_void_p), ("status", C.c_void_p)]


class DartLogprobsIn(C.Structure):
    _fields_ = [("batch", C.c_int32), ("rows", C.c_int32), ("vocab", C.c_int32), ("dtype", C.c_int32), ("n_tokens", C.c_int32),
                ("topk", C.c_int32), ("temperature", C.c_float), ("logits", C.c_void_p), ("row_stride", C.c_int64), ("tokens", C.c_void_p),
                ("token_row", C.c_void_p), ("n_rows", C.c_void_p), ("token_logprob", C.c_void_p), ("lse", C.c_void_p),
                ("entropy", C.c_void_p), ("top_ids", C.c_void_p), ("top_logprobs", C.c_void_p), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_size_t), ("status", C.c_void_p)]


_lib = None


def lib() -> C.CDLL:
    """Load libdart.so (once).  Raises if it has not been built: there is no CPU fallback."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2601_19278_b200.build` "
                               "(the drafting step has no CPU fallback)")
        L = C.CDLL(LIB_PATH)
        L.dart_draft_init.argtypes = [C.POINTER(DartConfig), C.POINTER(DartWeights), C.POINTER(DartNgramHost),
                                      C.POINTER(C.c_void_p)]
        L.dart_draft_init.restype = C.c_int
        L.dart_draft_step.argtypes = [C.c_void_p, C.POINTER(DartStepIn), C.POINTER(DartStepOut), C.c_void_p]
        L.dart_draft_step.restype = C.c_int
        L.dart_build_tree.argtypes = [C.c_void_p, C.POINTER(DartTreeIn), C.POINTER(DartTreeOut), C.c_void_p]
        L.dart_build_tree.restype = C.c_int
        L.dart_draft_step_host.argtypes = [C.c_void_p, C.POINTER(DartHostIo), C.POINTER(DartStepIn), C.POINTER(DartStepOut),
                                           C.POINTER(DartTreeIn), C.POINTER(DartTreeOut), C.c_void_p]
        L.dart_draft_step_host.restype = C.c_int
        L.dart_draft_destroy.argtypes = [C.c_void_p]
        L.dart_draft_destroy.restype = C.c_int
        L.dart_last_device_status.argtypes = [C.c_void_p, C.c_void_p]
        L.dart_last_device_status.restype = C.c_int
        L.dart_last_cuda_error.argtypes = [C.c_void_p]
        L.dart_last_cuda_error.restype = C.c_int
        L.dart_status_string.argtypes = [C.c_int]
        L.dart_status_string.restype = C.c_char_p
        L.dart_workspace_bytes.argtypes = [C.POINTER(DartConfig)]
        L.dart_workspace_bytes.restype = C.c_size_t
        L.dart_train_attention_fwd.argtypes = [C.POINTER(DartTrainAttnIn), C.c_void_p]
        L.dart_train_attention_fwd.restype = C.c_int
        L.dart_ngram_bytes.argtypes = [C.c_void_p]
        L.dart_ngram_bytes.restype = C.c_size_t
        L.dart_tree_verify_inputs.argtypes = [C.c_void_p, C.POINTER(DartVerifyIn), C.POINTER(DartVerifyOut), C.c_void_p]
        L.dart_tree_verify_inputs.restype = C.c_int
        L.dart_draft_prefill.argtypes = [C.c_void_p, C.POINTER(DartPrefillIn), C.c_void_p]
        L.dart_draft_prefill.restype = C.c_int
        L.dart_step_launch_count.argtypes = [C.c_void_p, C.c_int, C.c_int]
        L.dart_step_launch_count.restype = C.c_int
        L.dart_set_profile_events.argtypes = [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p]
        L.dart_set_profile_events.restype = C.c_int
        L.dart_topk_rows_noalloc.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_float, C.c_void_p,
                                             C.c_void_p, C.c_void_p]
        L.dart_topk_rows_noalloc.restype = C.c_int
        L.dart_selftest_bounded_wait.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p]
        L.dart_selftest_bounded_wait.restype = C.c_int
        P = C.c_void_p
        L.dart_kv8_attention.argtypes = [P, P, P]
        L.dart_kv8_attention_workspace_bytes.argtypes = [P, C.c_int32, C.c_int32, C.c_int32, C.c_int32]
        L.dart_kv8_attention_plan.argtypes = [P, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, P]
        L.dart_kv8_attention_plan.restype = C.c_int
        i32 = C.c_int32
        L.dart_kv8_attention_window.argtypes = [P, P, P, P]
        L.dart_kv8_attention_window_workspace_bytes.argtypes = [P, i32, i32, i32, i32, i32, i32]
        L.dart_kv8_attention_window_workspace_bytes.restype = C.c_size_t
        L.dart_kv8_attention_window_plan.argtypes = [P, i32, i32, i32, i32, i32, i32, i32, P]
        L.dart_kv8_trim.argtypes = [P, P, i32, i32, i32, P, P]
        L.dart_rope_frequencies.argtypes = [P, i32, P]
        L.dart_qk_norm_rope.argtypes = [P, P]
        L.dart_token_logprobs.argtypes = [P, P]
        L.dart_token_logprobs_workspace_bytes.argtypes = [i32, i32, i32, i32, i32]
        L.dart_token_logprobs_workspace_bytes.restype = C.c_size_t
        for n in ("kv8_attention_window", "kv8_attention_window_plan", "kv8_trim", "rope_frequencies", "qk_norm_rope", "token_logprobs"):
            getattr(L, "dart_" + n).restype = C.c_int
        L.dart_kv8_append.argtypes = [P, P, P]
        L.dart_kv8_append_owned.argtypes = [P, P, P, P]
        L.dart_kv8_fork.argtypes = [P, P, P, C.c_int32, P, P]
        L.dart_kv8_release.argtypes = [P, P, C.c_int32, P, P]
        L.dart_kv8_reserve.argtypes = [P, P, P, P, C.c_int32, P, C.c_size_t, P, P]
        L.dart_kv8_compact.argtypes = [P, P, P, P, C.c_size_t, P, P]
        L.dart_kv8_pages_workspace_bytes.argtypes = [P]
        L.dart_selftest_kv8_wait.argtypes = [P, P, C.c_int32, C.c_int32, P]
        L.dart_selftest_kv8_wait.restype = C.c_int
        L.dart_selftest_kv8_window_wait.argtypes = [P, P, P, C.c_int32, C.c_int32, P]
        L.dart_selftest_kv8_window_wait.restype = C.c_int
        for name in ("attention", "append", "append_owned", "fork", "release", "reserve", "compact"):
            getattr(L, "dart_kv8_" + name).restype = C.c_int
        L.dart_kv8_attention_workspace_bytes.restype = L.dart_kv8_pages_workspace_bytes.restype = C.c_size_t
        _lib = L
    return _lib


class DartError(RuntimeError):
    def __init__(self, status: int, where: str, cuda_error: int = 0):
        self.status = status
        name = lib().dart_status_string(status).decode()
        extra = f" (cudaError {cuda_error})" if cuda_error else ""
        super().__init__(f"{where}: {name}{extra}")


def make_config(w, **over) -> DartConfig:
    """dart_config from a synthetic.Workload (Appendix D defaults for the pruning constants)."""
    cfg = DartConfig()
    cfg.struct_size = C.sizeof(DartConfig)
    vals = dict(hidden=w.hidden, n_q_heads=w.n_q_heads, n_kv_heads=w.n_kv_heads, head_dim=w.head_dim,
                mlp_inter=w.mlp_inter, vocab=w.vocab, feat_in=w.feat_in, max_batch=w.batch,
                max_prefix=w.max_prefix, K=w.K, topk=w.topk, beam=w.beam, tree_budget=w.tree_budget,
                ngram_order=3, rope_theta=1e6, rms_eps=1e-6, w_ng=0.5, logit_decay=0.9, level_exp=0.7,
                eps_logit=1e-10, eps_ng=1e-10, temperature=w.temperature, philox_seed=1234,
                ngram_layout=NGRAM_HASH)
    vals.update(over)
    for k, v in vals.items():
        setattr(cfg, k, v)
    return cfg


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


class DartDraft:
    """Owner of a dart_handle.  Methods mirror the C entry points one to one."""

    def __init__(self, cfg: DartConfig, weights: Dict[str, torch.Tensor], ngram: Optional[Dict[str, np.ndarray]] = None):
        self._h = C.c_void_p()
        self.cfg = cfg
        names = [n for n in WEIGHT_NAMES if not (n == "w_fc" and cfg.feat_in == 0)]   # no fusion matrix without a feature FC
        self._weights = {n: weights[n] for n in names}             # keep the device tensors alive
        for n, t in self._weights.items():
            assert t.is_cuda and t.dtype == torch.bfloat16 and t.is_contiguous(), n
        ws = DartWeights(**{n: t.data_ptr() for n, t in self._weights.items()})
        ng = None
        if ngram is not None and len(ngram["next"]):
            self._ng = {k: np.ascontiguousarray(v) for k, v in ngram.items()}
            assert self._ng["order"].dtype == np.uint8 and self._ng["score"].dtype == np.float32
            ng = DartNgramHost(len(self._ng["next"]), self._ng["order"].ctypes.data, self._ng["ctx0"].ctypes.data,
                               self._ng["ctx1"].ctypes.data, self._ng["next"].ctypes.data, self._ng["score"].ctypes.data)
        rc = lib().dart_draft_init(C.byref(cfg), C.byref(ws), C.byref(ng) if ng is not None else None, C.byref(self._h))
        if rc != DART_OK:
            raise DartError(rc, "dart_draft_init", lib().dart_last_cuda_error(None))

    def close(self):
        if self._h:
            lib().dart_draft_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @staticmethod
    def _stream(stream) -> int:
        return (stream if stream is not None else torch.cuda.current_stream()).cuda_stream

    def draft_step(self, *, feats, tokens, seq_lens, seq_lens_host: np.ndarray, k_cache, v_cache, n_fresh,
                   topk_ids, topk_slogit, logits=None, step_counter: int = 0, stream=None) -> None:
        """dart_draft_step: all tensors are caller-owned device tensors; seq_lens_host is a host int32 array.
        n_fresh: one count for all sequences, or a sequence of per-sequence counts (fresh_counts_host)."""
        slh = np.ascontiguousarray(seq_lens_host, dtype=np.int32)
        counts = None if isinstance(n_fresh, (int, np.integer)) else np.ascontiguousarray(n_fresh, dtype=np.int32)
        sin = DartStepIn(len(slh), int(n_fresh) if counts is None else int(counts.max(initial=0)), _ptr(feats), _ptr(tokens),
                         _ptr(seq_lens), slh.ctypes.data, _ptr(k_cache), _ptr(v_cache), step_counter,
                         None if counts is None else counts.ctypes.data)
        sout = DartStepOut(_ptr(topk_ids), _ptr(topk_slogit), _ptr(logits))
        rc = lib().dart_draft_step(self._h, C.byref(sin), C.byref(sout), self._stream(stream))
        if rc != DART_OK:
            raise DartError(rc, "dart_draft_step", lib().dart_last_cuda_error(self._h))

    def host_step(self, *, in_host, in_dev, out_host, out_dev, feats, tokens, seq_lens, seq_lens_host, k_cache, v_cache,
                  n_fresh, topk_ids, topk_slogit, ctx_tail, tree_tokens, parents, depth, mask, n_nodes, scores=None,
                  logits=None, first_row=0, n_levels: Optional[int] = None, stream=None) -> "HostStep":
        """dart_draft_step_host with its argument structures built once: the returned object is called with the
        step counter and runs copy in, forward pass, tree, copy out, wait.  in_host / out_host are (pinned) host byte
        tensors, in_dev / out_dev the device buffers that the device tensors passed here are views of."""
        return HostStep(self, dict(in_host=in_host, in_dev=in_dev, out_host=out_host, out_dev=out_dev, feats=feats,
                                   tokens=tokens, seq_lens=seq_lens, seq_lens_host=seq_lens_host, k_cache=k_cache,
                                   v_cache=v_cache, n_fresh=n_fresh, topk_ids=topk_ids, topk_slogit=topk_slogit,
                                   ctx_tail=ctx_tail, tree_tokens=tree_tokens, parents=parents, depth=depth, mask=mask,
                                   n_nodes=n_nodes, scores=scores, logits=logits, first_row=first_row,
                                   n_levels=n_levels), stream)

    def prefill(self, *, feats, tokens, seq_lens_host, new_rows_host, k_cache, v_cache, stream=None) -> None:
        """dart_draft_prefill: append the k, v of new prefix rows (packed features / next-token ids) to the caches."""
        slh = np.ascontiguousarray(seq_lens_host, dtype=np.int32)
        nrh = np.ascontiguousarray(new_rows_host, dtype=np.int32)
        pin = DartPrefillIn(len(slh), _ptr(feats), _ptr(tokens), slh.ctypes.data, nrh.ctypes.data, _ptr(k_cache), _ptr(v_cache))
        rc = lib().dart_draft_prefill(self._h, C.byref(pin), self._stream(stream))
        if rc != DART_OK:
            raise DartError(rc, "dart_draft_prefill", lib().dart_last_cuda_error(self._h))

    def verify_inputs(self, *, batch: int, max_levels: int, parents, depth, n_nodes, root_pos, position_ids, retrieve, n_leaves,
                      stream=None) -> None:
        """dart_tree_verify_inputs: position ids and root-to-leaf paths of the trees dart_build_tree wrote."""
        vin = DartVerifyIn(batch, max_levels, _ptr(parents), _ptr(depth), _ptr(n_nodes), _ptr(root_pos))
        vout = DartVerifyOut(_ptr(position_ids), _ptr(retrieve), _ptr(n_leaves))
        rc = lib().dart_tree_verify_inputs(self._h, C.byref(vin), C.byref(vout), self._stream(stream))
        if rc != DART_OK:
            raise DartError(rc, "dart_tree_verify_inputs", lib().dart_last_cuda_error(self._h))

    def build_tree(self, *, batch: int, topk_ids, topk_slogit, ctx_tail, tokens, parents, depth, mask, n_nodes,
                   scores=None, first_row=0, n_levels: Optional[int] = None, stream=None) -> None:
        """dart_build_tree on caller-owned device tensors.  first_row: one row for all sequences, or a sequence
        of per-sequence first rows (first_rows_host)."""
        rows = None if isinstance(first_row, (int, np.integer)) else np.ascontiguousarray(first_row, dtype=np.int32)
        fr = int(first_row) if rows is None else int(rows.min())
        tin = DartTreeIn(batch, fr, self.cfg.K - fr if n_levels is None else n_levels,
                         _ptr(topk_ids), _ptr(topk_slogit), _ptr(ctx_tail), None if rows is None else rows.ctypes.data)
        tout = DartTreeOut(_ptr(tokens), _ptr(parents), _ptr(depth), _ptr(mask), _ptr(n_nodes), _ptr(scores))
        rc = lib().dart_build_tree(self._h, C.byref(tin), C.byref(tout), self._stream(stream))
        if rc != DART_OK:
            raise DartError(rc, "dart_build_tree", lib().dart_last_cuda_error(self._h))

    def device_status(self, stream=None) -> int:
        return lib().dart_last_device_status(self._h, self._stream(stream))

    def selftest_bounded_wait(self, spin_limit: int, leave_ticket: bool = False, stream=None) -> None:
        """dart_selftest_bounded_wait: enqueue a wait that runs out on purpose (device_status() then reports the time-out)."""
        rc = lib().dart_selftest_bounded_wait(self._h, spin_limit, 1 if leave_ticket else 0, self._stream(stream))
        if rc != DART_OK:
            raise DartError(rc, "dart_selftest_bounded_wait", lib().dart_last_cuda_error(self._h))

    def set_profile_events(self, stage: int, start: torch.cuda.Event, stop: torch.cuda.Event) -> None:
        """dart_set_profile_events: bracket one stage of the next call with two torch CUDA events."""
        rc = lib().dart_set_profile_events(self._h, stage, start.cuda_event, stop.cuda_event)
        if rc != DART_OK:
            raise DartError(rc, "dart_set_profile_events")

    def launch_count(self, batch: int, n_fresh: int) -> int:
        return lib().dart_step_launch_count(self._h, batch, n_fresh)

    def ngram_bytes(self) -> int:
        return lib().dart_ngram_bytes(self._h)


def topk_rows_noalloc(logits: torch.Tensor, topk: int, eps_logit: float, out_ids: torch.Tensor, out_slogit: torch.Tensor,
                      stream=None) -> None:
    """dart_topk_rows_noalloc: log-softmax + top-k of fp32 logits [rows, vocab] into caller-owned outputs.
    For callers that may not allocate device memory: the library uses a fixed scratch array of its own
    (at most 128 rows; calls on one GPU must not overlap)."""
    assert logits.is_cuda and logits.dtype == torch.float32 and logits.is_contiguous() and logits.dim() == 2
    rows, vocab = logits.shape
    st = (stream if stream is not None else torch.cuda.current_stream()).cuda_stream
    rc = lib().dart_topk_rows_noalloc(logits.data_ptr(), rows, vocab, topk, eps_logit, out_ids.data_ptr(),
                                      out_slogit.data_ptr(), st)
    if rc != DART_OK:
        raise DartError(rc, "dart_topk_rows_noalloc")


def train_attention_fwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, seq_lens, prompt_len: int, draft_len: int,
                        out: torch.Tensor, status: Optional[torch.Tensor] = None, stream=None) -> None:
    """dart_train_attention_fwd on caller-owned device tensors: q [B, Hq, L, dh], k, v [B, Hkv, L, dh] bf16,
    L = prompt_len * (1 + draft_len); seq_lens: host ints [B]."""
    lens = np.ascontiguousarray(seq_lens, dtype=np.int32)
    a = DartTrainAttnIn(batch=q.shape[0], n_q_heads=q.shape[1], n_kv_heads=k.shape[1], head_dim=q.shape[3], prompt_len=prompt_len,
                        draft_len=draft_len, q=q.data_ptr(), k=k.data_ptr(), v=v.data_ptr(), seq_lens_host=lens.ctypes.data,
                        out=out.data_ptr(), status=_ptr(status))
    st = stream if stream is not None else torch.cuda.current_stream(q.device)
    rc = lib().dart_train_attention_fwd(C.byref(a), C.c_void_p(st.cuda_stream))
    if rc != DART_OK:
        raise DartError(rc, "dart_train_attention_fwd", lib().dart_last_cuda_error(None))


# ---- the target's KV cache in 8 bits, in pages ------------------------------------------------------------------------
# A call's device time starts at a few microseconds, so the marshalling is kept as short: integer device comparisons, the
# argument structure packed by one struct.pack (its layout is the C structure's: native alignment), no objects per call.
_KV8_ATTN = struct.Struct("@7i3P2q7PNP")
_KV8_APPEND = struct.Struct("@7i2P2q6P")
_KV8_WINDOW = struct.Struct("@2iP")
_QK_ROPE = struct.Struct("@9if4P4q8P")
_LOGPROBS = struct.Struct("@6ifPq9PNP")
_KV8_FN: Dict[str, object] = {}
_BF16, _I32, _U8, _F32 = torch.bfloat16, torch.int32, torch.uint8, torch.float32


def _kv8_fn(name: str):
    fn = _KV8_FN.get(name)
    if fn is None:
        fn = _KV8_FN[name] = getattr(lib(), name)
    return fn


def _kv8_check(t: Optional[torch.Tensor], name: str, dtype, dev: int, shape=None) -> int:
    """Address of a contiguous tensor of this type, device index and shape (0 for None); ValueError otherwise."""
    if t is None:
        return 0
    if t.dtype is dtype and t.get_device() == dev and t.is_contiguous() and (shape is None or t.shape == shape):
        return t.data_ptr()
    if t.dtype != dtype or t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous {dtype} tensor on cuda:{dev} is needed, got {t.dtype} on {t.device}"
                         f"{'' if t.is_contiguous() else ', not contiguous'}")
    raise ValueError(f"{name}: shape {tuple(shape)} is needed, got {tuple(t.shape)}")


def _kv8_rows(t: torch.Tensor, name: str, heads: int, dim: int, dev: int, dtype=_BF16) -> int:
    """Row stride of [batch, rows, heads, dim] of this type whose heads are packed and whose batch entries are `rows` rows apart."""
    shape = t.shape
    if t.dtype is dtype and t.get_device() == dev and shape[2:] == (heads, dim) and len(shape) == 4 and t.is_contiguous():
        return heads * dim
    if t.dtype != dtype or t.get_device() != dev or len(shape) != 4 or shape[2] != heads or shape[3] != dim:
        kind = "bf16" if dtype == _BF16 else str(dtype)
        raise ValueError(f"{name}: {kind} [batch, rows, {heads}, {dim}] on cuda:{dev} is needed, got {t.dtype} {tuple(shape)} on {t.device}")
    B, R = shape[0], shape[1]
    s0, s1, s2, s3 = t.stride()
    row = s1 if R > 1 else s0 if B > 1 else heads * dim
    if s3 != 1 or (heads > 1 and s2 != dim) or (B > 1 and R > 1 and s0 != R * s1):
        raise ValueError(f"{name}: heads must be packed and batch entries {R} rows apart, got strides {t.stride()}")
    return row


def _kv8_call(name: str, dev: int, stream, *args) -> None:
    """One call with device `dev` current and the stream's handle as its last argument."""
    if dev != torch._C._cuda_getDevice():
        with torch.cuda.device(dev):
            return _kv8_call(name, dev, stream, *args)
    rc = _kv8_fn(name)(*args, torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream)
    if rc != DART_OK:
        raise DartError(rc, name, lib().dart_last_cuda_error(None) if rc == DART_ERR_CUDA else 0)


class Kv8Cache:
    """dart_kv8_cache over caller-owned tensors: k_pages, v_pages float8_e4m3fn or int8 [n_layers, n_pages, n_kv_heads,
    page_tokens, head_dim], k_scale, v_scale fp32 [n_layers, n_pages, n_kv_heads]."""

    def __init__(self, k_pages: torch.Tensor, v_pages: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor):
        if k_pages.dtype not in (torch.float8_e4m3fn, torch.int8) or k_pages.dim() != 5:
            raise ValueError("k_pages: float8_e4m3fn or int8 [n_layers, n_pages, n_kv_heads, page_tokens, head_dim] is needed, got "
                             f"{k_pages.dtype} {tuple(k_pages.shape)}")
        if not k_pages.is_cuda:
            raise ValueError("k_pages must be on a CUDA device (there is no CPU fallback)")
        self.device = k_pages.device
        self.index = k_pages.get_device()
        shape = k_pages.shape
        self.n_layers, self.n_pages, self.n_kv_heads, self.page_tokens, self.head_dim = shape
        self.k_pages, self.v_pages, self.k_scale, self.v_scale = k_pages, v_pages, k_scale, v_scale    # keep the tensors alive
        self.c = DartKv8Cache(KV8_E4M3 if k_pages.dtype == torch.float8_e4m3fn else KV8_INT8, *shape,
                              _kv8_check(k_pages, "k_pages", k_pages.dtype, self.index),
                              _kv8_check(v_pages, "v_pages", k_pages.dtype, self.index, shape),
                              _kv8_check(k_scale, "k_scale", torch.float32, self.index, shape[:3]),
                              _kv8_check(v_scale, "v_scale", torch.float32, self.index, shape[:3]))
        self.ref = C.addressof(self.c)


class Kv8Pages:
    """dart_kv8_pages over caller-owned int32 tensors: page_table [max_seqs, max_pages], seq_lens [max_seqs], ref_count
    [n_pages].  A new pool starts with table -1, lengths 0, counts 0."""

    def __init__(self, page_table: torch.Tensor, seq_lens: torch.Tensor, ref_count: torch.Tensor, page_tokens: int):
        if not page_table.is_cuda:
            raise ValueError("page_table must be on a CUDA device (there is no CPU fallback)")
        self.device = page_table.device
        self.index = page_table.get_device()
        self.page_table, self.seq_lens, self.ref_count = page_table, seq_lens, ref_count
        if page_table.dim() != 2 or ref_count.dim() != 1:
            raise ValueError("page_table [max_seqs, max_pages] and ref_count [n_pages] are needed")
        S, M = page_table.shape
        self.c = DartKv8Pages(ref_count.shape[0], page_tokens, S, M, _kv8_check(page_table, "page_table", _I32, self.index),
                              _kv8_check(seq_lens, "seq_lens", _I32, self.index, (S,)),
                              _kv8_check(ref_count, "ref_count", _I32, self.index))
        self.ref = C.addressof(self.c)


def kv8_attention_workspace_bytes(cache: Kv8Cache, batch: int, rows: int, n_q_heads: int, max_len: int) -> int:
    return lib().dart_kv8_attention_workspace_bytes(cache.ref, batch, rows, n_q_heads, max_len)


def kv8_attention_plan(cache: Kv8Cache, batch: int, rows: int, n_q_heads: int, max_len: int, new_rows: bool = True) -> Dict[str, int]:
    """dart_kv8_attention_plan: which kernel a call of this shape runs on and how its key axis is split (by max_len: a bound near the
    longest length is a faster call)."""
    p = DartKv8Plan()
    rc = lib().dart_kv8_attention_plan(cache.ref, batch, rows, n_q_heads, max_len, int(new_rows), C.byref(p))
    if rc != DART_OK:
        raise DartError(rc, "dart_kv8_attention_plan")
    return {f[0]: getattr(p, f[0]) for f in p._fields_}


def _kv8_attn_args(cache: Kv8Cache, layer, q, k_new, v_new, seq_lens, page_table, out, max_len, workspace, slots, n_rows, mask, status) -> bytes:
    dev = cache.index
    shape = q.shape
    if len(shape) != 4:
        raise ValueError(f"q: [batch, rows, n_q_heads, head_dim] is needed, got {tuple(shape)}")
    B, R, H, d = shape
    qs = _kv8_rows(q, "q", H, cache.head_dim, dev)
    kp = vp = ns = 0
    if k_new is not None:
        if v_new is None or k_new.shape[:2] != (B, R) or v_new.shape[:2] != (B, R):
            raise ValueError("k_new and v_new: both [batch, rows, n_kv_heads, head_dim] with q's batch and rows, or neither")
        ns = _kv8_rows(k_new, "k_new", cache.n_kv_heads, d, dev)
        if _kv8_rows(v_new, "v_new", cache.n_kv_heads, d, dev) != ns:
            raise ValueError("k_new and v_new must have the same row stride")
        kp, vp = k_new.data_ptr(), v_new.data_ptr()
    elif v_new is not None:
        raise ValueError("v_new without k_new")
    table_shape = page_table.shape
    if len(table_shape) != 2:
        raise ValueError("page_table: [max_seqs, max_pages] is needed")
    S, M = table_shape
    return _KV8_ATTN.pack(layer, B, R, H, S, M, max_len, q.data_ptr(), kp, vp, qs, ns, 0 if slots is None else _kv8_check(slots, "slots", _I32, dev, (B,)),
                          _kv8_check(seq_lens, "seq_lens", _I32, dev, (S,)), _kv8_check(page_table, "page_table", _I32, dev),
                          0 if n_rows is None else _kv8_check(n_rows, "n_rows", _I32, dev, (B,)),
                          0 if mask is None else _kv8_check(mask, "mask", _U8, dev, (B, R, R)), _kv8_check(out, "out", _BF16, dev, shape),
                          _kv8_check(workspace, "workspace", _U8, dev), workspace.numel(), 0 if status is None else _kv8_check(status, "status", _I32, dev))


def kv8_attention(cache: Kv8Cache, layer: int, q: torch.Tensor, k_new: Optional[torch.Tensor], v_new: Optional[torch.Tensor],
                  seq_lens: torch.Tensor, page_table: torch.Tensor, out: torch.Tensor, *, max_len: int, workspace: torch.Tensor,
                  slots: Optional[torch.Tensor] = None, n_rows: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
                  status: Optional[torch.Tensor] = None, stream=None) -> None:
    """dart_kv8_attention: q, out [batch, rows, n_q_heads, head_dim], k_new, v_new [batch, rows, n_kv_heads, head_dim] bf16 (q and the
    new rows may be slices of one QKV matrix); seq_lens, page_table, slots, n_rows int32 on the device; mask u8
    [batch, rows, rows] (dart_tree_out.mask) or None: causal.  max_len: host bound of the lengths."""
    a = _kv8_attn_args(cache, layer, q, k_new, v_new, seq_lens, page_table, out, max_len, workspace, slots, n_rows, mask, status)
    _kv8_call("dart_kv8_attention", cache.index, stream, cache.ref, a)


def kv8_attention_window_workspace_bytes(cache: Kv8Cache, batch: int, rows: int, n_q_heads: int, max_len: int, window: int, sinks: int = 0) -> int:
    return lib().dart_kv8_attention_window_workspace_bytes(cache.ref, batch, rows, n_q_heads, max_len, window, sinks)


def kv8_attention_window_plan(cache: Kv8Cache, batch: int, rows: int, n_q_heads: int, max_len: int, window: int, sinks: int = 0,
                              new_rows: bool = True) -> Dict[str, int]:
    """dart_kv8_attention_window_plan: as kv8_attention_plan, with a window."""
    p = DartKv8Plan()
    rc = lib().dart_kv8_attention_window_plan(cache.ref, batch, rows, n_q_heads, max_len, window, sinks, int(new_rows), C.byref(p))
    if rc != DART_OK:
        raise DartError(rc, "dart_kv8_attention_window_plan")
    return {f[0]: getattr(p, f[0]) for f in p._fields_}


def kv8_attention_window(cache: Kv8Cache, layer: int, q: torch.Tensor, k_new: Optional[torch.Tensor], v_new: Optional[torch.Tensor],
                         seq_lens: torch.Tensor, page_table: torch.Tensor, out: torch.Tensor, *, max_len: int, window: int, sinks: int = 0,
                         positions: Optional[torch.Tensor] = None, workspace: torch.Tensor, slots: Optional[torch.Tensor] = None,
                         n_rows: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                         stream=None) -> None:
    """dart_kv8_attention_window: kv8_attention in which the row at position p sees positions t < sinks and t > p - window alone.
    positions int32 [batch, rows] (dart_tree_verify_inputs' position_ids) with a mask; without one row r sits at seq_len + r."""
    a = _kv8_attn_args(cache, layer, q, k_new, v_new, seq_lens, page_table, out, max_len, workspace, slots, n_rows, mask, status)
    w = _KV8_WINDOW.pack(window, sinks, 0 if positions is None else _kv8_check(positions, "positions", _I32, cache.index, q.shape[:2]))
    _kv8_call("dart_kv8_attention_window", cache.index, stream, cache.ref, a, w)


def kv8_append(cache: Kv8Cache, first_layer: int, k_new: torch.Tensor, v_new: torch.Tensor, seq_lens: torch.Tensor,
               page_table: torch.Tensor, *, n_append: Optional[torch.Tensor] = None, row_index: Optional[torch.Tensor] = None,
               max_append: Optional[int] = None, slots: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
               pages: Optional[Kv8Pages] = None, stream=None) -> None:
    """dart_kv8_append: k_new, v_new bf16 [n_layers, batch, rows, n_kv_heads, head_dim]; row_index int32 [batch, max_append] (an
    accepted path of dart_tree_verify_inputs) or None: the rows in order.  The caller advances seq_lens.  With `pages` (whose
    page_table is then meant) dart_kv8_append_owned: pages that other sequences share are left alone and reported."""
    dev = cache.index
    if k_new.dim() != 5 or v_new.shape != k_new.shape:
        raise ValueError("k_new and v_new: [n_layers, batch, rows, n_kv_heads, head_dim] are needed, of one shape")
    L, B, R, hkv, d = k_new.shape
    if L < 1:
        raise ValueError("k_new: at least one layer is needed")
    ls, s0, rs, s2, s3 = k_new.stride()
    if hkv != cache.n_kv_heads or d != cache.head_dim or k_new.dtype != _BF16 or v_new.dtype != _BF16 or k_new.get_device() != dev or \
            v_new.get_device() != dev:
        raise ValueError(f"k_new and v_new: bf16 with {cache.n_kv_heads} heads of {cache.head_dim} on cuda:{dev} are needed")
    if R == 1:
        rs = s0 if B > 1 else hkv * d
    if L == 1:
        ls = 0
    if s3 != 1 or (hkv > 1 and s2 != d) or (B > 1 and s0 != R * rs):
        raise ValueError(f"k_new: heads must be packed and batch entries {R} rows apart, got strides {k_new.stride()}")
    if v_new.stride() != k_new.stride():
        raise ValueError("k_new and v_new must have the same strides")
    if page_table.dim() != 2:
        raise ValueError("page_table: [max_seqs, max_pages] is needed")
    A = max_append if max_append is not None else row_index.shape[1] if row_index is not None else R
    S, M = page_table.shape
    a = _KV8_APPEND.pack(first_layer, L, B, R, A, S, M, k_new.data_ptr(), v_new.data_ptr(), rs, ls, _kv8_check(slots, "slots", _I32, dev, (B,)),
                         _kv8_check(seq_lens, "seq_lens", _I32, dev, (S,)), _kv8_check(page_table, "page_table", _I32, dev),
                         _kv8_check(n_append, "n_append", _I32, dev, (B,)), _kv8_check(row_index, "row_index", _I32, dev, (B, A)),
                         _kv8_check(status, "status", _I32, dev))
    if pages is None:
        return _kv8_call("dart_kv8_append", dev, stream, cache.ref, a)
    _kv8_same_pool(pages, cache)
    _kv8_call("dart_kv8_append_owned", dev, stream, cache.ref, pages.ref, a)


def kv8_pages_workspace_bytes(pages: Kv8Pages) -> int:
    return lib().dart_kv8_pages_workspace_bytes(pages.ref)


def kv8_fork(pages: Kv8Pages, src: torch.Tensor, dst: torch.Tensor, *, status: Optional[torch.Tensor] = None, stream=None) -> None:
    """dart_kv8_fork: slot dst[i] becomes a copy of slot src[i] (shared pages)."""
    dev, n = pages.index, src.numel()
    _kv8_call("dart_kv8_fork", dev, stream, pages.ref, _kv8_check(src, "src", _I32, dev, (n,)), _kv8_check(dst, "dst", _I32, dev, (n,)), n,
              _kv8_check(status, "status", _I32, dev))


def kv8_release(pages: Kv8Pages, seqs: torch.Tensor, *, status: Optional[torch.Tensor] = None, stream=None) -> None:
    """dart_kv8_release: the slots give back all their pages."""
    dev, n = pages.index, seqs.numel()
    _kv8_call("dart_kv8_release", dev, stream, pages.ref, _kv8_check(seqs, "seqs", _I32, dev, (n,)), n, _kv8_check(status, "status", _I32, dev))


def kv8_trim(pages: Kv8Pages, seqs: torch.Tensor, *, window: int, sinks: int = 0, status: Optional[torch.Tensor] = None, stream=None) -> None:
    """dart_kv8_trim: the slots give back the pages that lie behind the window of every row to come and hold no sink (their table
    entries become KV8_GIVEN_BACK)."""
    dev, n = pages.index, seqs.numel()
    _kv8_call("dart_kv8_trim", dev, stream, pages.ref, _kv8_check(seqs, "seqs", _I32, dev, (n,)), n, window, sinks,
              _kv8_check(status, "status", _I32, dev))


def _kv8_same_pool(pages: Kv8Pages, cache: Kv8Cache) -> None:
    if cache.index != pages.index:
        raise ValueError("the cache and its bookkeeping must be on one device")


def kv8_reserve(pages: Kv8Pages, cache: Kv8Cache, seqs: torch.Tensor, n_new: torch.Tensor, *, workspace: torch.Tensor,
                status: Optional[torch.Tensor] = None, stream=None) -> None:
    """dart_kv8_reserve: pages for the next n_new[i] positions of slot seqs[i]; shared ones are replaced by copies."""
    _kv8_same_pool(pages, cache)
    dev, n = pages.index, seqs.numel()
    _kv8_call("dart_kv8_reserve", dev, stream, pages.ref, cache.ref, _kv8_check(seqs, "seqs", _I32, dev, (n,)),
              _kv8_check(n_new, "n_new", _I32, dev, (n,)), n, _kv8_check(workspace, "workspace", _U8, dev), workspace.numel(),
              _kv8_check(status, "status", _I32, dev))


def kv8_compact(pages: Kv8Pages, cache: Kv8Cache, *, workspace: torch.Tensor, n_live: Optional[torch.Tensor] = None,
                status: Optional[torch.Tensor] = None, stream=None) -> None:
    """dart_kv8_compact: the pages in use move to the front of the pool."""
    _kv8_same_pool(pages, cache)
    dev = pages.index
    _kv8_call("dart_kv8_compact", dev, stream, pages.ref, cache.ref, _kv8_check(n_live, "n_live", _I32, dev),
              _kv8_check(workspace, "workspace", _U8, dev), workspace.numel(), _kv8_check(status, "status", _I32, dev))


# ---- around the target's attention: rotation, log probabilities ---------------------------------------------------------
_DTYPES = {torch.bfloat16: DART_BF16, torch.float16: DART_FP16, torch.float32: DART_FP32}


def rope_frequencies(rope_theta: float, rotary_dim: int, device, inv_freq=None) -> torch.Tensor:
    """dart_rope_frequencies, on the device: int64 [rotary_dim / 2] for qk_norm_rope.  inv_freq: radians per position of the pairs
    (a scaled form of rope_theta^(-2i / rotary_dim), which is the default)."""
    f = np.ascontiguousarray(rope_theta ** (-np.arange(0, rotary_dim, 2, dtype=np.float64) / rotary_dim) if inv_freq is None else inv_freq, dtype=np.float64)
    if f.ndim != 1 or 2 * f.size != rotary_dim:
        raise ValueError(f"inv_freq: {rotary_dim // 2} frequencies are needed, got shape {f.shape}")
    out = np.zeros(f.size, dtype=np.int64)
    rc = lib().dart_rope_frequencies(f.ctypes.data, f.size, out.ctypes.data)
    if rc != DART_OK:
        raise DartError(rc, "dart_rope_frequencies")
    return torch.from_numpy(out).to(device)


def qk_norm_rope(q: torch.Tensor, k: Optional[torch.Tensor], q_out: torch.Tensor, k_out: Optional[torch.Tensor], freqs: torch.Tensor, *,
                 positions: Optional[torch.Tensor] = None, seq_lens: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None,
                 n_rows: Optional[torch.Tensor] = None, q_norm: Optional[torch.Tensor] = None, k_norm: Optional[torch.Tensor] = None,
                 eps: float = 1e-6, interleaved: bool = False, status: Optional[torch.Tensor] = None, stream=None) -> None:
    """dart_qk_norm_rope: q, q_out [batch, rows, n_q_heads, head_dim], k, k_out [batch, rows, n_k_heads, head_dim] (or None) bf16, fp16 or
    fp32, heads packed (q and k may be slices of one QKV matrix, the outputs may be the inputs); q_norm, k_norm [head_dim] or neither;
    freqs of rope_frequencies.  Positions: int32 [batch, rows], or seq_lens of the slots + row."""
    dev, dt, shape = q.get_device(), q.dtype, q.shape
    if len(shape) != 4 or dt not in _DTYPES or dev < 0:
        raise ValueError(f"q: bf16, fp16 or fp32 [batch, rows, n_q_heads, head_dim] on a CUDA device is needed, got {dt} {tuple(shape)} on {q.device}")
    B, R, H, d = shape
    hk = kp = kop = ks = kos = 0
    if k is not None and k_out is not None:
        k_shape = k.shape
        if len(k_shape) != 4 or k_shape[:2] != (B, R) or k_out.shape != k_shape:
            raise ValueError("k and k_out: [batch, rows, n_k_heads, head_dim] with q's batch and rows are needed, of one shape")
        hk = k_shape[2]
        ks, kos, kp, kop = _kv8_rows(k, "k", hk, d, dev, dt), _kv8_rows(k_out, "k_out", hk, d, dev, dt), k.data_ptr(), k_out.data_ptr()
    elif k is not None or k_out is not None:
        raise ValueError("k and k_out: both or neither")
    if q_out.shape != shape:
        raise ValueError("q_out must have q's shape")
    a = _QK_ROPE.pack(B, R, H, hk, d, 2 * freqs.numel(), interleaved, _DTYPES[dt], 0 if seq_lens is None else seq_lens.numel(), eps,
                      q.data_ptr(), kp, q_out.data_ptr(), kop, _kv8_rows(q, "q", H, d, dev, dt), ks, _kv8_rows(q_out, "q_out", H, d, dev, dt), kos,
                      0 if q_norm is None else _kv8_check(q_norm, "q_norm", dt, dev, (d,)), 0 if k_norm is None else _kv8_check(k_norm, "k_norm", dt, dev, (d,)),
                      _kv8_check(freqs, "freqs", torch.int64, dev), 0 if positions is None else _kv8_check(positions, "positions", _I32, dev, (B, R)),
                      0 if seq_lens is None else _kv8_check(seq_lens, "seq_lens", _I32, dev), 0 if slots is None else _kv8_check(slots, "slots", _I32, dev, (B,)),
                      0 if n_rows is None else _kv8_check(n_rows, "n_rows", _I32, dev, (B,)), 0 if status is None else _kv8_check(status, "status", _I32, dev))
    _kv8_call("dart_qk_norm_rope", dev, stream, a)


def token_logprobs_workspace_bytes(logits: torch.Tensor, topk: int = 0) -> int:
    """Bytes for token_logprobs of logits of this shape ([batch, rows, vocab]) and type."""
    B, R, V = logits.shape
    return lib().dart_token_logprobs_workspace_bytes(B, R, V, _DTYPES.get(logits.dtype, -1), topk)


def token_logprobs(logits: torch.Tensor, tokens: Optional[torch.Tensor], out: Optional[torch.Tensor], *, workspace: torch.Tensor,
                   temperature: float = 1.0, token_row: Optional[torch.Tensor] = None, n_rows: Optional[torch.Tensor] = None,
                   lse: Optional[torch.Tensor] = None, entropy: Optional[torch.Tensor] = None, top_ids: Optional[torch.Tensor] = None,
                   top_logprobs: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None, stream=None) -> None:
    """dart_token_logprobs: logits bf16, fp16 or fp32 [batch, rows, vocab] (rows packed, any row stride); tokens int32, out fp32
    [batch, n] (or neither), scored by row token_row[b][j] (a draft tree's parents), or token j by row j; lse, entropy fp32 [batch, rows];
    top_ids int32, top_logprobs fp32 [batch, rows, k]."""
    dev, shape = logits.get_device(), logits.shape
    if len(shape) != 3 or logits.dtype not in _DTYPES or dev < 0:
        raise ValueError(f"logits: bf16, fp16 or fp32 [batch, rows, vocab] on a CUDA device are needed, got {logits.dtype} {tuple(shape)} on {logits.device}")
    B, R, V = shape
    row = V
    if not logits.is_contiguous():
        s0, s1, s2 = logits.stride()
        row = s1 if R > 1 else s0 if B > 1 else V
        if (s2 != 1 and V > 1) or (B > 1 and R > 1 and s0 != R * s1):
            raise ValueError(f"logits: a row's logits must be packed and batch entries {R} rows apart, got strides {logits.stride()}")
    if (tokens is None) != (out is None) or (top_ids is None) != (top_logprobs is None) or (tokens is None and token_row is not None):
        raise ValueError("tokens and out, and top_ids and top_logprobs, go together; token_row needs tokens")
    n = k = tp = op = ip = lp = 0
    if tokens is not None:
        n = tokens.shape[1] if tokens.dim() == 2 else -1
        tp, op = _kv8_check(tokens, "tokens", _I32, dev, (B, n)), _kv8_check(out, "out", _F32, dev, (B, n))
    if top_ids is not None:
        k = top_ids.shape[2] if top_ids.dim() == 3 else -1
        ip, lp = _kv8_check(top_ids, "top_ids", _I32, dev, (B, R, k)), _kv8_check(top_logprobs, "top_logprobs", _F32, dev, (B, R, k))
    a = _LOGPROBS.pack(B, R, V, _DTYPES[logits.dtype], n, k, temperature, logits.data_ptr(), row, tp,
                       0 if token_row is None else _kv8_check(token_row, "token_row", _I32, dev, (B, n)),
                       0 if n_rows is None else _kv8_check(n_rows, "n_rows", _I32, dev, (B,)), op,
                       0 if lse is None else _kv8_check(lse, "lse", _F32, dev, (B, R)), 0 if entropy is None else _kv8_check(entropy, "entropy", _F32, dev, (B, R)),
                       ip, lp, _kv8_check(workspace, "workspace", _U8, dev), workspace.numel(), 0 if status is None else _kv8_check(status, "status", _I32, dev))
    _kv8_call("dart_token_logprobs", dev, stream, a)


def workspace_bytes(cfg: DartConfig) -> int:
    return lib().dart_workspace_bytes(C.byref(cfg))


class HostStep:
    """One prepared dart_draft_step_host call (argument marshalling only; see DartDraft.host_step)."""

    def __init__(self, draft: "DartDraft", a: dict, stream) -> None:
        self._draft, self._keep = draft, a
        self._slh = np.ascontiguousarray(a["seq_lens_host"], dtype=np.int32)
        nf = a["n_fresh"]
        self._counts = None if isinstance(nf, (int, np.integer)) else np.ascontiguousarray(nf, dtype=np.int32)
        fr = a["first_row"]
        self._rows = None if isinstance(fr, (int, np.integer)) else np.ascontiguousarray(fr, dtype=np.int32)
        B = len(self._slh)
        any_fresh = (int(nf) if self._counts is None else int(self._counts.max(initial=0))) > 0
        self.io = DartHostIo(_ptr(a["in_host"]), _ptr(a["in_dev"]), a["in_host"].numel() * a["in_host"].element_size(),
                             _ptr(a["out_dev"]), _ptr(a["out_host"]), a["out_host"].numel() * a["out_host"].element_size())
        self.sin = DartStepIn(B, int(nf) if self._counts is None else int(self._counts.max(initial=0)),
                              _ptr(a["feats"]) if any_fresh else None, _ptr(a["tokens"]) if any_fresh else None,
                              _ptr(a["seq_lens"]), self._slh.ctypes.data, _ptr(a["k_cache"]), _ptr(a["v_cache"]), 0,
                              None if self._counts is None else self._counts.ctypes.data)
        self.sout = DartStepOut(_ptr(a["topk_ids"]), _ptr(a["topk_slogit"]), _ptr(a["logits"]))
        f0 = int(fr) if self._rows is None else int(self._rows.min())
        self.tin = DartTreeIn(B, f0, draft.cfg.K - f0 if a["n_levels"] is None else a["n_levels"], _ptr(a["topk_ids"]),
                              _ptr(a["topk_slogit"]), _ptr(a["ctx_tail"]), None if self._rows is None else self._rows.ctypes.data)
        self.tout = DartTreeOut(_ptr(a["tree_tokens"]), _ptr(a["parents"]), _ptr(a["depth"]), _ptr(a["mask"]),
                                _ptr(a["n_nodes"]), _ptr(a["scores"]))
        self._st = draft._stream(stream)
        self._fn = lib().dart_draft_step_host
        self._args = (draft._h, C.byref(self.io), C.byref(self.sin), C.byref(self.sout), C.byref(self.tin), C.byref(self.tout),
                      self._st)

    def __call__(self, step_counter: int = 0) -> None:
        self.sin.step_counter = step_counter
        rc = self._fn(*self._args)
        if rc != DART_OK:
            raise DartError(rc, "dart_draft_step_host", lib().dart_last_cuda_error(self._draft._h))
