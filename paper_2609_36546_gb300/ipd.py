"""ctypes binding of libipd.so: argument marshalling only.

Every function here forwards torch tensors (device memory) as raw pointers to
the C ABI declared in include/ipd.h and raises IpdError on a non-zero status.
No step of the computation runs in Python, and there is no fallback: if the
shared library cannot be loaded, importing the binding fails.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_lib", "libipd.so")

IPD_OK = 0
STATUS = {0: "IPD_OK", 1: "IPD_ERR_INVALID_ARG", 2: "IPD_ERR_UNSUPPORTED", 3: "IPD_ERR_WORKSPACE",
          4: "IPD_ERR_CUDA", 5: "IPD_ERR_TIMEOUT", 6: "IPD_ERR_DEVICE", 7: "IPD_ERR_CAPACITY"}
STATUS_CODES = {v: k for k, v in STATUS.items()}
DEVERR = {0: "none", 1: "page id", 2: "seq len", 3: "token id", 4: "plan overflow", 5: "wait",
          6: "span offsets", 7: "rotary position", 8: "sampling settings"}

DIR_SPLIT, DIR_REVERSE, DIR_FORWARD, DIR_INVERSE = 0, 1, 2, 3
AGG_SEQ_MEAN_TOKEN_MEAN, AGG_GLOBAL_TOKEN_MEAN = 0, 1
LOSS_FIELDS = ("loss", "sum_on", "sum_off", "n_on", "n_off", "intervention_ratio", "numer", "denom")

# Exported symbols of include/ipd.h (checked by the CPU test suite).
EXPORTS = ("ipd_attn_workspace_size", "ipd_verify_attn", "ipd_decode_attn",
           "ipd_score_workspace_size", "ipd_score_span", "ipd_loss_workspace_size",
           "ipd_split_loss", "ipd_get_device_error", "ipd_status_string", "ipd_version",
           "ipd_score_span_static", "ipd_score_span_ex", "ipd_score_span_needed", "ipd_full_kl",
           "ipd_loss_grad_workspace_size", "ipd_split_loss_grad", "ipd_sample_workspace_size",
           "ipd_sample", "ipd_kv_append", "ipd_kv_append_many", "ipd_set_attn_kernel_timing",
           "ipd_attn_kernel_time", "ipd_device_readable", "ipd_rope_table", "ipd_rope",
           "ipd_rope_append", "ipd_prompt_attn", "ipd_sample_trunc")
# takeover / handback rules (IPD_RULE_*)
RULE_TOPK, RULE_ENTROPY_S, RULE_ENTROPY_T, RULE_ALWAYS, RULE_NEVER = 0, 1, 2, 3, 4
# element type of the dense gradient (IPD_DTYPE_*)
DTYPE_F32, DTYPE_BF16 = 0, 1
TRUNC_MAX_VOCAB = 262136  # IPD_TRUNC_MAX_VOCAB
STATIC_MAX_TOKENS = 4096  # IPD_STATIC_MAX_TOKENS
# rotary layouts and frequency scalings (IPD_ROPE_*, IPD_ROPE_SCALE_*)
ROPE_HALF, ROPE_INTERLEAVED = 0, 1
ROPE_SCALE = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}


class IpdError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {STATUS.get(status, status)}")
        self.status = status


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"libipd.so not built ({LIB_PATH}); run __graft_entry__.build()")
    return ctypes.CDLL(LIB_PATH)


_lib = _load()

c_p = ctypes.c_void_p
c_i = ctypes.c_int
c_sz = ctypes.c_size_t


class _KVCache(ctypes.Structure):
    _fields_ = [("k_pages", c_p), ("v_pages", c_p), ("num_pages", ctypes.c_int64),
                ("page_size", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32)]


class _ScoreExt(ctypes.Structure):
    _fields_ = [("takeover_rule", ctypes.c_int32), ("handback_rule", ctypes.c_int32),
                ("takeover_tau", ctypes.c_float), ("handback_tau", ctypes.c_float),
                ("entropy_s", c_p), ("entropy_t", c_p), ("topk_overlap", c_p),
                ("topk_s", c_p), ("topk_t", c_p), ("next_token", c_p), ("draw_base", c_p),
                ("sample_seed", ctypes.c_uint64), ("inv_temperature", ctypes.c_float)]


class _KvAppendDesc(ctypes.Structure):
    _fields_ = [("k_pages", c_p), ("v_pages", c_p), ("num_pages", ctypes.c_int64),
                ("num_kv_heads", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("k_new", c_p), ("v_new", c_p), ("cu_new", c_p),
                ("seq_len", c_p), ("page_table", c_p), ("max_pages", ctypes.c_int32),
                ("num_reqs", ctypes.c_int32), ("total_new", ctypes.c_int32)]


class _AttnBatch(ctypes.Structure):
    _fields_ = [("cache", ctypes.POINTER(_KVCache)), ("num_q_heads", ctypes.c_int32),
                ("num_reqs", ctypes.c_int32), ("q", c_p), ("cu_q", c_p), ("seq_len", c_p),
                ("page_table", c_p), ("max_pages", ctypes.c_int32), ("total_q", ctypes.c_int32),
                ("max_q_len", ctypes.c_int32), ("max_seq_len", ctypes.c_int32), ("out", c_p)]


class _RopeScaling(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("base", ctypes.c_double), ("factor", ctypes.c_double),
                ("trained_len", ctypes.c_double), ("beta_fast", ctypes.c_double),
                ("beta_slow", ctypes.c_double)]


class _RopeArgs(ctypes.Structure):
    _fields_ = [("x", c_p), ("y", c_p), ("x_stride", ctypes.c_int64), ("y_stride", ctypes.c_int64),
                ("pos", c_p), ("table", c_p)] + \
        [(n, ctypes.c_int32) for n in ("dtype", "n_tokens", "n_heads", "head_dim", "max_pos",
                                       "rot_dim", "layout", "inverse")]


class _RopeAppendDesc(ctypes.Structure):
    _fields_ = [(n, c_p) for n in ("q", "k", "v", "q_out", "k_out")] + \
        [(n, ctypes.c_int64) for n in ("q_stride", "k_stride", "v_stride", "q_out_stride",
                                       "k_out_stride")] + \
        [("k_pages", c_p), ("v_pages", c_p), ("num_pages", ctypes.c_int64), ("cu_new", c_p),
         ("seq_len", c_p), ("page_table", c_p), ("table", c_p)] + \
        [(n, ctypes.c_int32) for n in ("num_q_heads", "num_kv_heads", "page_size", "head_dim",
                                       "max_pages", "num_reqs", "total_new", "max_pos", "rot_dim",
                                       "layout")]


class _PromptArgs(ctypes.Structure):
    _fields_ = [(n, c_p) for n in ("q", "k", "v", "out", "lse", "cu_seq")] + \
        [(n, ctypes.c_int64) for n in ("q_stride", "k_stride", "v_stride", "out_stride")] + \
        [(n, ctypes.c_int32) for n in ("num_q_heads", "num_kv_heads", "head_dim", "num_seqs",
                                       "total", "max_len")] + [("softmax_scale", ctypes.c_float)]


# The same three layouts as packed bytes: filling a ctypes structure field by
# field takes longer than the smallest of these calls runs.
_PACK_ROPE = struct.Struct("2P2q2P8i")
_PACK_ROPE_APPEND = struct.Struct("5P5q2Pq4P10i")
_PACK_PROMPT = struct.Struct("6P4q6if0P")
for _s, _c in ((_PACK_ROPE, _RopeArgs), (_PACK_ROPE_APPEND, _RopeAppendDesc),
               (_PACK_PROMPT, _PromptArgs)):
    assert _s.size == ctypes.sizeof(_c), _c.__name__

_lib.ipd_attn_workspace_size.restype = c_sz
_lib.ipd_attn_workspace_size.argtypes = [ctypes.POINTER(_AttnBatch), c_i,
                                         ctypes.POINTER(_AttnBatch), c_i]
_lib.ipd_verify_attn.restype = c_i
_lib.ipd_verify_attn.argtypes = [ctypes.POINTER(_AttnBatch), c_i, ctypes.POINTER(_AttnBatch), c_i,
                                 ctypes.c_float, c_p, c_sz, c_p]
_lib.ipd_decode_attn.restype = c_i
_lib.ipd_decode_attn.argtypes = [ctypes.POINTER(_AttnBatch), c_i, ctypes.c_float, c_p, c_sz, c_p]
_lib.ipd_score_workspace_size.restype = c_sz
_lib.ipd_score_workspace_size.argtypes = [c_i, c_i, c_i, c_i]
_lib.ipd_score_span.restype = c_i
_lib.ipd_score_span.argtypes = [c_p] * 6 + [c_i] * 5 + [c_p] * 13 + [c_p, c_sz, c_p]
_lib.ipd_device_readable.restype = c_i
_lib.ipd_device_readable.argtypes = [c_p, ctypes.POINTER(c_i)]
_lib.ipd_score_span_needed.restype = c_i
_lib.ipd_score_span_needed.argtypes = [c_p] * 6 + [c_i] * 6 + [c_p] * 13 + [c_p, c_sz, c_p]
_lib.ipd_score_span_ex.restype = c_i
_lib.ipd_score_span_ex.argtypes = ([c_p] * 6 + [c_i] * 5 + [c_p] * 13 +
                                   [ctypes.POINTER(_ScoreExt), c_p, c_sz, c_p])
_lib.ipd_full_kl.restype = c_i
_lib.ipd_full_kl.argtypes = [c_p, c_p, c_i, c_i, c_p, c_p, c_p]
_lib.ipd_score_span_static.restype = c_i
_lib.ipd_score_span_static.argtypes = [c_p] * 6 + [c_i] * 5 + [c_p] * 13 + [c_p]
_lib.ipd_loss_workspace_size.restype = c_sz
_lib.ipd_loss_workspace_size.argtypes = [c_i]
_lib.ipd_split_loss.restype = c_i
_lib.ipd_split_loss.argtypes = [c_p] * 6 + [c_i, c_i, c_i, c_p, c_p, c_sz, c_p]
_lib.ipd_loss_grad_workspace_size.restype = c_sz
_lib.ipd_loss_grad_workspace_size.argtypes = [c_i, c_i]
_lib.ipd_split_loss_grad.restype = c_i
_lib.ipd_split_loss_grad.argtypes = ([c_p] * 9 + [c_i] * 6 + [ctypes.c_float, c_p, c_p, c_p, c_i,
                                      c_p, c_sz, c_p])
_lib.ipd_sample_workspace_size.restype = c_sz
_lib.ipd_sample_workspace_size.argtypes = [c_i, c_i]
_lib.ipd_sample.restype = c_i
_lib.ipd_sample.argtypes = [c_p, c_i, c_i, ctypes.c_uint64, c_p, ctypes.c_float, c_p, c_p, c_sz,
                            c_p]
_lib.ipd_kv_append.restype = c_i
_lib.ipd_kv_append.argtypes = [c_p, c_p, ctypes.c_int64, c_i, c_i, c_i, c_p, c_p, c_p, c_p, c_p,
                               c_i, c_i, c_i, c_p]
_lib.ipd_kv_append_many.restype = c_i
_lib.ipd_kv_append_many.argtypes = [ctypes.POINTER(_KvAppendDesc), c_i, c_p]
_lib.ipd_rope_table.restype = c_i
_lib.ipd_rope_table.argtypes = [c_p, c_i, c_i, ctypes.POINTER(_RopeScaling), c_p]
_lib.ipd_rope.restype = c_i
_lib.ipd_rope.argtypes = [c_p, c_p]  # (a packed _RopeArgs, as bytes)
_lib.ipd_rope_append.restype = c_i
_lib.ipd_rope_append.argtypes = [c_p, c_p]  # (a packed _RopeAppendDesc)
_lib.ipd_prompt_attn.restype = c_i
_lib.ipd_prompt_attn.argtypes = [c_p, c_p]  # (a packed _PromptArgs)
_lib.ipd_sample_trunc.restype = c_i
_lib.ipd_sample_trunc.argtypes = [c_p, ctypes.c_int64, c_i, c_i] + [c_p] * 9
_lib.ipd_set_attn_kernel_timing.restype = c_i
_lib.ipd_set_attn_kernel_timing.argtypes = [c_i]
_lib.ipd_attn_kernel_time.restype = c_i
_lib.ipd_attn_kernel_time.argtypes = [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(c_i)]
_lib.ipd_get_device_error.restype = c_i
_lib.ipd_get_device_error.argtypes = [ctypes.POINTER(ctypes.c_uint32)]
_lib.ipd_status_string.restype = ctypes.c_char_p
_lib.ipd_status_string.argtypes = [c_i]
_lib.ipd_version.restype = c_i


def lib() -> ctypes.CDLL:
    return _lib


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    return t.data_ptr()


_F32, _BF16, _I32 = torch.float32, torch.bfloat16, torch.int32
# the raw handle of the current stream, without the objects around it (a few
# microseconds a call; the small operators run for as little)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_on_gpu = False  # set once a device has been seen


def _stream(stream) -> Optional[int]:
    global _on_gpu
    if stream is None:
        if not _on_gpu:
            if not torch.cuda.is_available():
                return None
            torch.cuda.current_stream()  # initialises CUDA in this process
            _on_gpu = True
        if _raw_stream is not None:
            return _raw_stream(_device())
        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _check(st: int, what: str):
    if st != IPD_OK:
        raise IpdError(st, what)


class KVCache:
    """A paged KV cache: k_pages / v_pages are [num_pages, Hkv, 16, 128] bf16."""

    def __init__(self, k_pages: torch.Tensor, v_pages: torch.Tensor):
        assert k_pages.shape == v_pages.shape and k_pages.dim() == 4
        self.k_pages, self.v_pages = k_pages, v_pages
        self._c = None

    @property
    def c(self) -> _KVCache:
        """The C descriptor (made when first asked for)."""
        if self._c is None:
            k = self.k_pages
            self._c = _KVCache(_ptr(k), _ptr(self.v_pages), k.shape[0], k.shape[2], k.shape[1],
                               k.shape[3])
        return self._c

    @property
    def num_kv_heads(self) -> int:
        return self.k_pages.shape[1]


class AttnBatch:
    """One sub-batch of requests attending one cache (see ipd_attn_batch).

    q [total_q, Hq, 128] bf16, cu_q [R+1] int32, seq_len [R] int32,
    page_table [R, max_pages] int32, out [total_q, Hq, 128] bf16 (all device);
    max_q_len / max_seq_len are host-known bounds."""

    def __init__(self, cache: KVCache, q, cu_q, seq_len, page_table, out, max_q_len: int,
                 max_seq_len: int):
        self.cache = cache
        self._keep = (q, cu_q, seq_len, page_table, out)
        R = seq_len.numel()
        self.c = _AttnBatch(ctypes.pointer(cache.c), q.shape[1], R, _ptr(q), _ptr(cu_q),
                            _ptr(seq_len), _ptr(page_table), page_table.shape[1], q.shape[0],
                            max_q_len, max_seq_len, _ptr(out))
        self.out = out


def _arr(batches: Sequence[AttnBatch]):
    n = len(batches)
    if n == 0:
        return None, 0
    a = (_AttnBatch * n)(*[b.c for b in batches])
    return a, n


def attn_workspace_size(verify: Sequence[AttnBatch], decode: Sequence[AttnBatch] = ()) -> int:
    va, nv = _arr(verify)
    da, nd = _arr(decode)
    return int(_lib.ipd_attn_workspace_size(va, nv, da, nd))


def verify_attn(verify: Sequence[AttnBatch], decode: Sequence[AttnBatch], softmax_scale: float,
                workspace: torch.Tensor, stream=None):
    va, nv = _arr(verify)
    da, nd = _arr(decode)
    _check(_lib.ipd_verify_attn(va, nv, da, nd, softmax_scale, _ptr(workspace),
                                workspace.numel() * workspace.element_size(), _stream(stream)),
           "ipd_verify_attn")


def decode_attn(decode: Sequence[AttnBatch], softmax_scale: float, workspace: torch.Tensor,
                stream=None):
    da, nd = _arr(decode)
    _check(_lib.ipd_decode_attn(da, nd, softmax_scale, _ptr(workspace),
                                workspace.numel() * workspace.element_size(), _stream(stream)),
           "ipd_decode_attn")


def score_workspace_size(num_reqs: int, total_tokens: int, vocab: int, K: int) -> int:
    return int(_lib.ipd_score_workspace_size(num_reqs, total_tokens, vocab, K))


SCORE_TOKEN_OUTPUTS = (("logp_s", torch.float32), ("logp_t", torch.float32),
                       ("feedback", torch.float32), ("kl_rev", torch.float32),
                       ("kl_fwd", torch.float32), ("covered", torch.uint8),
                       ("margin", torch.float32), ("source", torch.uint8))
SCORE_REQ_OUTPUTS = (("first_trans", torch.int32), ("n_emit", torch.int32),
                     ("next_driver", torch.uint8), ("new_len", torch.int32), ("done", torch.uint8))


def alloc_score_outputs(num_reqs: int, total_tokens: int, device) -> dict:
    out = {n: torch.empty(total_tokens, dtype=dt, device=device) for n, dt in SCORE_TOKEN_OUTPUTS}
    out.update({n: torch.empty(num_reqs, dtype=dt, device=device) for n, dt in SCORE_REQ_OUTPUTS})
    return out


def score_span(logits_student, logits_teacher, tokens, cu_span, driver, prefix_len, K: int,
               eos_id: int, out: dict, workspace: torch.Tensor, stream=None):
    R = driver.numel()
    T, V = logits_student.shape
    _check(_lib.ipd_score_span(
        _ptr(logits_student), _ptr(logits_teacher), _ptr(tokens), _ptr(cu_span), _ptr(driver),
        _ptr(prefix_len), R, T, V, K, eos_id,
        *[_ptr(out[n]) for n, _ in SCORE_TOKEN_OUTPUTS],
        *[_ptr(out[n]) for n, _ in SCORE_REQ_OUTPUTS],
        _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
        "ipd_score_span")


def device_readable(t: torch.Tensor) -> bool:
    """Whether the library's kernels can read tensor t where it lives (device
    memory, or pinned host memory mapped into the device's address space)."""
    r = c_i(0)
    _check(_lib.ipd_device_readable(_ptr(t), ctypes.byref(r)), "ipd_device_readable")
    return bool(r.value)


def score_span_needed(logits_student, logits_teacher, tokens, cu_span, driver, prefix_len,
                      K: int, eos_id: int, max_span: int, out: dict, workspace: torch.Tensor,
                      stream=None):
    """ipd_score_span reading only the rows the verdict and the emitted
    positions need; ``max_span`` bounds every request's span length."""
    R = driver.numel()
    T, V = logits_student.shape
    _check(_lib.ipd_score_span_needed(
        _ptr(logits_student), _ptr(logits_teacher), _ptr(tokens), _ptr(cu_span), _ptr(driver),
        _ptr(prefix_len), R, T, V, K, eos_id, max_span,
        *[_ptr(out[n]) for n, _ in SCORE_TOKEN_OUTPUTS],
        *[_ptr(out[n]) for n, _ in SCORE_REQ_OUTPUTS],
        _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
        "ipd_score_span_needed")


def score_span_ex(logits_student, logits_teacher, tokens, cu_span, driver, prefix_len, K: int,
                  eos_id: int, out: dict, workspace: torch.Tensor, takeover_rule: int = RULE_TOPK,
                  handback_rule: int = RULE_TOPK, takeover_tau: float = 0.0,
                  handback_tau: float = 0.0, entropy_s: Optional[torch.Tensor] = None,
                  entropy_t: Optional[torch.Tensor] = None,
                  topk_overlap: Optional[torch.Tensor] = None,
                  topk_s: Optional[torch.Tensor] = None, topk_t: Optional[torch.Tensor] = None,
                  next_token: Optional[torch.Tensor] = None,
                  draw_base: Optional[torch.Tensor] = None, sample_seed: int = 0,
                  inv_temperature: float = 1.0, stream=None):
    """ipd_score_span with selectable takeover / handback rules and the
    optional per-token entropies and top-K overlap ratio (fp32 [T] tensors),
    top-K id lists (int32 [T, K]) and the next span's first token per request
    (int32 [R]; draw numbers from ``draw_base``, uint64 as int64 [R])."""
    R = driver.numel()
    T, V = logits_student.shape
    ext = _ScoreExt(takeover_rule, handback_rule, takeover_tau, handback_tau,
                    _ptr(entropy_s), _ptr(entropy_t), _ptr(topk_overlap), _ptr(topk_s),
                    _ptr(topk_t), _ptr(next_token), _ptr(draw_base),
                    sample_seed & 0xFFFFFFFFFFFFFFFF, inv_temperature)
    _check(_lib.ipd_score_span_ex(
        _ptr(logits_student), _ptr(logits_teacher), _ptr(tokens), _ptr(cu_span), _ptr(driver),
        _ptr(prefix_len), R, T, V, K, eos_id,
        *[_ptr(out[n]) for n, _ in SCORE_TOKEN_OUTPUTS],
        *[_ptr(out[n]) for n, _ in SCORE_REQ_OUTPUTS],
        ctypes.byref(ext), _ptr(workspace), workspace.numel() * workspace.element_size(),
        _stream(stream)), "ipd_score_span_ex")


def full_kl(logits_student, logits_teacher, kl_rev_full: torch.Tensor, kl_fwd_full: torch.Tensor,
            stream=None):
    """Full-vocabulary KL in both directions at every span position."""
    T, V = logits_student.shape
    _check(_lib.ipd_full_kl(_ptr(logits_student), _ptr(logits_teacher), T, V, _ptr(kl_rev_full),
                            _ptr(kl_fwd_full), _stream(stream)), "ipd_full_kl")


def score_span_static(logits_student, logits_teacher, tokens, cu_span, driver, prefix_len,
                      K: int, eos_id: int, out: dict, stream=None):
    """ipd_score_span without a workspace: for callers that cannot allocate
    device memory (the scratch is the library's static device array, at most
    STATIC_MAX_TOKENS span positions; overlapping calls race on it)."""
    R = driver.numel()
    T, V = logits_student.shape
    _check(_lib.ipd_score_span_static(
        _ptr(logits_student), _ptr(logits_teacher), _ptr(tokens), _ptr(cu_span), _ptr(driver),
        _ptr(prefix_len), R, T, V, K, eos_id,
        *[_ptr(out[n]) for n, _ in SCORE_TOKEN_OUTPUTS],
        *[_ptr(out[n]) for n, _ in SCORE_REQ_OUTPUTS],
        _stream(stream)), "ipd_score_span_static")


def split_loss(kl_rev, kl_fwd, source, cu_span, n_emit, resp_len, agg_mode: int, dir_mode: int,
               out8: torch.Tensor, stream=None):
    R = cu_span.numel() - 1
    _check(_lib.ipd_split_loss(_ptr(kl_rev), _ptr(kl_fwd), _ptr(source), _ptr(cu_span),
                               _ptr(n_emit), _ptr(resp_len), R, agg_mode, dir_mode, _ptr(out8),
                               None, 0, _stream(stream)), "ipd_split_loss")


def kv_append(cache: "KVCache", k_new, v_new, cu_new, seq_len, page_table, stream=None):
    """Writes the new tokens' K/V rows ([n, Hkv, 128] bf16) into the cache's
    pages at the last positions of each request's sequence (``seq_len`` is
    the length after the append)."""
    R = cu_new.numel() - 1
    _check(_lib.ipd_kv_append(_ptr(cache.k_pages), _ptr(cache.v_pages), cache.k_pages.shape[0],
                              cache.k_pages.shape[1], 16, 128, _ptr(k_new), _ptr(v_new),
                              _ptr(cu_new), _ptr(seq_len), _ptr(page_table),
                              page_table.shape[1], R, k_new.shape[0], _stream(stream)),
           "ipd_kv_append")


def kv_append_many(appends, stream=None):
    """Several appends in one launch: ``appends`` is a sequence of (cache,
    k_new, v_new, cu_new, seq_len, page_table) tuples, each as in kv_append."""
    n = len(appends)
    arr = (_KvAppendDesc * max(n, 1))()
    for i, (cache, k_new, v_new, cu_new, seq_len, page_table) in enumerate(appends):
        arr[i] = _KvAppendDesc(_ptr(cache.k_pages), _ptr(cache.v_pages), cache.k_pages.shape[0],
                               cache.k_pages.shape[1], 16, 128, _ptr(k_new), _ptr(v_new),
                               _ptr(cu_new), _ptr(seq_len), _ptr(page_table),
                               page_table.shape[1], cu_new.numel() - 1, k_new.shape[0])
    _check(_lib.ipd_kv_append_many(arr, n, _stream(stream)), "ipd_kv_append_many")


def sample_workspace_size(n_rows: int, vocab: int) -> int:
    return int(_lib.ipd_sample_workspace_size(n_rows, vocab))


def sample(logits, seed: int, draw_id: Optional[torch.Tensor], tokens: torch.Tensor,
           workspace: torch.Tensor, inv_temperature: float = 1.0, stream=None):
    """One seeded draw per row of ``logits`` ([n, V] bf16) into ``tokens``
    (int32 [n]); ``draw_id`` holds the rows' uint64 draw numbers (as int64)."""
    n, V = logits.shape
    _check(_lib.ipd_sample(_ptr(logits), n, V, seed & 0xFFFFFFFFFFFFFFFF, _ptr(draw_id),
                           inv_temperature, _ptr(tokens), _ptr(workspace),
                           workspace.numel() * workspace.element_size(), _stream(stream)),
           "ipd_sample")


def split_loss_grad(logits_student, logits_teacher, topk_s, topk_t, source, cu_span, n_emit,
                    resp_len, loss_out8, K: int, agg_mode: int, dir_mode: int, grad_scale: float,
                    grad_idx: torch.Tensor, grad_val: torch.Tensor,
                    grad_dense: Optional[torch.Tensor] = None, stream=None):
    """Gradient of grad_scale * loss with respect to the student's logits:
    sparse [T, 2K] ids / values, and the dense [T, V] form when ``grad_dense``
    (fp32 or bf16) is given."""
    R = cu_span.numel() - 1
    T, V = logits_student.shape
    dtype = DTYPE_F32
    if grad_dense is not None:
        if grad_dense.dtype == torch.bfloat16:
            dtype = DTYPE_BF16
        elif grad_dense.dtype != torch.float32:
            raise IpdError(STATUS_CODES["IPD_ERR_INVALID_ARG"], "ipd_split_loss_grad: dense dtype")
    _check(_lib.ipd_split_loss_grad(
        _ptr(logits_student), _ptr(logits_teacher), _ptr(topk_s), _ptr(topk_t), _ptr(source),
        _ptr(cu_span), _ptr(n_emit), _ptr(resp_len), _ptr(loss_out8), R, T, V, K, agg_mode,
        dir_mode, grad_scale, _ptr(grad_idx), _ptr(grad_val), _ptr(grad_dense), dtype, None, 0,
        _stream(stream)), "ipd_split_loss_grad")


def _refuse(what: str):
    raise IpdError(STATUS_CODES["IPD_ERR_INVALID_ARG"], what)


def _rows(t: torch.Tensor, shape, dtype, what: str) -> int:
    """Token stride of a [n, heads, head_dim] tensor whose rows are contiguous."""
    if t.shape != shape or t.dtype is not dtype:
        _refuse(what)
    n, h, d = shape
    s0, s1, s2 = t.stride()
    if (s2 != 1 or s1 != d) and ((d > 1 and s2 != 1) or (h > 1 and s1 != d)):
        _refuse(what)
    return s0 if n > 1 else h * d


def _check_table(table: torch.Tensor, what: str):
    """(positions, rotated entries) of a rotary table."""
    s = table.shape
    if len(s) != 3 or s[2] != 2 or table.dtype is not _F32 or not table.is_contiguous():
        _refuse(what)
    return s[0], 2 * s[1]


def rope_table(table: torch.Tensor, base: float = 1e6, scaling: str = "none", factor: float = 1.0,
               trained_len: float = 32768.0, beta_fast: float = 32.0, beta_slow: float = 1.0,
               stream=None):
    """Fills ``table`` ([max_pos, rot_dim / 2, 2] fp32) with (cos, sin) of
    position times frequency; ``scaling`` is a key of ROPE_SCALE."""
    _check_table(table, "ipd_rope_table: table")
    if scaling not in ROPE_SCALE:
        _refuse("ipd_rope_table: scaling")
    c = _RopeScaling(ROPE_SCALE[scaling], base, factor, trained_len, beta_fast, beta_slow)
    _check(_lib.ipd_rope_table(table.data_ptr(), table.shape[0], 2 * table.shape[1],
                               ctypes.byref(c), _stream(stream)), "ipd_rope_table")


def rope(x: torch.Tensor, out: torch.Tensor, pos: torch.Tensor, table: torch.Tensor,
         layout: int = ROPE_HALF, inverse: bool = False, stream=None):
    """Rotates the heads of ``x`` ([n, H, D] bf16 or fp32, rows contiguous) by
    their positions ``pos`` (int32 [n]) into ``out`` (may be ``x``); ``inverse``
    applies the transpose, the rotation's gradient."""
    max_pos, rot = _check_table(table, "ipd_rope: table")
    shape, dt = tuple(x.shape), x.dtype
    if len(shape) != 3 or (dt is not _BF16 and dt is not _F32) or pos.dtype is not _I32 or \
            pos.shape != shape[:1] or not pos.is_contiguous():
        _refuse("ipd_rope: shapes or types")
    n, h, d = shape
    a = _PACK_ROPE.pack(x.data_ptr(), out.data_ptr(), _rows(x, shape, dt, "ipd_rope: x"),
                        _rows(out, shape, dt, "ipd_rope: out"), pos.data_ptr(), table.data_ptr(),
                        DTYPE_BF16 if dt is _BF16 else DTYPE_F32, n, h, d, max_pos, rot,
                        layout, 1 if inverse else 0)
    _check(_lib.ipd_rope(a, _stream(stream)), "ipd_rope")


def rope_append(cache: "KVCache", q: Optional[torch.Tensor], q_out: Optional[torch.Tensor],
                k_new, v_new, cu_new, seq_len, page_table, table: torch.Tensor,
                layout: int = ROPE_HALF, k_out: Optional[torch.Tensor] = None, stream=None):
    """Rotates the new tokens' queries ([n, Hq, 128] bf16, or None) into
    ``q_out`` and their keys ([n, Hkv, 128]) into the cache's pages (and
    ``k_out``), and writes their values beside them: kv_append of the rotated
    rows in one launch.  Each row's position is its place in its sequence.
    ``cu_new`` [R + 1], ``seq_len`` [R] and ``page_table`` [R, max_pages] are
    contiguous int32 (the last two may hold more rows than R, not fewer)."""
    max_pos, rot = _check_table(table, "ipd_rope_append: table")
    bf, kp, vp, kshape = _BF16, cache.k_pages, cache.v_pages, tuple(k_new.shape)
    pshape = kp.shape
    pages, hkv, ps, hd = pshape
    n, hq, R = kshape[0], 0, cu_new.numel() - 1
    # what goes on as a bare pointer is read and written as laid out here
    if kp.dtype is not bf or vp.dtype is not bf or vp.shape != pshape or \
            not kp.is_contiguous() or not vp.is_contiguous():
        _refuse("ipd_rope_append: pools")
    tshape = page_table.shape
    if cu_new.dtype is not _I32 or seq_len.dtype is not _I32 or page_table.dtype is not _I32 or \
            cu_new.dim() != 1 or R < 0 or seq_len.numel() < R or len(tshape) != 2 or \
            tshape[0] < R or not cu_new.is_contiguous() or not seq_len.is_contiguous() or \
            not page_table.is_contiguous():
        _refuse("ipd_rope_append: offsets, lengths or page table")
    q_ptr = qo_ptr = ko_ptr = qs = qos = kos = 0
    if kshape != (n, hkv, 128) or (q is None) != (q_out is None):
        _refuse("ipd_rope_append: shapes")
    if q is not None:
        qshape = tuple(q.shape)
        hq = qshape[1] if len(qshape) == 3 else 0
        if qshape != (n, hq, 128):
            _refuse("ipd_rope_append: q")
        q_ptr, qs = q.data_ptr(), _rows(q, qshape, bf, "ipd_rope_append: q")
        qo_ptr, qos = q_out.data_ptr(), _rows(q_out, qshape, bf, "ipd_rope_append: q_out")
    if k_out is not None:
        ko_ptr, kos = k_out.data_ptr(), _rows(k_out, kshape, bf, "ipd_rope_append: k_out")
    a = _PACK_ROPE_APPEND.pack(
        q_ptr, k_new.data_ptr(), v_new.data_ptr(), qo_ptr, ko_ptr, qs,
        _rows(k_new, kshape, bf, "ipd_rope_append: k_new"),
        _rows(v_new, kshape, bf, "ipd_rope_append: v_new"), qos, kos, kp.data_ptr(),
        vp.data_ptr(), pages, cu_new.data_ptr(), seq_len.data_ptr(),
        page_table.data_ptr(), table.data_ptr(), hq, hkv, ps, hd, tshape[1],
        R, n, max_pos, rot, layout)
    _check(_lib.ipd_rope_append(a, _stream(stream)), "ipd_rope_append")


def prompt_attn(q, k, v, cu_seq, max_len: int, out, softmax_scale: float,
                lse: Optional[torch.Tensor] = None, stream=None):
    """Causal attention of packed prompts: q [total, Hq, 128], k and v
    [total, Hkv, 128], out [total, Hq, 128] bf16 (rows contiguous, any row
    stride), cu_seq int32 [num_seqs + 1] (device), ``max_len`` a host-known
    bound on the lengths (0: every sequence is empty, and nothing is done);
    lse fp32 [Hq, total] when given."""
    shape, kshape, bf = tuple(q.shape), tuple(k.shape), _BF16
    if len(shape) != 3 or len(kshape) != 3 or kshape[0] != shape[0] or kshape[2] != shape[2] or \
            cu_seq.dtype is not _I32 or not cu_seq.is_contiguous():
        _refuse("ipd_prompt_attn: shapes or types")
    n, hq, d = shape
    if lse is not None and (lse.shape != (hq, n) or lse.dtype is not torch.float32 or
                            not lse.is_contiguous()):
        _refuse("ipd_prompt_attn: lse")
    a = _PACK_PROMPT.pack(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                          0 if lse is None else lse.data_ptr(), cu_seq.data_ptr(),
                          _rows(q, shape, bf, "ipd_prompt_attn: q"),
                          _rows(k, kshape, bf, "ipd_prompt_attn: k"),
                          _rows(v, kshape, bf, "ipd_prompt_attn: v"),
                          _rows(out, shape, bf, "ipd_prompt_attn: out"), hq, kshape[1], d,
                          cu_seq.shape[0] - 1, n, max_len, softmax_scale)
    _check(_lib.ipd_prompt_attn(a, _stream(stream)), "ipd_prompt_attn")


def sample_trunc(logits: torch.Tensor, u: torch.Tensor, tokens: torch.Tensor,
                 inv_temperature: Optional[torch.Tensor] = None,
                 top_k: Optional[torch.Tensor] = None, top_p: Optional[torch.Tensor] = None,
                 min_p: Optional[torch.Tensor] = None, logp: Optional[torch.Tensor] = None,
                 n_kept: Optional[torch.Tensor] = None, stream=None):
    """One token per row of ``logits`` ([n, V] bf16, entries contiguous, any row
    stride) into ``tokens`` (int32 [n]), drawn with the uniform numbers ``u``
    (fp32 [n]) after the rows' own settings (fp32 [n]; ``top_k`` int32 [n]);
    ``logp`` (fp32) and ``n_kept`` (int32) take the log-probability of the token
    among the kept entries and their number."""
    n, V = logits.shape
    one, f, i = (n,), _F32, _I32
    for t, dt in ((u, f), (tokens, i), (inv_temperature, f), (top_k, i), (top_p, f), (min_p, f),
                  (logp, f), (n_kept, i)):
        if t is not None and (t.shape != one or t.dtype is not dt or not t.is_contiguous()):
            _refuse("ipd_sample_trunc: per-row tensors")
    row, col = logits.stride()
    if logits.dtype is not torch.bfloat16 or (V > 1 and col != 1):
        _refuse("ipd_sample_trunc: logits")
    _check(_lib.ipd_sample_trunc(logits.data_ptr(), row if n > 1 else V, n, V,
                                 u.data_ptr(), _ptr(inv_temperature), _ptr(top_k), _ptr(top_p),
                                 _ptr(min_p), tokens.data_ptr(), _ptr(logp), _ptr(n_kept),
                                 _stream(stream)), "ipd_sample_trunc")


def set_attn_kernel_timing(on: bool):
    _check(_lib.ipd_set_attn_kernel_timing(1 if on else 0), "ipd_set_attn_kernel_timing")


def attn_kernel_time():
    """(summed ms, launches) of the attention kernels timed since timing was
    switched on or last read (synchronises)."""
    ms = ctypes.c_double(0.0)
    n = c_i(0)
    _check(_lib.ipd_attn_kernel_time(ctypes.byref(ms), ctypes.byref(n)), "ipd_attn_kernel_time")
    return float(ms.value), int(n.value)


def device_error() -> int:
    """Reads and clears the device-side error word (synchronises)."""
    v = ctypes.c_uint32(0)
    _check(_lib.ipd_get_device_error(ctypes.byref(v)), "ipd_get_device_error")
    return int(v.value)
