"""Thin ctypes binding of libdopr.so (the C ABI in include/dopr.h).

Only argument marshalling lives here: every step of the scoring pass runs in
the library's CUDA kernels.  Importing this module loads the library and
raises if it has not been built (``python -m paper_2609_03311_gb300.build``);
there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
import struct

import numpy as np
import torch

from . import build as _build

_LIB = None

(OK, ERR_INVALID_ARG, ERR_UNKNOWN_DOC, ERR_INCOMPLETE, ERR_OUT_OF_MEMORY, ERR_CUDA, ERR_TIMEOUT, ERR_UNSUPPORTED,
 ERR_INTERNAL, ERR_RANGE) = range(10)
STATUS_NAMES = ["OK", "INVALID_ARG", "UNKNOWN_DOC", "INCOMPLETE", "OUT_OF_MEMORY", "CUDA", "TIMEOUT", "UNSUPPORTED",
                "INTERNAL", "RANGE"]

(W_EMBED, W_ATTN_NORM, W_Q, W_K, W_V, W_Q_NORM, W_K_NORM, W_O, W_MLP_NORM, W_GATE, W_UP, W_DOWN, W_FINAL_NORM,
 W_SCORE_HEAD) = range(14)

EPI_STORE, EPI_RESID_ADD, EPI_SWIGLU, EPI_QKV = 0, 1, 2, 3  # EPI_QKV: gemm_plan only


class DoprError(RuntimeError):
    def __init__(self, status: int, msg: str):
        self.status = status
        name = STATUS_NAMES[status] if 0 <= status < len(STATUS_NAMES) else str(status)
        super().__init__(f"DOPR_ERR_{name}: {msg}")


class KernelStat(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 24), ("launches", ctypes.c_int64), ("time_ms", ctypes.c_double),
                ("flops", ctypes.c_double), ("bytes", ctypes.c_double)]


class ModelConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_layers", "hidden", "n_q_heads", "n_kv_heads", "head_dim", "ffn",
                                              "vocab", "score_token_id", "max_position")] + \
               [("rope_theta", ctypes.c_float), ("rms_eps", ctypes.c_float)]


def lib_path() -> str:
    """The library this process loads: the checked build when DOPR_CHECKED=1."""
    return _build.LIB_CHECKED if os.environ.get("DOPR_CHECKED") == "1" else _build.LIB


def load():
    """Load libdopr.so; raises OSError if it is missing."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = lib_path()
    if not os.path.exists(path):
        raise OSError(f"libdopr.so not built at {path}; run paper_2609_03311_gb300.build.build()")
    L = ctypes.CDLL(path)
    P, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    sig = {
        "dopr_model_create": ([P, P], i32),
        "dopr_model_put_weight": ([P, i32, i32, P, i64, i32], i32),
        "dopr_model_destroy": ([P], i32),
        "dopr_store_create": ([P, i64, i64, P], i32),
        "dopr_store_put": ([P, i64, i32, i32, P, P, i32], i32),
        "dopr_store_destroy": ([P], i32),
        "dopr_prefix_bytes": ([P, i32], i64),
        "dopr_score": ([P, P, i32, P, P, P, P, P, i32], i32),
        "dopr_debug_pack_plan": ([P, P, i32, P, P, P, P, P, P, P, P], i32),
        "dopr_debug_gemm": ([i32, i32, i32, P, P, P, i32, P], i32),
        "dopr_debug_gemm_plan": ([i32, i32, i32, i32, i32, P], i32),
        "dopr_debug_wait_timeout": ([i32], i32),
        "dopr_pack_order_noalloc": ([P, i32, P, P, P, P, P], i32),
        "dopr_profile_enable": ([P, i32], i32),
        "dopr_profile_read": ([P, P, i32], i32),
        "dopr_build_prefixes": ([P, P, i32, P, P, P, i32, P], i32),
        "dopr_debug_store_read": ([P, i64, i32, P, P], i32),
        "dopr_debug_attention_plan": ([i32, i32, i32, P, i32, P], i32),
        "dopr_select_prefix_inputs": ([P, i32, P, P, i32, i32, P, P, P, P], i32),
        "dopr_model_set_mlp_head": ([P, i32, i32, P, P, P, ctypes.c_float, i32], i32),
        "dopr_cache_extend": ([P] * 7 + [i32] + [P] * 8, i32),
        "dopr_cache_extend_workspace": ([P], i64),
        "dopr_rope_create": ([P, P], i32),
        "dopr_rope_destroy": ([P], i32),
        "dopr_rope_apply": ([P, i32, i32, i32, P, P, P, P, P, i32, P, P], i32),
        "dopr_cache_append": ([P, P, i32] + [P] * 10, i32),
        "dopr_head_norm_rope": ([P, i32, i32, i32, P, ctypes.c_float, i32] + [P] * 8, i32),
        "dopr_head_norm_rope_backward": ([P, i32, i32, i32, P, ctypes.c_float, i32] + [P] * 13, i32),
        "dopr_head_norm_rope_workspace": ([i32], i64),
        "dopr_cache_4bit_pool_bytes": ([P], i64),
        "dopr_cache_append_4bit": ([P, P, i32, P, P, ctypes.c_float, i32] + [P] * 10, i32),
        "dopr_cache_read_4bit": ([P, i32] + [P] * 7, i32),
        "dopr_shared_attention_plan": ([P, i32, i32] + [P] * 6, i32),
        "dopr_shared_attention_plan_bytes": ([P, i32, i32], i64),
        "dopr_shared_attention": ([P, P, i32, P, P, P, P, ctypes.c_float] + [P] * 5, i32),
        "dopr_shared_attention_4bit": ([P, P, i32, P, P, P, P, ctypes.c_float] + [P] * 5, i32),
        "dopr_shared_attention_workspace": ([P, i32, i32], i64),
        "dopr_last_error": ([], ctypes.c_char_p),
        "dopr_version": ([], ctypes.c_char_p),
    }
    for name, (args, res) in sig.items():
        fn = getattr(L, name)
        fn.argtypes = args
        fn.restype = res
    _LIB = L
    return L


def _check(status: int):
    if status != OK:
        raise DoprError(status, load().dopr_last_error().decode())


def _ptr(x):
    """Pointer of a torch tensor or numpy array (None passes NULL)."""
    if x is None:
        return None
    if isinstance(x, torch.Tensor):
        return ctypes.c_void_p(x.data_ptr())
    return x.ctypes.data_as(ctypes.c_void_p)


def _host(a, dtype):
    if isinstance(a, torch.Tensor):
        a = a.cpu().numpy()
    return np.ascontiguousarray(np.asarray(a, dtype=dtype))


def make_config(shape, max_position: int = 8192) -> ModelConfig:
    """ModelConfig from any object with the synth.ModelShape fields."""
    c = ModelConfig()
    c.n_layers, c.hidden, c.n_q_heads, c.n_kv_heads = shape.n_layers, shape.hidden, shape.n_q_heads, shape.n_kv_heads
    c.head_dim, c.ffn, c.vocab = shape.head_dim, shape.ffn, shape.vocab
    c.score_token_id = shape.score_token_id
    c.max_position = max_position
    c.rope_theta, c.rms_eps = shape.rope_theta, shape.rms_eps
    return c


def prefix_bytes(cfg: ModelConfig, m: int) -> int:
    return int(load().dopr_prefix_bytes(ctypes.byref(cfg), int(m)))


def version() -> str:
    return load().dopr_version().decode()


_PER_LAYER = [("attn_norm", W_ATTN_NORM), ("wq", W_Q), ("wk", W_K), ("wv", W_V), ("q_norm", W_Q_NORM),
              ("k_norm", W_K_NORM), ("wo", W_O), ("mlp_norm", W_MLP_NORM), ("w_gate", W_GATE), ("w_up", W_UP),
              ("w_down", W_DOWN)]


class Model:
    """A decoder on the GPU.  ``weights`` follows synth.make_weights (bf16
    torch tensors on the host or the current CUDA device)."""

    def __init__(self, cfg: ModelConfig, weights: dict | None = None):
        self.cfg = cfg
        self._h = ctypes.c_void_p()
        _check(load().dopr_model_create(ctypes.byref(cfg), ctypes.byref(self._h)))
        if weights is not None:
            self.put_weights(weights)

    def put(self, kind: int, layer: int, t: torch.Tensor):
        assert t.dtype == torch.bfloat16
        t = t.contiguous()
        _check(load().dopr_model_put_weight(self._h, kind, layer, _ptr(t), t.numel(), int(t.is_cuda)))

    def put_weights(self, w: dict):
        self.put(W_EMBED, 0, w["embed"])
        self.put(W_FINAL_NORM, 0, w["final_norm"])
        self.put(W_SCORE_HEAD, 0, w["score_head"])
        for name, kind in _PER_LAYER:
            for l, t in enumerate(w[name]):
                self.put(kind, l, t)

    def close(self):
        if self._h:
            load().dopr_model_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Store:
    """Device prefix store for doc ids 0..max_doc_id in a pool of pool_bytes."""

    def __init__(self, cfg: ModelConfig, max_doc_id: int, pool_bytes: int):
        self.cfg = cfg
        self._h = ctypes.c_void_p()
        # the library places the store on the calling thread's current device
        self.device = torch.cuda.current_device() if torch.cuda.is_available() else 0
        _check(load().dopr_store_create(ctypes.byref(cfg), int(max_doc_id), int(pool_bytes), ctypes.byref(self._h)))

    def put_layer(self, doc_id: int, layer: int, k: torch.Tensor, v: torch.Tensor):
        """k, v: bf16 [m, n_kv_heads, 128] for one layer."""
        assert k.dtype == torch.bfloat16 and v.dtype == torch.bfloat16 and k.shape == v.shape
        k, v = k.contiguous(), v.contiguous()
        _check(load().dopr_store_put(self._h, int(doc_id), int(k.shape[0]), int(layer), _ptr(k), _ptr(v),
                                     int(k.is_cuda)))

    def put(self, doc_id: int, k: torch.Tensor, v: torch.Tensor):
        """k, v: bf16 [n_layers, m, n_kv_heads, 128]."""
        for l in range(k.shape[0]):
            self.put_layer(doc_id, l, k[l], v[l])

    def read_layer(self, doc_id: int, layer: int, m: int):
        """The stored (fp16) K and V of one layer as float16 [m, n_kv_heads, 128] numpy arrays."""
        shape = (m, self.cfg.n_kv_heads, self.cfg.head_dim)
        k, v = np.zeros(shape, np.float16), np.zeros(shape, np.float16)
        _check(load().dopr_debug_store_read(self._h, int(doc_id), int(layer), k.ctypes.data, v.ctypes.data))
        return k, v

    def close(self):
        if self._h:
            load().dopr_store_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def set_mlp_head(model: Model, head: dict | None):
    """Use the MLP scoring head {w1 bf16 [d, H], b1 bf16 [d], w2 bf16 [d], b2 float,
    act 0..3} instead of the yes/no rows; None restores the rows."""
    if head is None:
        _check(load().dopr_model_set_mlp_head(model._h, 0, 0, None, None, None, 0.0, 0))
        return
    w1, b1, w2 = (head[k].contiguous() for k in ("w1", "b1", "w2"))
    assert w1.dtype == b1.dtype == w2.dtype == torch.bfloat16
    _check(load().dopr_model_set_mlp_head(model._h, int(w1.shape[0]), int(head["act"]), _ptr(w1), _ptr(b1), _ptr(w2),
                                          float(head["b2"]), int(w1.is_cuda)))


def build_prefixes(model: Model, store: Store, doc_ids, x_offsets, x: torch.Tensor, stream=None):
    """Offline prefix construction: forward each document's representations
    x[x_offsets[d]:x_offsets[d+1]] (bf16 [rows, hidden], on the GPU or the host)
    and store every layer's keys and values for doc_ids[d]."""
    di, xo = _host(doc_ids, np.int64), _host(x_offsets, np.int32)
    assert x.dtype == torch.bfloat16 and x.dim() == 2
    x = x.contiguous()
    st = ctypes.c_void_p(stream.cuda_stream if stream is not None else
                         (torch.cuda.current_stream().cuda_stream if x.is_cuda else 0))
    _check(load().dopr_build_prefixes(model._h, store._h, len(di), di.ctypes.data, xo.ctypes.data, _ptr(x),
                                      int(x.is_cuda), st))


def select_prefix_inputs(model: Model, doc_offsets, doc_tokens, top_k: int, top_p: int, stream=None):
    """Attention-based key token selection: (positions int32 [n_docs, top_k]
    ascending with -1 padding, states bf16 [n_docs, top_k, hidden], salience
    float32 [tokens])."""
    off, tok = _host(doc_offsets, np.int32), _host(doc_tokens, np.int32)
    n = len(off) - 1
    H = model.cfg.hidden
    pos = np.full((max(n, 1), top_k), -1, np.int32)
    x = torch.zeros((max(n, 1), top_k, H), dtype=torch.bfloat16)
    u = np.zeros(max(int(off[-1]) if n > 0 else 0, 1), np.float32)
    st = ctypes.c_void_p(stream.cuda_stream if stream is not None else torch.cuda.current_stream().cuda_stream)
    _check(load().dopr_select_prefix_inputs(model._h, n, off.ctypes.data, tok.ctypes.data, int(top_k), int(top_p),
                                            pos.ctypes.data, _ptr(x), u.ctypes.data, st))
    return pos[:n], x[:n], u[:int(off[-1]) if n > 0 else 0]


def score(model: Model, store: Store, q_offsets, q_tokens, doc_ids, out=None, stream=None) -> torch.Tensor:
    """Score pairs.  CUDA tensors in -> scored in place on the device
    (io_on_device=1); anything else -> host arrays copied by the library."""
    n = len(q_offsets) - 1
    st = ctypes.c_void_p(stream.cuda_stream if stream is not None else torch.cuda.current_stream().cuda_stream)
    if isinstance(q_offsets, torch.Tensor) and q_offsets.is_cuda:
        assert q_offsets.dtype == torch.int32 and q_tokens.dtype == torch.int32 and doc_ids.dtype == torch.int64
        if out is None:
            out = torch.empty(n, dtype=torch.float32, device=q_offsets.device)
        _check(load().dopr_score(model._h, store._h, n, _ptr(q_offsets), _ptr(q_tokens), _ptr(doc_ids), _ptr(out),
                                 st, 1))
        return out
    qo, qt, di = _host(q_offsets, np.int32), _host(q_tokens, np.int32), _host(doc_ids, np.int64)
    if out is None:
        out = torch.empty(n, dtype=torch.float32)
    assert out.device.type == "cpu" and out.dtype == torch.float32
    _check(load().dopr_score(model._h, store._h, n, _ptr(qo), _ptr(qt) if qt.size else None, _ptr(di), _ptr(out),
                             st, 0))
    return out


def pack_plan(model: Model, store: Store, q_offsets, q_tokens, doc_ids) -> dict:
    qo, qt, di = _host(q_offsets, np.int32), _host(q_tokens, np.int32), _host(doc_ids, np.int64)
    n = len(qo) - 1
    T = int(qo[-1] - qo[0]) + n if n > 0 else 0
    perm = np.zeros(max(n, 1), np.int32)
    tok_off = np.zeros(n + 1, np.int32)
    tok_pos = np.zeros(max(T, 1), np.int32)
    tok_id = np.zeros(max(T, 1), np.int32)
    tok_pair = np.zeros(max(T, 1), np.int32)
    _check(load().dopr_debug_pack_plan(model._h, store._h, n, _ptr(qo), _ptr(qt) if qt.size else None, _ptr(di),
                                       _ptr(perm), _ptr(tok_off), _ptr(tok_pos), _ptr(tok_id), _ptr(tok_pair)))
    return {"perm": perm[:n], "tok_off": tok_off, "tok_pos": tok_pos[:T], "tok_id": tok_id[:T],
            "tok_pair": tok_pair[:T]}


def attention_plan(m: int, rows_per_tile: int, tok_len) -> np.ndarray:
    """The attention tiles of one document's run of pairs (host-only, no GPU):
    int32 [n_tiles, 24] rows {kind, tok_begin, n_tok, n_keys, n_seg, 0, 0, 0, seg[16]}."""
    tl = _host(tok_len, np.int32)
    cap = int(tl.sum()) + 1
    out = np.zeros((cap, 24), np.int32)
    n = load().dopr_debug_attention_plan(int(m), int(rows_per_tile), len(tl), _ptr(tl), cap, _ptr(out))
    if n < 0:
        _check(-n)
    return out[:n]


def gemm(A: torch.Tensor, B: torch.Tensor, epilogue: int = EPI_STORE, out: torch.Tensor | None = None):
    """The projection kernel alone: A [M,K] fp16, B [N,K] fp16 (CUDA)."""
    assert A.dtype == torch.float16 and B.dtype == torch.float16 and A.is_contiguous() and B.is_contiguous()
    M, K = A.shape
    N = B.shape[0]
    if out is None:
        if epilogue == EPI_RESID_ADD:
            out = torch.zeros(M, N, dtype=torch.float32, device=A.device)
        elif epilogue == EPI_SWIGLU:
            out = torch.empty(M, N // 2, dtype=torch.float16, device=A.device)
        else:
            out = torch.empty(M, N, dtype=torch.float16, device=A.device)
    st = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    _check(load().dopr_debug_gemm(M, N, K, _ptr(A), _ptr(B), _ptr(out), epilogue, st))
    return out


def gemm_plan(epilogue: int, M: int, N: int, K: int, num_sms: int = 152) -> dict:
    """The tiles a projection of M rows takes (host-only, no GPU): few (narrow tiles take every row), rows per CTA and
    cols of the narrow tile, wide_rows (rows in wide tiles when the others go to a narrow launch beside them, else 0)."""
    out = (ctypes.c_int32 * 4)()
    _check(load().dopr_debug_gemm_plan(int(epilogue), int(M), int(N), int(K), int(num_sms), out))
    return {"few": bool(out[0]), "rows": out[1], "cols": out[2], "wide_rows": out[3]}


def pack_order_noalloc(store: Store, q_offsets: torch.Tensor, doc_ids: torch.Tensor, perm: torch.Tensor,
                       tok_off: torch.Tensor, stream=None):
    """The allocation-free packer ordering step (device tensors in and out)."""
    assert q_offsets.is_cuda and doc_ids.is_cuda and perm.is_cuda and tok_off.is_cuda
    assert q_offsets.dtype == torch.int32 and doc_ids.dtype == torch.int64
    assert perm.dtype == torch.int32 and tok_off.dtype == torch.int32
    n = q_offsets.numel() - 1
    # the C ABI takes no buffer sizes: every extent the packer kernels index is checked here
    if n < 0 or doc_ids.numel() < n or perm.numel() < n or tok_off.numel() < n + 1:
        raise ValueError(f"pack_order_noalloc: buffers too short for {n} pairs (doc_ids {doc_ids.numel()}, "
                         f"perm {perm.numel()}, tok_off {tok_off.numel()}; need {n}, {n}, {n + 1})")
    for name, t in (("q_offsets", q_offsets), ("doc_ids", doc_ids), ("perm", perm), ("tok_off", tok_off)):
        if not t.is_contiguous() or t.device.index != store.device:
            raise ValueError(f"pack_order_noalloc: {name} must be contiguous on cuda:{store.device}")
    st = ctypes.c_void_p(stream.cuda_stream if stream is not None else torch.cuda.current_stream().cuda_stream)
    _check(load().dopr_pack_order_noalloc(store._h, n, _ptr(q_offsets), _ptr(doc_ids), _ptr(perm), _ptr(tok_off),
                                          st))


# ------------------------------------------------------------------ paged prefix cache
# Every call below runs on the tensors' device, on `stream` (default: that device's current stream), and returns once
# its work is queued.  `status`: an int32 tensor of one element that keeps the first device error (a status number); without
# it device errors go unnoticed.  Rows that a call leaves as they were (a position that is negative or beyond the table, places
# behind the last token) are undefined in outputs that the binding allocates.

class CacheLayout(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_blocks", "page", "n_kv_heads", "head_dim", "dtype", "n_seqs",
                                              "max_blocks")]


class Heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("n_heads", ctypes.c_int32)]


class RopeConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("max_position", "rotary_dim", "layout", "scaling")] + \
               [("theta", ctypes.c_double), ("factor", ctypes.c_double), ("original_max_position", ctypes.c_int32),
                ("low", ctypes.c_double), ("high", ctypes.c_double), ("attention_factor", ctypes.c_double)]


ROPE_HALF, ROPE_INTERLEAVED = 0, 1
ROPE_PLAIN, ROPE_LINEAR, ROPE_NTK, ROPE_BANDS, ROPE_RAMP = range(5)
_DTYPES = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}
_TORCH_TYPES = (torch.float16, torch.bfloat16, torch.float32)
_pack_heads = struct.Struct("@Pqqi4x").pack
assert struct.calcsize("@Pqqi4x") == ctypes.sizeof(Heads)


# Calls of a few microseconds on the device are bound by what is done here: device and stream are asked for as numbers, and
# a device or stream guard is made only where the current one is another.
def _on(device, stream):
    """The device of the call's tensors and the stream made current, where they are not, so that what the call
    allocates belongs to the stream that uses it.  (stream's handle, entered guard or None, device's number)"""
    if device.type != "cuda":
        raise ValueError(f"the paged cache's calls take CUDA tensors, got one on {device}")
    index = device.index
    if stream is not None:
        if stream.device != device:
            raise ValueError(f"the stream is on {stream.device}, the tensors on {device}")
        guard = torch.cuda.stream(stream)
        guard.__enter__()
        return stream.cuda_stream, guard, index
    guard = None
    if torch._C._cuda_getDevice() != index:
        guard = torch.cuda.device(device)
        guard.__enter__()
    return torch._C._cuda_getCurrentRawStream(index), guard, index


def _buf(name, t, dtype, n, device):
    """Pointer of a contiguous tensor of at least n elements on the numbered device; None passes NULL."""
    if t is None:
        return None
    if t.dtype != dtype or t.get_device() != device or not t.is_contiguous() or t.numel() < n:
        raise ValueError(f"{name}: need {n} contiguous {dtype} on cuda:{device}, got {tuple(t.shape)} {t.dtype} on {t.device}")
    return t.data_ptr()


def _no_grad(name, t):
    """The calls are not recorded for autograd: a tensor whose gradient would be lost is refused."""
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} requires a gradient, which this call does not record: use torch.no_grad() (the gradient of a "
                         "rotation is rope_apply with inverse=True)")


def _heads(name, t, tokens, head_dim, dtype, device):
    """A [tokens, heads, head_dim] tensor as the C ABI's view (strided, the last dimension contiguous): the bytes of a
    Heads, which a call takes faster than the structure."""
    if t is None:
        return None
    shape, strides = t.shape, t.stride()
    if tokens > 0x7fffffff:
        raise ValueError(f"{name}: {tokens} tokens, a call takes at most 2^31 - 1")
    _no_grad(name, t)
    if len(shape) != 3 or shape[0] < tokens or shape[2] != head_dim or t.dtype != dtype or t.get_device() != device or \
            (head_dim > 1 and strides[2] != 1):
        raise ValueError(f"{name}: need [{tokens}, heads, {head_dim}] {dtype} on cuda:{device} with a contiguous last "
                         f"dimension, got {tuple(shape)} {t.dtype} on {t.device}, strides {strides}")
    return _pack_heads(t.data_ptr(), strides[0], strides[1], shape[1])


def _sized(fn, layout, *sizes):
    """Bytes that a call with this layout and these sizes needs."""
    n = fn(ctypes.byref(layout), *sizes)
    if n < 0:
        raise DoprError(ERR_INVALID_ARG, load().dopr_last_error().decode())
    return n


def make_cache_layout(n_blocks: int, page: int, n_kv_heads: int, head_dim: int, dtype: torch.dtype, n_seqs: int,
                      max_blocks: int) -> CacheLayout:
    """Pools of one layer's keys and values [n_blocks, n_kv_heads, page, head_dim] and tables [n_seqs, max_blocks]."""
    return CacheLayout(n_blocks, page, n_kv_heads, head_dim, _DTYPES[dtype], n_seqs, max_blocks)


class CacheBatch:
    """A step's new tokens: tok_off [n_seqs + 1], slots and positions [max_tokens], seq_lens [n_seqs] and n_free [1]
    after the step.  For a cache that is updated in place set seq_lens and n_free to the cache's own tensors."""

    def __init__(self, layout: CacheLayout, max_tokens: int, device):
        i32 = dict(dtype=torch.int32, device=device)
        if max_tokens > 0x7fffffff:
            raise ValueError(f"{max_tokens} tokens, a step takes at most 2^31 - 1")
        self.max_tokens = max_tokens
        self.tok_off = torch.empty(layout.n_seqs + 1, **i32)
        self.slots = torch.empty(max_tokens, dtype=torch.int64, device=device)
        self.positions = torch.empty(max_tokens, **i32)
        self.seq_lens = torch.empty(layout.n_seqs, **i32)
        self.n_free = torch.empty(1, **i32)
        self.n_seqs, self.workspace_bytes = layout.n_seqs, _sized(load().dopr_cache_extend_workspace, layout)
        self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=device)


def cache_batch(layout: CacheLayout, max_tokens: int, device="cuda") -> CacheBatch:
    return CacheBatch(layout, max_tokens, device)


def cache_extend(layout: CacheLayout, seq_lens, block_tables, free_blocks, n_free, new_lens, max_tokens: int, prefix=None,
                 out: CacheBatch | None = None, status=None, stream=None) -> CacheBatch:
    """Pages, slots and positions for every row's new tokens (new_lens -1: the row is released), on the device.
    block_tables and free_blocks are updated in place, lengths and the stack's height in `out`."""
    dev = seq_lens.device
    n, i32 = layout.n_seqs, torch.int32
    if max_tokens > 0x7fffffff:
        raise ValueError(f"{max_tokens} tokens, a step takes at most 2^31 - 1")
    st, guard, on = _on(dev, stream)
    try:
        if out is None:
            out = CacheBatch(layout, max_tokens, dev)
        elif out.n_seqs < n:
            raise ValueError(f"out: its workspace is for {out.n_seqs} rows, the layout has {n}")
        _check(load().dopr_cache_extend(
            ctypes.byref(layout), _buf("seq_lens", seq_lens, i32, n, on),
            _buf("block_tables", block_tables, i32, n * layout.max_blocks, on),
            _buf("free_blocks", free_blocks, i32, layout.n_blocks, on), _buf("n_free", n_free, i32, 1, on),
            _buf("prefix", prefix, i32, n, on), _buf("new_lens", new_lens, i32, n, on), max_tokens,
            _buf("out.seq_lens", out.seq_lens, i32, n, on), _buf("out.n_free", out.n_free, i32, 1, on),
            _buf("out.tok_off", out.tok_off, i32, n + 1, on), _buf("out.slots", out.slots, torch.int64, max_tokens, on),
            _buf("out.positions", out.positions, i32, max_tokens, on),
            _buf("out.workspace", out.workspace, torch.uint8, out.workspace_bytes, on), _buf("status", status, i32, 1, on), st))
    finally:
        if guard is not None:
            guard.__exit__(None, None, None)
    return out


class Rope:
    """Rotary positions 0 .. max_position - 1 over the first rotary_dim elements of a head: a table on the current
    device.  scaling and its arguments as in include/dopr.h."""

    def __init__(self, max_position: int, rotary_dim: int, theta: float = 1e6, layout: int = ROPE_HALF,
                 scaling: int = ROPE_PLAIN, factor: float = 1.0, original_max_position: int = 0, low: float = 1.0,
                 high: float = 32.0, attention_factor: float = 0.0):
        self.cfg = RopeConfig(max_position, rotary_dim, layout, scaling, theta, factor, original_max_position, low, high,
                              attention_factor)
        self._h = ctypes.c_void_p()
        _check(load().dopr_rope_create(ctypes.byref(self.cfg), ctypes.byref(self._h)))

    def handle(self):
        """The table's handle: a closed one's is NULL, which the library takes for no rotation."""
        if not self._h:
            raise ValueError("the rotary table is closed")
        return self._h

    def close(self):
        if self._h:
            load().dopr_rope_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def rope_apply(rope: Rope, positions, q, k=None, q_out=None, k_out=None, inverse: bool = False, status=None, stream=None):
    """Rotary positions on q and, with it, k: [tokens, heads, head_dim] views of float16, bfloat16 or float32.  Returns
    (q_out, k_out); pass q_out=q, k_out=k to work in place.  inverse: the gradient of the rotation, for a backward pass of the
    caller's own (tensors that require a gradient are refused unless gradients are off)."""
    (T, _, D), dt, dev = q.shape, q.dtype, q.device
    if dt not in _DTYPES:
        raise ValueError(f"rope_apply: float16, bfloat16 or float32, got {dt}")
    handle = rope.handle()
    st, guard, on = _on(dev, stream)
    try:
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=dt, device=dev)
        if k is not None and k_out is None:
            k_out = torch.empty(k.shape, dtype=dt, device=dev)
        _check(load().dopr_rope_apply(
            handle, _DTYPES[dt], D, T, _buf("positions", positions, torch.int32, T, on), _heads("q", q, T, D, dt, on),
            _heads("q_out", q_out, T, D, dt, on), _heads("k", k, T, D, dt, on),
            _heads("k_out", k_out if k is not None else None, T, D, dt, on), int(inverse),
            _buf("status", status, torch.int32, 1, on), st))
    finally:
        if guard is not None:
            guard.__exit__(None, None, None)
    return q_out, k_out


def cache_append(layout: CacheLayout, slots, k, v, k_pool, v_pool, rope: Rope | None = None, positions=None, q=None,
                 q_out=None, status=None, stream=None):
    """One layer's new rows k (rotated) and v [tokens, kv heads, head_dim] into the pages at slots; returns rotated q
    where q is given.  Not recorded for autograd."""
    _no_grad("k_pool", k_pool)
    _no_grad("v_pool", v_pool)
    T, D, dt, dev = k.shape[0], layout.head_dim, _TORCH_TYPES[layout.dtype], k.device
    handle = rope.handle() if rope is not None else None
    pool = layout.n_blocks * layout.n_kv_heads * layout.page * D
    st, guard, on = _on(dev, stream)
    try:
        if q is not None and q_out is None:
            q_out = torch.empty(q.shape, dtype=dt, device=dev)
        _check(load().dopr_cache_append(
            ctypes.byref(layout), handle, T,
            _buf("positions", positions, torch.int32, T, on), _buf("slots", slots, torch.int64, T, on),
            _heads("q", q, T, D, dt, on), _heads("q_out", q_out if q is not None else None, T, D, dt, on),
            _heads("k", k, T, D, dt, on), _heads("v", v, T, D, dt, on), _buf("k_pool", k_pool, dt, pool, on),
            _buf("v_pool", v_pool, dt, pool, on), _buf("status", status, torch.int32, 1, on), st))
    finally:
        if guard is not None:
            guard.__exit__(None, None, None)
    return q_out


def shared_attention_plan(layout: CacheLayout, n_q_heads: int, tok_off, seq_lens, prefix, max_tokens: int, plan=None,
                          status=None, stream=None) -> torch.Tensor:
    """How a step's attention is split: made once a step, used by every layer (of this very layout, n_q_heads and max_tokens,
    on this device)."""
    dev = seq_lens.device
    n = layout.n_seqs
    st, guard, on = _on(dev, stream)
    try:
        need = _sized(load().dopr_shared_attention_plan_bytes, layout, n_q_heads, max_tokens)
        if plan is None:
            plan = torch.empty(need, dtype=torch.uint8, device=dev)
        _check(load().dopr_shared_attention_plan(
            ctypes.byref(layout), n_q_heads, max_tokens, _buf("tok_off", tok_off, torch.int32, n + 1, on),
            _buf("seq_lens", seq_lens, torch.int32, n, on), _buf("prefix", prefix, torch.int32, n, on),
            _buf("plan", plan, torch.uint8, need, on), _buf("status", status, torch.int32, 1, on), st))
    finally:
        if guard is not None:
            guard.__exit__(None, None, None)
    return plan


def shared_attention_workspace(layout: CacheLayout, n_q_heads: int, max_tokens: int, device="cuda") -> torch.Tensor:
    with torch.cuda.device(device):
        n = _sized(load().dopr_shared_attention_workspace, layout, n_q_heads, max_tokens)
    return torch.empty(n, dtype=torch.uint8, device=device)


def _attention(fn, layout, plan, q, k_pool, v_pool, pool, pool_type, block_tables, scale, out, lse, workspace, status, stream):
    _no_grad("k_pool", k_pool)
    _no_grad("v_pool", v_pool)
    T, hq, D = q.shape
    dt, dev = _TORCH_TYPES[layout.dtype], q.device
    if scale is None:
        scale = D ** -0.5
    lib = load()
    st, guard, on = _on(dev, stream)
    try:
        if out is None:
            out = torch.empty((T, hq, D), dtype=dt, device=dev)
        need = _sized(lib.dopr_shared_attention_workspace, layout, hq, T)
        if workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        _check(fn(
            ctypes.byref(layout),
            _buf("plan", plan, torch.uint8, _sized(lib.dopr_shared_attention_plan_bytes, layout, hq, T), on), T,
            _heads("q", q, T, layout.head_dim, dt, on), _buf("k_pool", k_pool, pool_type, pool, on),
            _buf("v_pool", v_pool, pool_type, pool, on),
            _buf("block_tables", block_tables, torch.int32, layout.n_seqs * layout.max_blocks, on), scale,
            _heads("out", out, T, layout.head_dim, dt, on), _buf("lse", lse, torch.float32, T * hq, on),
            _buf("workspace", workspace, torch.uint8, need, on), _buf("status", status, torch.int32, 1, on), st))
    finally:
        if guard is not None:
            guard.__exit__(None, None, None)
    return out


def shared_attention(layout: CacheLayout, plan, q, k_pool, v_pool, block_tables, scale: float | None = None, out=None,
                     lse=None, workspace=None, status=None, stream=None) -> torch.Tensor:
    """Attention of q [max_tokens, q heads, head_dim], the plan's tokens, over their rows' prefixes and own keys.  lse:
    float32 [max_tokens, q heads] to fill, or None.  workspace: shared_attention_workspace(...), for all layers; without
    it each call allocates one, hundreds of megabytes for thousands of tokens.  Not recorded for autograd: it has no
    backward pass."""
    pool = layout.n_blocks * layout.n_kv_heads * layout.page * layout.head_dim
    return _attention(load().dopr_shared_attention, layout, plan, q, k_pool, v_pool, pool, _TORCH_TYPES[layout.dtype], block_tables,
                      scale, out, lse, workspace, status, stream)


# ------------------------------------------------------------------ norms of heads
def _gains(q_gain, k_gain, head_dim, device):
    """The two gains' pointers and type; each may be None."""
    one = q_gain if q_gain is not None else k_gain
    if one is None:
        return None, None, 0
    if one.dtype not in _DTYPES:
        raise ValueError(f"gains are float16, bfloat16 or float32, got {one.dtype}")
    for name, g in (("q_gain", q_gain), ("k_gain", k_gain)):
        if g is not None:
            _no_grad(name, g)
    return (_buf("q_gain", q_gain, one.dtype, head_dim, device), _buf("k_gain", k_gain, one.dtype, head_dim, device),
            _DTYPES[one.dtype])


def head_norm_rope(q, k=None, q_gain=None, k_gain=None, eps: float = 1e-6, rope: Rope | None = None, positions=None, q_out=None,
                   k_out=None, status=None, stream=None):
    """RMSNorm over each head of q and, with it, k ([tokens, heads, head_dim] views of float16, bfloat16 or float32), times a
    gain [head_dim] each, then rotary positions.  Returns (q_out, k_out); pass q_out=q, k_out=k to work in place.  Its gradients:
    head_norm_rope_backward, for a backward pass of the caller's own."""
    (T, _, D), dt, dev = q.shape, q.dtype, q.device
    if dt not in _DTYPES:
        raise ValueError(f"head_norm_rope: float16, bfloat16 or float32, got {dt}")
    handle = rope.handle() if rope is not None else None
    st, guard, on = _on(dev, stream)
    try:
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=dt, device=dev)
        if k is not None and k_out is None:
            k_out = torch.empty(k.shape, dtype=dt, device=dev)
        qg, kg, gain_dtype = _gains(q_gain, k_gain, D, on)
        _check(load().dopr_head_norm_rope(
            handle, _DTYPES[dt], D, T, _buf("positions", positions, torch.int32, T, on), eps, gain_dtype,
            _heads("q", q, T, D, dt, on), qg, _heads("q_out", q_out, T, D, dt, on), _heads("k", k, T, D, dt, on), kg,
            _heads("k_out", k_out if k is not None else None, T, D, dt, on), _buf("status", status, torch.int32, 1, on), st))
    finally:
        if guard is not None:
            guard.__exit__(None, None, None)
    return q_out, k_out


def head_norm_rope_workspace(head_dim: int, device="cuda") -> torch.Tensor:
    n = load().dopr_head_norm_rope_workspace(head_dim)
    if n < 0:
        raise DoprError(ERR_UNSUPPORTED, load().dopr_last_error().decode())
    return torch.empty(n, dtype=torch.uint8, device=device)


def head_norm_rope_backward(dq_out, q, dk_out=None, k=None, q_gain=None, k_gain=None, eps: float = 1e-6, rope: Rope | None = None,
                            positions=None, dq=None, dk=None, dq_gain=None, dk_gain=None, workspace=None, status=None, stream=None):
    """Gradients of head_norm_rope, from those of its outputs and its inputs: (dq, dk, dq_gain, dk_gain).  dq and dk may be dq_out
    and dk_out themselves.  Gains' gradients are float32 [head_dim], of the gains that are given.  workspace:
    head_norm_rope_workspace(head_dim); without it each call allocates one."""
    (T, _, D), dt, dev = q.shape, q.dtype, q.device
    if dt not in _DTYPES:
        raise ValueError(f"head_norm_rope_backward: float16, bfloat16 or float32, got {dt}")
    handle = rope.handle() if rope is not None else None
    st, guard, on = _on(dev, stream)
    try:
        if dq is None:
            dq = torch.empty(q.shape, dtype=dt, device=dev)
        if k is not None and dk is None:
            dk = torch.empty(k.shape, dtype=dt, device=dev)
        if q_gain is not None and dq_gain is None:
            dq_gain = torch.empty(D, dtype=torch.float32, device=dev)
        if k_gain is not None and dk_gain is None:
            dk_gain = torch.empty(D, dtype=torch.float32, device=dev)
        need = max(0, load().dopr_head_norm_rope_workspace(D))
        if workspace is None and (dq_gain is not None or dk_gain is not None):
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        qg, kg, gain_dtype = _gains(q_gain, k_gain, D, on)
        _check(load().dopr_head_norm_rope_backward(
            handle, _DTYPES[dt], D, T, _buf("positions", positions, torch.int32, T, on), eps, gain_dtype,
            _heads("dq_out", dq_out, T, D, dt, on), _heads("q", q, T, D, dt, on), qg, _heads("dq", dq, T, D, dt, on),
            _buf("dq_gain", dq_gain, torch.float32, D, on), _heads("dk_out", dk_out, T, D, dt, on), _heads("k", k, T, D, dt, on),
            kg, _heads("dk", dk if k is not None else None, T, D, dt, on), _buf("dk_gain", dk_gain, torch.float32, D, on),
            _buf("workspace", workspace, torch.uint8, need, on), _buf("status", status, torch.int32, 1, on), st))
    finally:
        if guard is not None:
            guard.__exit__(None, None, None)
    return dq, dk, dq_gain, dk_gain


# ------------------------------------------------------------------ the paged cache in 4 bits
# Layouts, tables, slots and plans are those of the cache above; the layout's dtype is that of the rows.

def cache_pools_4bit(layout: CacheLayout, device="cuda"):
    """One layer's pools of keys and values in 4 bits, cleared: uint8 [n_blocks, n_kv_heads, bytes of a page]."""
    n = _sized(load().dopr_cache_4bit_pool_bytes, layout)
    shape = (layout.n_blocks, layout.n_kv_heads, n // (layout.n_blocks * layout.n_kv_heads))
    return torch.zeros(shape, dtype=torch.uint8, device=device), torch.zeros(shape, dtype=torch.uint8, device=device)


def cache_append_4bit(layout: CacheLayout, slots, k, v, k_pool, v_pool, k_gain=None, eps: float = 0.0, rope: Rope | None = None,
                      positions=None, q=None, q_gain=None, q_out=None, status=None, stream=None):
    """One layer's new rows k and v [tokens, kv heads, head_dim] into the 4-bit pages at slots; k, and q where it is given,
    are normed first where eps > 0 and turned where there is a rope.  Returns q_out.  status, an int32 of the device, is what tells of
    rows that could not be held.  Not recorded for autograd."""
    T, D, dt, dev = k.shape[0], layout.head_dim, _TORCH_TYPES[layout.dtype], k.device
    handle = rope.handle() if rope is not None else None
    pool = _sized(load().dopr_cache_4bit_pool_bytes, layout)
    st, guard, on = _on(dev, stream)
    try:
        if q is not None and q_out is None:
            q_out = torch.empty(q.shape, dtype=dt, device=dev)
        qg, kg, gain_dtype = _gains(q_gain, k_gain, D, on)
        _check(load().dopr_cache_append_4bit(
            ctypes.byref(layout), handle, T, _buf("positions", positions, torch.int32, T, on),
            _buf("slots", slots, torch.int64, T, on), eps, gain_dtype, _heads("q", q, T, D, dt, on), qg,
            _heads("q_out", q_out if q is not None else None, T, D, dt, on), _heads("k", k, T, D, dt, on), kg,
            _heads("v", v, T, D, dt, on), _buf("k_pool", k_pool, torch.uint8, pool, on),
            _buf("v_pool", v_pool, torch.uint8, pool, on), _buf("status", status, torch.int32, 1, on), st))
    finally:
        if guard is not None:
            guard.__exit__(None, None, None)
    return q_out


def cache_read_4bit(layout: CacheLayout, slots, k_pool, v_pool, k_out=None, v_out=None, status=None, stream=None):
    """What the 4-bit pages hold at slots: (k_out, v_out) [rows, kv heads, head_dim] of the layout's type; NaN where a group could not
    be held."""
    T, D, dt, dev = slots.numel(), layout.head_dim, _TORCH_TYPES[layout.dtype], slots.device
    pool = _sized(load().dopr_cache_4bit_pool_bytes, layout)
    st, guard, on = _on(dev, stream)
    try:
        if k_out is None:
            k_out = torch.empty((T, layout.n_kv_heads, D), dtype=dt, device=dev)
        if v_out is None:
            v_out = torch.empty((T, layout.n_kv_heads, D), dtype=dt, device=dev)
        _check(load().dopr_cache_read_4bit(
            ctypes.byref(layout), T, _buf("slots", slots, torch.int64, T, on), _buf("k_pool", k_pool, torch.uint8, pool, on),
            _buf("v_pool", v_pool, torch.uint8, pool, on), _heads("k_out", k_out, T, D, dt, on), _heads("v_out", v_out, T, D, dt, on),
            _buf("status", status, torch.int32, 1, on), st))
    finally:
        if guard is not None:
            guard.__exit__(None, None, None)
    return k_out, v_out


def shared_attention_4bit(layout: CacheLayout, plan, q, k_pool, v_pool, block_tables, scale: float | None = None, out=None, lse=None,
                          workspace=None, status=None, stream=None) -> torch.Tensor:
    """shared_attention over 4-bit pools: the same plan and workspace, q and out of the layout's type.  Groups that could not be held
    count as zeros, so a program that may have stored some passes status (ERR_RANGE).  Not recorded for autograd."""
    pool = _sized(load().dopr_cache_4bit_pool_bytes, layout)
    return _attention(load().dopr_shared_attention_4bit, layout, plan, q, k_pool, v_pool, pool, torch.uint8, block_tables, scale, out,
                      lse, workspace, status, stream)


def profile_enable(model: Model, on: bool = True):
    """Clear the per-kernel counters; time each launch with CUDA events while on."""
    _check(load().dopr_profile_enable(model._h, int(bool(on))))


def profile_read(model: Model) -> dict:
    """{family: {launches, time_ms, flops, bytes}} accumulated since profile_enable."""
    buf = (KernelStat * 32)()
    n = load().dopr_profile_read(model._h, buf, 32)
    return {buf[i].name.decode(): {"launches": int(buf[i].launches), "time_ms": float(buf[i].time_ms),
                                   "flops": float(buf[i].flops), "bytes": float(buf[i].bytes)} for i in range(n)}


def wait_timeout_probe(timeout_ms: int) -> int:
    """Returns the status of the bounded-wait probe (TIMEOUT expected)."""
    return int(load().dopr_debug_wait_timeout(int(timeout_ms)))
