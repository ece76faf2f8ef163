"""ESTP feature extraction on GB300: Python binding of the C ABI in include/estp.h.

This module only marshals arguments: every step of the path runs in the CUDA
kernels of ``libestp.so`` (built in-tree by ``build.py``).  Importing it without
the built library raises ImportError; there is no CPU fallback.

The raw ctypes functions carry the C names (``lib.estp_token_entropy`` ...); the
``Context`` methods wrap them for torch CUDA tensors:

    ctx = Context(device=0)
    H   = ctx.token_entropy(logits)                       # Eq. 2-1
    lse = ctx.attn_lse(Q, K, cu_seqlens, max_seqlen)      # row normalisers of A
    ctx.attn_importance(Q, K, cu_seqlens, max_seqlen, lse=None, accumulate=False)
    S   = ctx.attn_importance_finalize(n_layers)          # Eq. 2-0
    pooled, y = ctx.pool(hidden, H, S, cu_seqlens, mix, head)   # Eqs. 2-2..2-4, 3-2
"""
from __future__ import annotations

import ctypes
import math
import os
from dataclasses import dataclass

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_build", "libestp.so")
# the same library built with -DESTP_CHECKS (device bounds checks), for tests and debugging
CHECKS_LIB_PATH = os.path.join(_HERE, "_build_checks", "libestp_checks.so")

ESTP_OK, ESTP_ERR_INVALID_ARG, ESTP_ERR_UNSUPPORTED = 0, 1, 2
ESTP_ERR_CUDA, ESTP_ERR_TIMEOUT, ESTP_ERR_WORKSPACE = 3, 4, 5
ESTP_ERR_BOUNDS = 6
ESTP_F32, ESTP_BF16 = 0, 1
ESTP_IMP_EXCLUDE_SELF = 1
ESTP_IMP_DIV_CAUSAL = 2
ESTP_IMP_DIV_NONE = 4
_DIVISOR_FLAGS = {"length": 0, "causal": ESTP_IMP_DIV_CAUSAL, "none": ESTP_IMP_DIV_NONE}

# every entry point declared in include/estp.h
EXPORTS = ("estp_create", "estp_destroy", "estp_last_error", "estp_sync_status",
           "estp_token_entropy", "estp_attn_lse", "estp_attn_importance",
           "estp_attn_importance_finalize", "estp_pool", "estp_token_entropy_noalloc",
           "estp_head_loss", "estp_misalignment", "estp_lm_head_entropy",
           "estp_mlp_head_predict", "estp_mlp_head_loss", "estp_attn_forward_importance",
           "estp_set_wait_limit", "estp_cache_append", "estp_cache_attention",
           "estp_cache_evict", "estp_token_logprobs", "estp_token_logprobs_grad", "estp_distill_loss")


class EstpError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"estp status {status}: {msg}")
        self.status = status


class MixParams(ctypes.Structure):
    """estp_mix_params: T_i = lambda1 S_i + lambda2 H_i, e = softmax(T / alpha)."""
    _fields_ = [("lambda1", ctypes.c_float), ("lambda2", ctypes.c_float),
                ("alpha", ctypes.c_float)]


class _Head(ctypes.Structure):
    _fields_ = [("W", ctypes.c_void_p), ("bias", ctypes.c_void_p),
                ("centers", ctypes.c_void_p), ("K", ctypes.c_int32)]


class _MlpHead(ctypes.Structure):
    _fields_ = [("W1", ctypes.c_void_p), ("b1", ctypes.c_void_p), ("W2", ctypes.c_void_p),
                ("b2", ctypes.c_void_p), ("centers", ctypes.c_void_p), ("F", ctypes.c_int32),
                ("K", ctypes.c_int32)]


class _MlpGrads(ctypes.Structure):
    _fields_ = [("W1", ctypes.c_void_p), ("b1", ctypes.c_void_p), ("W2", ctypes.c_void_p),
                ("b2", ctypes.c_void_p), ("pooled", ctypes.c_void_p)]


class _KVCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("weight", ctypes.c_void_p),
                ("position", ctypes.c_void_p), ("page_table", ctypes.c_void_p),
                ("page_stride", ctypes.c_int64), ("slot_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64), ("n_pages", ctypes.c_int64),
                ("max_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("Hkv", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int)]


def load_library(path: str = LIB_PATH):
    """ctypes handle of a build of the C ABI with every entry point's signature set:
    libestp.so by default, or CHECKS_LIB_PATH for the bounds-checked build."""
    if not os.path.exists(path):
        raise ImportError(f"ESTP CUDA library not built ({path} missing): run "
                          "paper_2608_15592_gb300/build.py or __graft_entry__.build()")
    lib = ctypes.CDLL(path)
    P, I32, I64, F, U32 = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float,
                           ctypes.c_uint32)
    sigs = {
        "estp_create": ([ctypes.POINTER(ctypes.c_void_p), ctypes.c_int], ctypes.c_int),
        "estp_destroy": ([P], None),
        "estp_last_error": ([P], ctypes.c_char_p),
        "estp_sync_status": ([P, P], ctypes.c_int),
        "estp_set_wait_limit": ([P, I64], ctypes.c_int),
        "estp_token_entropy": ([P, P, ctypes.c_int, I64, I64, I64, P, I32, P, P], ctypes.c_int),
        "estp_attn_lse": ([P, P, P, ctypes.c_int, I32, I32, I32, F, P, I32, I64, I32, P, P],
                          ctypes.c_int),
        "estp_attn_importance": ([P, P, P, ctypes.c_int, P, I32, I32, I32, F, P, I32, P, I32,
                                  I64, I32, ctypes.c_int, U32, P], ctypes.c_int),
        "estp_attn_importance_finalize": ([P, I32, P, P], ctypes.c_int),
        "estp_attn_forward_importance": ([P, P, P, P, ctypes.c_int, P, I32, I32, I32, F, P, I32,
                                          I64, I32, ctypes.c_int, U32, P, P], ctypes.c_int),
        "estp_token_entropy_noalloc": ([P, ctypes.c_int, I64, I64, I64, P, P], ctypes.c_int),
        "estp_pool": ([P, P, ctypes.c_int, I64, I64, P, P, P, I32, I64, MixParams,
                       ctypes.POINTER(_Head), P, P, P], ctypes.c_int),
        "estp_head_loss": ([P, P, I32, I64, ctypes.POINTER(_Head), P, F, P, P, P, P, P],
                           ctypes.c_int),
        "estp_misalignment": ([P, P, P, P, I32, I64, I32, P, P], ctypes.c_int),
        "estp_mlp_head_predict": ([P, P, I32, I64, ctypes.POINTER(_MlpHead), P, P, P],
                                  ctypes.c_int),
        "estp_mlp_head_loss": ([P, P, I32, I64, ctypes.POINTER(_MlpHead), P, F, P,
                                ctypes.POINTER(_MlpGrads), P], ctypes.c_int),
        "estp_lm_head_entropy": ([P, P, I64, P, I64, ctypes.c_int, I64, I64, I64, P, P],
                                 ctypes.c_int),
        "estp_cache_append": ([P, P, P, P, P, P, I32, P, P, I64, I64, P, P, P, I64, P], ctypes.c_int),
        "estp_cache_attention": ([P, P, P, I32, I64, P, I64, I32, P, P, I64, P, I64, I32, F, P, I32, P,
                                  ctypes.c_int, P, P, P, P], ctypes.c_int),
        "estp_cache_evict": ([P, P, P, P, P, I32, I32, I32, I32, P], ctypes.c_int),
        "estp_token_logprobs": ([P, P, ctypes.c_int, I64, I64, I64, P, F, I32, P, P, P, P, P, P], ctypes.c_int),
        "estp_token_logprobs_grad": ([P, P, ctypes.c_int, I64, I64, I64, P, P, P, F, I32, P, P, P, P, P, P, I64, P],
                                     ctypes.c_int),
        "estp_distill_loss": ([P, P, ctypes.c_int, I64, I64, I64, P, P, I32, F, ctypes.c_int, P, P, P, I64, P],
                              ctypes.c_int),
    }
    for name, (args, res) in sigs.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = res
    return lib


lib = load_library()


def _check(status: int):
    if status != ESTP_OK:
        raise EstpError(status, lib.estp_last_error(None).decode())


def _dtype(t) -> int:
    import torch
    if t.dtype == torch.bfloat16:
        return ESTP_BF16
    if t.dtype == torch.float32:
        return ESTP_F32
    raise TypeError(f"tensors are bf16 or fp32, got {t.dtype}")


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


def _stream(stream) -> int | None:
    if stream is not None:
        return stream.cuda_stream or None
    import torch
    if not torch.cuda.is_initialized():
        torch.cuda.init()
    # the handle alone: building the Stream object that wraps it costs 2.9 us a call, this 0.5
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice()) or None


@dataclass
class Head:
    """Linear length head (Eq. 3-2): W [K, D], bias [K] or None, centers [K], fp32 CUDA."""
    W: "object"
    bias: "object"
    centers: "object"


@dataclass
class MlpHead:
    """MLP predictor (Sec. 3.3): u = relu(W1 h + b1), z = W2 u + b2, then Eq. 3-2.
    W1 [F, D], b1 [F] or None, W2 [K, F], b2 [K] or None, centers [K], fp32 CUDA."""
    W1: "object"
    b1: "object"
    W2: "object"
    b2: "object"
    centers: "object"


@dataclass
class TokenLogprobs:
    """What token_logprobs returns: logprob [n] (None without targets), entropy [n], norm [n, 2] (the
    greatest logit and the sum of exponentials against it), top_ids and top_logprobs [n, top_k]
    (None without), and the temperature they belong to."""
    logprob: "object"
    entropy: "object"
    norm: "object"
    top_ids: "object"
    top_logprobs: "object"
    temperature: float = 1.0

    @property
    def lse(self):
        """ln sum_v exp(z_v / temperature) per row, fp32 [n]."""
        return self.norm[:, 0] / self.temperature + self.norm[:, 1].log()


def _like(t, dtype, shape, name):
    """A dense tensor of this type and shape (None passes)."""
    if t is not None and (t.dtype != dtype or t.shape != shape or not t.is_contiguous()):
        raise ValueError(f"{name} is a contiguous {dtype} tensor of shape {shape}")


class KVCache:
    """A paged KV cache of one layer (estp_kv_cache) over tensors that the caller owns.

    k, v       [n_pages, page_size, Hkv, d] bf16 or fp32, in any order of strides (a permuted
               view of head-major pages, for instance), d contiguous
    page_table int32 [B, max_pages];  length, seen: int32 [B], updated in place
    weight     fp32 [n_pages, Hkv, page_size], position: int32 of that shape, or None
    max_slots  a bound of the slots in use over all sequences (default: what the page table can
               hold; with weights, which need every page in one sequence only, at most the pool's).
               The scratch of cache_attention grows with it, that of cache_evict with the table

    Each is an attribute that may be replaced (a longer page table, a larger pool); the call after
    that looks all of them over again, together.
    """

    _TENSORS = frozenset(("k", "v", "page_table", "length", "seen", "weight", "position"))

    def __init__(self, k, v, page_table, length, seen, weight=None, position=None, max_slots=None):
        self.k, self.v, self.page_table, self.length, self.seen = k, v, page_table, length, seen
        self.weight, self.position = weight, position
        self.max_slots = max_slots
        self._struct()

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value)
        if name in self._TENSORS:
            object.__setattr__(self, "_ref", None)

    @property
    def max_slots(self) -> int:
        self._struct()
        return self._bound if self._slots is None else self._slots

    @max_slots.setter
    def max_slots(self, value):
        self._slots = None if value is None else int(value)

    def _struct(self):
        """Address of the estp_kv_cache, formed anew where a tensor was replaced."""
        if self._ref is not None:
            return self._ref
        import torch
        k, v, page_table, weight, position = self.k, self.v, self.page_table, self.weight, self.position
        n_pages, page, Hkv, d = k.shape
        if v.shape != k.shape or v.stride() != k.stride() or v.dtype != k.dtype or (k.numel() and k.stride(3) != 1):
            raise ValueError("k and v share their type, shape and strides, with contiguous rows")
        B, per = page_table.shape
        _like(page_table, torch.int32, (B, per), "page_table")
        _like(self.length, torch.int32, (B,), "length")
        _like(self.seen, torch.int32, (B,), "seen")
        _like(weight, torch.float32, (n_pages, Hkv, page), "weight")
        _like(position, torch.int32, (n_pages, Hkv, page), "position")
        self.B, self._cu_shape = B, (B + 1,)
        self.Hkv, self.head_dim, self.dtype = Hkv, d, k.dtype
        self._bound = B * per * page if weight is None else min(B * per, n_pages) * page
        self._c = _KVCache(_ptr(k), _ptr(v), _ptr(weight), _ptr(position), _ptr(page_table), k.stride(0),
                           k.stride(1), k.stride(2), n_pages, per, page, Hkv, d, _dtype(k))
        self._ref = ctypes.addressof(self._c)
        return self._ref

    def _rows(self, t, heads, name):
        """Row stride of a [rows, heads, d] tensor of the cache's type whose heads are contiguous."""
        if t.dim() != 3:
            raise ValueError(f"{name} is a {self.dtype} tensor [rows, {heads}, {self.head_dim}]")
        rows, h, d = t.shape
        s0, s1, s2 = t.stride()
        if h != heads or d != self.head_dim or t.dtype != self.dtype:
            raise ValueError(f"{name} is a {self.dtype} tensor [rows, {heads}, {self.head_dim}]")
        if rows and (s2 != 1 or (heads > 1 and s1 != d)):
            raise ValueError(f"{name}: a row's heads are contiguous")
        return s0 if rows > 1 else heads * d

    def _new_rows(self, k_new, v_new):
        """The row stride that new rows' K and V share."""
        ld = self._rows(k_new, self.Hkv, "k_new")
        if v_new.shape != k_new.shape or v_new.dtype != k_new.dtype:
            raise ValueError("k_new and v_new share their type and shape")
        # strides of one row or one head are never stepped by and need not agree
        if v_new.stride() != k_new.stride() and self._rows(v_new, self.Hkv, "v_new") != ld:
            raise ValueError("k_new and v_new share their row stride")
        return ld


class Context:
    """One estp_ctx (status word + workspace) on a CUDA device, in `library` (the release
    build by default; load_library(CHECKS_LIB_PATH) for the bounds-checked one)."""

    def __init__(self, device: int = 0, library=None):
        self.device = device
        self._dev = None  # the torch.device, built at its first use
        self._lib = lib if library is None else library
        h = ctypes.c_void_p()
        self._check(self._lib.estp_create(ctypes.byref(h), device))
        self._h = h

    def _torch_device(self):
        if self._dev is None:
            import torch
            self._dev = torch.device("cuda", self.device)
        return self._dev

    def _check(self, status: int):
        if status != ESTP_OK:
            raise EstpError(status, self._lib.estp_last_error(None).decode())

    def close(self):
        if getattr(self, "_h", None):
            self._lib.estp_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def sync_status(self, stream=None):
        """estp_sync_status: synchronise the stream; raise on a device-side error."""
        self._check(self._lib.estp_sync_status(self._h, _stream(stream)))

    def set_wait_limit(self, cycles: int = 0):
        """estp_set_wait_limit: limit (SM cycles) of the attention kernels' abortable
        waits for later calls; 0 restores the default.  A testing aid."""
        self._check(self._lib.estp_set_wait_limit(self._h, int(cycles)))

    # ------------------------------------------------------------------ (a)
    def lm_head_entropy(self, hidden, W, out=None, stream=None):
        """estp_lm_head_entropy: entropy (nats) of softmax(hidden @ W^T) per row, the logits
        formed on the tensor cores and never stored.  hidden: bf16 [rows, D], W: bf16 [V, D]
        (row views of wider arrays allowed: stride(1) == 1)."""
        import torch
        assert hidden.dim() == 2 and W.dim() == 2 and hidden.shape[1] == W.shape[1]
        assert hidden.numel() == 0 or hidden.stride(1) == 1
        assert W.stride(1) == 1
        rows, D = hidden.shape
        V = W.shape[0]
        ldh = hidden.stride(0) if rows > 1 else D
        ldw = W.stride(0) if V > 1 else D
        out = torch.empty(rows, dtype=torch.float32, device=hidden.device) if out is None else out
        self._check(self._lib.estp_lm_head_entropy(self._h, _ptr(hidden), ldh, _ptr(W), ldw, _dtype(hidden),
                                        rows, D, V, _ptr(out), _stream(stream)))
        return out

    def token_entropy(self, logits, V: int | None = None, cu_seqlens=None, out=None,
                      stream=None):
        """estp_token_entropy on a 2-D [rows, ld] tensor (stride(1) == 1)."""
        import torch
        assert logits.dim() == 2 and (logits.numel() == 0 or logits.stride(1) == 1)
        rows, ld = logits.shape[0], logits.stride(0) if logits.shape[0] > 1 else logits.shape[1]
        V = logits.shape[1] if V is None else V
        out = torch.empty(rows, dtype=torch.float32, device=logits.device) if out is None else out
        B = 0 if cu_seqlens is None else cu_seqlens.numel() - 1
        self._check(self._lib.estp_token_entropy(self._h, _ptr(logits), _dtype(logits), rows, V, ld,
                                      _ptr(cu_seqlens), B, _ptr(out), _stream(stream)))
        return out

    # ------------------------------------------------------------------ (b)
    def attn_lse(self, Q, K, cu_seqlens, max_seqlen: int, scale: float | None = None,
                 out=None, stream=None):
        """estp_attn_lse: fp32 [Hq, sumT] row log-normalisers."""
        import torch
        sumT, Hq, d = Q.shape
        Hkv = K.shape[1]
        scale = 1.0 / math.sqrt(d) if scale is None else scale
        out = torch.empty(Hq, sumT, dtype=torch.float32, device=Q.device) if out is None else out
        self._check(self._lib.estp_attn_lse(self._h, _ptr(Q), _ptr(K), _dtype(Q), Hq, Hkv, d, scale,
                                 _ptr(cu_seqlens), cu_seqlens.numel() - 1, sumT, max_seqlen,
                                 _ptr(out), _stream(stream)))
        return out

    def attn_importance(self, Q, K, cu_seqlens, max_seqlen: int, lse=None,
                        scale: float | None = None, heads=None, accumulate: bool = False,
                        exclude_self: bool = False, divisor: str = "length", stream=None):
        """estp_attn_importance for one layer (column sums into the context).
        divisor: "length" (Eq. 2-0's 1/N), "causal" or "none" (ESTP_IMP_DIV_*), applied
        by attn_importance_finalize and fixed by the call that opens the accumulation."""
        sumT, Hq, d = Q.shape
        Hkv = K.shape[1]
        scale = 1.0 / math.sqrt(d) if scale is None else scale
        if heads is None:
            hp, nh = None, Hq
        else:
            arr = (ctypes.c_int32 * len(heads))(*[int(h) for h in heads])
            hp, nh = ctypes.cast(arr, ctypes.c_void_p), len(heads)
        self._check(self._lib.estp_attn_importance(self._h, _ptr(Q), _ptr(K), _dtype(Q), _ptr(lse), Hq,
                                        Hkv, d, scale, hp, nh, _ptr(cu_seqlens),
                                        cu_seqlens.numel() - 1, sumT, max_seqlen,
                                        1 if accumulate else 0,
                                        (ESTP_IMP_EXCLUDE_SELF if exclude_self else 0)
                                        | _DIVISOR_FLAGS[divisor],
                                        _stream(stream)))

    def attn_forward_importance(self, Q, K, V, cu_seqlens, max_seqlen: int, lse=None,
                                scale: float | None = None, accumulate: bool = False,
                                exclude_self: bool = False, divisor: str = "length", out=None,
                                stream=None):
        """estp_attn_forward_importance for one layer: returns the attention output bf16
        [sumT, Hq, 128] and adds the column sums of all Hq heads into the context's
        importance accumulation (same accumulation and flags as attn_importance)."""
        import torch
        sumT, Hq, d = Q.shape
        Hkv = K.shape[1]
        scale = 1.0 / math.sqrt(d) if scale is None else scale
        if out is None:
            out = torch.empty(sumT, Hq, d, dtype=Q.dtype, device=Q.device)
        self._check(self._lib.estp_attn_forward_importance(
            self._h, _ptr(Q), _ptr(K), _ptr(V), _dtype(Q), _ptr(lse), Hq, Hkv, d, scale,
            _ptr(cu_seqlens), cu_seqlens.numel() - 1, sumT, max_seqlen, 1 if accumulate else 0,
            (ESTP_IMP_EXCLUDE_SELF if exclude_self else 0) | _DIVISOR_FLAGS[divisor], _ptr(out),
            _stream(stream)))
        return out

    def attn_importance_finalize(self, n_layers: int, sumT: int, device=None, out=None,
                                 stream=None):
        """estp_attn_importance_finalize: S [sumT] (Eq. 2-0)."""
        import torch
        if out is None:
            out = torch.empty(sumT, dtype=torch.float32,
                              device=device if device is not None else self._torch_device())
        self._check(self._lib.estp_attn_importance_finalize(self._h, n_layers, _ptr(out), _stream(stream)))
        return out

    # ------------------------------------------------------------------ (c)
    def misalignment(self, entropy, importance, cu_seqlens, pct: int = 40, out=None,
                     stream=None):
        """estp_misalignment: int32 [B, 3] = (k, |TopH & BotS|, |BotH & TopS|) per prompt."""
        import torch
        B = cu_seqlens.numel() - 1
        out = torch.empty(B, 3, dtype=torch.int32, device=entropy.device) if out is None else out
        self._check(self._lib.estp_misalignment(self._h, _ptr(entropy), _ptr(importance), _ptr(cu_seqlens),
                                     B, entropy.numel(), pct, _ptr(out), _stream(stream)))
        return out

    def head_loss(self, pooled, head: Head, targets, lambda3: float, grads: bool = True,
                  stream=None):
        """estp_head_loss (Eqs. 3-1 to 3-3): returns (loss [1], and if grads:
        dL/dW [K, D], dL/dbias [K], dL/dpooled [B, D]), fp32 CUDA tensors."""
        import torch
        B, D = pooled.shape
        K = head.W.shape[0]
        dev = pooled.device
        loss = torch.empty(1, dtype=torch.float32, device=dev)
        gW = torch.empty(K, D, dtype=torch.float32, device=dev) if grads else None
        gb = torch.empty(K, dtype=torch.float32, device=dev) if grads else None
        gp = torch.empty(B, D, dtype=torch.float32, device=dev) if grads else None
        hp = ctypes.byref(_Head(_ptr(head.W), _ptr(head.bias), _ptr(head.centers), K))
        self._check(self._lib.estp_head_loss(self._h, _ptr(pooled), B, D, hp, _ptr(targets), lambda3,
                                  _ptr(loss), _ptr(gW), _ptr(gb), _ptr(gp), _stream(stream)))
        return (loss, gW, gb, gp) if grads else loss

    @staticmethod
    def _mlp(head: "MlpHead"):
        return ctypes.byref(_MlpHead(_ptr(head.W1), _ptr(head.b1), _ptr(head.W2), _ptr(head.b2),
                                       _ptr(head.centers), head.W1.shape[0], head.W2.shape[0]))

    def mlp_head_predict(self, pooled, head: "MlpHead", probs: bool = False, stream=None):
        """estp_mlp_head_predict: predicted lengths [B] (and p_hat [B, K] if probs)."""
        import torch
        B, D = pooled.shape
        pred = torch.empty(B, dtype=torch.float32, device=pooled.device)
        p = torch.empty(B, head.W2.shape[0], dtype=torch.float32, device=pooled.device) if probs else None
        self._check(self._lib.estp_mlp_head_predict(self._h, _ptr(pooled), B, D, self._mlp(head), _ptr(pred),
                                         _ptr(p), _stream(stream)))
        return (pred, p) if probs else pred

    def mlp_head_loss(self, pooled, head: "MlpHead", targets, lambda3: float, grads=True,
                      stream=None):
        """estp_mlp_head_loss (Eqs. 3-1, 3-3 through the MLP predictor): returns loss [1]
        and, if grads, (dL/dW1 [F, D], dL/db1 [F], dL/dW2 [K, F], dL/db2 [K], dL/dpooled
        [B, D]).  grads may also be a set of those names to compute only some of them."""
        import torch
        B, D = pooled.shape
        F, K = head.W1.shape[0], head.W2.shape[0]
        dev = pooled.device
        shapes = {"W1": (F, D), "b1": (F,), "W2": (K, F), "b2": (K,), "pooled": (B, D)}
        want = set(shapes) if grads is True else (set(grads) if grads else set())
        out = {k: torch.empty(v, dtype=torch.float32, device=dev) if k in want else None
               for k, v in shapes.items()}
        loss = torch.empty(1, dtype=torch.float32, device=dev)
        gp = ctypes.byref(_MlpGrads(*[_ptr(out[k]) for k in ("W1", "b1", "W2", "b2", "pooled")]))
        self._check(self._lib.estp_mlp_head_loss(self._h, _ptr(pooled), B, D, self._mlp(head), _ptr(targets),
                                      lambda3, _ptr(loss), gp if want else None, _stream(stream)))
        if not grads:
            return loss
        return (loss, *[out[k] for k in ("W1", "b1", "W2", "b2", "pooled")])

    def pool(self, hidden, entropy, importance, cu_seqlens, lambda1: float, lambda2: float,
             alpha: float, head: Head | None = None, D: int | None = None, pooled=None,
             pred=None, stream=None):
        """estp_pool: returns (pooled [B, D], predicted lengths [B] or None)."""
        import torch
        assert hidden.dim() == 2 and (hidden.numel() == 0 or hidden.stride(1) == 1)
        sumT = hidden.shape[0]
        ldh = hidden.stride(0) if sumT > 1 else hidden.shape[1]
        D = hidden.shape[1] if D is None else D
        B = cu_seqlens.numel() - 1
        dev = hidden.device
        pooled = torch.empty(B, D, dtype=torch.float32, device=dev) if pooled is None else pooled
        hp = None
        if head is not None:
            pred = torch.empty(B, dtype=torch.float32, device=dev) if pred is None else pred
            hp = ctypes.byref(_Head(_ptr(head.W), _ptr(head.bias), _ptr(head.centers),
                                      head.W.shape[0]))
        mix = MixParams(lambda1, lambda2, alpha)
        self._check(self._lib.estp_pool(self._h, _ptr(hidden), _dtype(hidden), D, ldh, _ptr(entropy),
                             _ptr(importance), _ptr(cu_seqlens), B, sumT, mix, hp,
                             _ptr(pooled), _ptr(pred) if head is not None else None,
                             _stream(stream)))
        return pooled, (pred if head is not None else None)

    # ------------------------------------------------------------------ (e)
    def cache_append(self, cache: KVCache, k_new, v_new, cu_rows, weight=None, rows=None,
                     fresh: bool = False, stream=None):
        """estp_cache_append: rows of k_new, v_new [n, Hkv, d] enter the cache, cu_rows[b] ..
        cu_rows[b+1]-1 into sequence b; `rows` (int32) picks rows of k_new, `weight` [n, Hkv]
        gives their attention weights so far: of cache_attention, or one layer's importance with
        divisor="none" times Hq / Hkv, which is the same scale.  fresh: the sequences start empty.  cache.length
        and cache.seen are updated in place."""
        import torch
        ref = cache._struct()
        n = k_new.shape[0]
        ld = cache._new_rows(k_new, v_new)
        if weight is not None:
            _like(weight, torch.float32, (n, cache.Hkv), "weight")
        _like(cu_rows, torch.int32, cache._cu_shape, "cu_rows")
        if rows is not None:
            _like(rows, torch.int32, (rows.numel(),), "rows")
        length, seen = cache.length.data_ptr(), cache.seen.data_ptr()
        self._check(self._lib.estp_cache_append(
            self._h, ref, None if fresh else length, None if fresh else seen, length, seen, cache.B,
            k_new.data_ptr(), v_new.data_ptr(), ld, n, _ptr(weight), _ptr(rows), cu_rows.data_ptr(),
            n if rows is None else rows.numel(), _stream(stream)))

    def cache_attention(self, cache: KVCache, Q, k_new, v_new, cu_rows, max_rows: int,
                        scale: float | None = None, tree_mask=None, row_weight=None,
                        accumulate: bool = False, details: bool = False, out=None, stream=None):
        """estp_cache_attention: Q [n, Hq, d] over the cache and the rows' own k_new, v_new
        [n, Hkv, d] (None: the cache alone); returns out [n, Hq, d], with details (out,
        lse [Hq, n], weight_new [n, Hkv] or None).  tree_mask: int64 or uint64 [n, words], bit j
        of a row set where it sees the sequence's j-th row.  accumulate adds the attention the
        slots receive, times row_weight [n], to cache.weight."""
        import torch
        ref = cache._struct()
        n, Hq, d = Q.shape
        ldq = cache._rows(Q, Hq, "Q")
        ld, kp, vp = 0, None, None
        if k_new is not None:
            if k_new.shape[0] != n or v_new.shape[0] != n:
                raise ValueError("k_new and v_new have a row for each of Q's")
            ld, kp, vp = cache._new_rows(k_new, v_new), k_new.data_ptr(), v_new.data_ptr()
        _like(cu_rows, torch.int32, cache._cu_shape, "cu_rows")
        words = 0
        if tree_mask is not None:
            words = tree_mask.shape[-1]
            _like(tree_mask, torch.uint64 if tree_mask.dtype == torch.uint64 else torch.int64, (n, words), "tree_mask")
        if row_weight is not None:
            _like(row_weight, torch.float32, (n,), "row_weight")
        dev = Q.device
        if out is None:
            out = torch.empty((n, Hq, d), dtype=cache.dtype, device=dev)
        else:
            _like(out, cache.dtype, (n, Hq, d), "out")
        lse = w_new = lp = wp = None
        if details:
            lse = torch.empty((Hq, n), dtype=torch.float32, device=dev)
            lp = lse.data_ptr()
            if kp is not None:
                w_new = torch.empty((n, cache.Hkv), dtype=torch.float32, device=dev)
                wp = w_new.data_ptr()
        status = self._lib.estp_cache_attention(
            self._h, ref, cache.length.data_ptr(), cache.B, cache.max_slots, Q.data_ptr(), ldq, Hq, kp, vp, ld,
            cu_rows.data_ptr(), n, max_rows, d ** -0.5 if scale is None else scale, _ptr(tree_mask), words,
            _ptr(row_weight), 1 if accumulate else 0, out.data_ptr(), lp, wp, _stream(stream))
        if status:
            self._check(status)
        return (out, lse, w_new) if details else out

    def cache_evict(self, cache: KVCache, budget: int, recent: int = 0, sinks: int = 0, stream=None):
        """estp_cache_evict: every sequence is cut to at most `budget` slots, each KV head keeping
        its last `recent` and first `sinks` tokens and then those of the greatest weight;
        cache.length is updated in place."""
        ref, length = cache._struct(), cache.length.data_ptr()
        self._check(self._lib.estp_cache_evict(self._h, ref, length, cache.seen.data_ptr(), length, cache.B,
                                               budget, recent, sinks, _stream(stream)))

    # ------------------------------------------------------------------ (f)
    def _logits(self, logits, V):
        """Rows, V and row stride of logits [rows, >= V] whose rows are contiguous."""
        if logits.dim() != 2:
            raise ValueError("logits is a [rows, V] tensor with contiguous rows")
        rows, cols = logits.shape
        s0, s1 = logits.stride()
        if s1 != 1 and rows and cols > 1:
            raise ValueError("logits is a [rows, V] tensor with contiguous rows")
        if logits.get_device() != self.device:
            raise ValueError(f"logits is not on the context's device cuda:{self.device}")
        if V is None:
            V = cols
        elif not 1 <= V <= cols:
            raise ValueError("V is in 1 .. the columns of logits")
        return rows, V, s0 if rows > 1 else cols + -cols % (16 // logits.element_size())

    def _is(self, t, dtype, shape, name):
        """A dense tensor of this type and shape on the context's device."""
        if t.dtype != dtype or t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{name} is a contiguous {dtype} tensor of shape {shape}")
        if t.get_device() != self.device:
            raise ValueError(f"{name} is not on the context's device cuda:{self.device}")
        return t.data_ptr()

    @staticmethod
    def _empty(shape, dtype, device, stream):
        """An output for work on `stream` (None: the current one)."""
        import torch
        if stream is None:
            return torch.empty(shape, dtype=dtype, device=device)
        with torch.cuda.stream(stream):
            return torch.empty(shape, dtype=dtype, device=device)

    def _grad_out(self, logits, rows, V, out, stream):
        """Where the gradient of logits goes, [rows, V]: `out`, or a new tensor whose rows start on 16 bytes."""
        per = 16 // logits.element_size()
        if out is None:
            wide = V + -V % per
            out = self._empty((rows, wide), logits.dtype, logits.device, stream)
            return (out if wide == V else out[:, :V]), wide
        if out.dim() != 2 or out.shape[0] != rows or out.shape[1] < V or out.dtype != logits.dtype or (
                out.numel() and out.stride(1) != 1):
            raise ValueError("out is a [rows, >= V] tensor of the logits' type with contiguous rows")
        if out.get_device() != self.device:
            raise ValueError(f"out is not on the context's device cuda:{self.device}")
        return out, out.stride(0) if rows > 1 else out.shape[1] + -out.shape[1] % per

    def token_logprobs(self, logits, targets=None, top_k: int = 0, temperature: float = 1.0, V: int | None = None,
                       stream=None) -> TokenLogprobs:
        """estp_token_logprobs on logits [rows, >= V]: ln p of `targets` (int32 [rows], negative: none),
        the entropy, what the gradient needs, and the top_k greatest alternatives.  Uses the context's scratch: calls on
        several streams that may overlap are ordered by the caller or take a context each."""
        import torch
        rows, V, ld = self._logits(logits, V)
        f32, dev = torch.float32, logits.device
        lp = ids = tops = tp = lpp = ip = kp = None
        if targets is not None:
            tp = self._is(targets, torch.int32, (rows,), "targets")
            lp = self._empty((rows,), f32, dev, stream)
            lpp = lp.data_ptr()
        entropy, norm = self._empty((rows,), f32, dev, stream), self._empty((rows, 2), f32, dev, stream)
        if top_k > 0:
            ids, tops = self._empty((rows, top_k), torch.int32, dev, stream), self._empty((rows, top_k), f32, dev, stream)
            ip, kp = ids.data_ptr(), tops.data_ptr()
        status = self._lib.estp_token_logprobs(
            self._h, logits.data_ptr(), _dtype(logits), rows, V, ld, tp, temperature, top_k, lpp, entropy.data_ptr(),
            norm.data_ptr(), ip, kp, _stream(stream))
        if status:
            self._check(status)
        return TokenLogprobs(lp, entropy, norm, ids, tops, temperature)

    def token_logprobs_grad(self, logits, targets, lp: TokenLogprobs, grad_logprob=None, grad_entropy=None,
                            grad_lse=None, grad_top=None, V: int | None = None, out=None, stream=None):
        """estp_token_logprobs_grad: the gradient of the logits [rows, V], of the fields of `lp` (from
        token_logprobs on the same logits and targets) with the upstream gradients grad_logprob,
        grad_entropy, grad_lse [rows] and grad_top [rows, top_k].  out: where it goes, logits itself allowed."""
        import torch
        rows, V, ld = self._logits(logits, V)
        f32, per_row, k = torch.float32, (rows,), 0
        norm = self._is(lp.norm, f32, (rows, 2), "norm")
        tp = gp = hp = ep = sp = ap = ip = None
        if targets is not None:
            tp = self._is(targets, torch.int32, per_row, "targets")
        if grad_logprob is not None:
            gp = self._is(grad_logprob, f32, per_row, "grad_logprob")
        if grad_entropy is not None:
            hp, ep = self._is(grad_entropy, f32, per_row, "grad_entropy"), self._is(lp.entropy, f32, per_row, "entropy")
        if grad_lse is not None:
            sp = self._is(grad_lse, f32, per_row, "grad_lse")
        if grad_top is not None:
            if lp.top_ids is None:
                raise ValueError("grad_top needs the alternatives that it belongs to")
            k = lp.top_ids.shape[-1]
            ip, ap = self._is(lp.top_ids, torch.int32, (rows, k), "top_ids"), self._is(grad_top, f32, (rows, k), "grad_top")
        out, ldo = self._grad_out(logits, rows, V, out, stream)
        status = self._lib.estp_token_logprobs_grad(
            self._h, logits.data_ptr(), _dtype(logits), rows, V, ld, norm, ep, tp, lp.temperature, k, ip, gp, hp, sp, ap,
            out.data_ptr(), ldo, _stream(stream))
        if status:
            self._check(status)
        return out

    def distill_loss(self, logits, teacher_ids, teacher_logits, temperature: float = 1.0, tail: bool = False,
                     row_weight=None, grads: bool = True, V: int | None = None, out=None, stream=None):
        """estp_distill_loss: the divergence of the student's logits [rows, >= V] from the teacher's top
        tokens (teacher_ids int32, teacher_logits fp32 [rows, K]): the loss [rows] and, with grads, its
        gradient [rows, V] times row_weight [rows].  tail: teacher_logits are log probabilities
        at this temperature and the rest of the vocabulary is one bucket.  out: where the
        gradient goes, logits itself allowed.  The loss alone uses the context's scratch, as token_logprobs does."""
        import torch
        rows, V, ld = self._logits(logits, V)
        K = teacher_ids.shape[-1]
        ip = self._is(teacher_ids, torch.int32, (rows, K), "teacher_ids")
        xp = self._is(teacher_logits, torch.float32, (rows, K), "teacher_logits")
        wp = None if row_weight is None else self._is(row_weight, torch.float32, (rows,), "row_weight")
        loss, gp, ldo = self._empty((rows,), torch.float32, logits.device, stream), None, 0
        if grads:
            out, ldo = self._grad_out(logits, rows, V, out, stream)
            gp = out.data_ptr()
        status = self._lib.estp_distill_loss(
            self._h, logits.data_ptr(), _dtype(logits), rows, V, ld, ip, xp, K, temperature, 1 if tail else 0, wp,
            loss.data_ptr(), gp, ldo, _stream(stream))
        if status:
            self._check(status)
        return (loss, out) if grads else loss
