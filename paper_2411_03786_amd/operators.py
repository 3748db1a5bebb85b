"""The operators of a batched tree verification: rotary positions, a paged cache of 16 or 8 bits, tree attention and log
probabilities (argument marshalling; the work is done in libngg's kernels, ngg.h states what each computes).

Outputs and workspaces come from torch's allocator on the stream that the call runs on: the current one, or `stream`, which
then has to have been made to wait for whatever wrote the inputs.  Nothing is synchronised.
"""
from __future__ import annotations

import collections
import contextlib
import ctypes as C
import math

import numpy as np
import torch

from . import NGG_BF16, NGG_F32, NGG_FP8, NGG_OK, NggError, load_library
from . import ngg_kv_pages, ngg_rope, ngg_rope_scaling, ngg_rotary_rows, ngg_score_args, ngg_tree_args

_DTYPES = {torch.float32: NGG_F32, torch.bfloat16: NGG_BF16}
_KINDS = {"linear": 1, "base": 2, "bands": 3, "ramp": 4}
_CACHES = {"f32": NGG_F32, "bf16": NGG_BF16, "fp8": NGG_FP8}

TokenLogprobs = collections.namedtuple("TokenLogprobs", "logprobs entropy lse top_ids top_logprobs")


def _raise(st):
    raise NggError(st, load_library().ngg_last_error(None).decode())


def _dtype(t, what):
    dt = _DTYPES.get(t.dtype)
    if dt is None:
        raise TypeError(f"{what} must be float32 or bfloat16, not {t.dtype}")
    return dt


def _on_gpu(first, *others):
    """All tensors on one GPU, the current one."""
    d = first.device
    if d.type != "cuda":
        raise RuntimeError("ngg needs a GPU: there is no CPU fallback")
    for t in others:
        if t is not None and t.device != d:
            raise ValueError(f"tensors on {d} and {t.device}")
    if d.index != torch.cuda.current_device():
        raise ValueError(f"tensors on {d}, the current device is cuda:{torch.cuda.current_device()}")


def _inner(t, what):
    if t.stride(-1) != 1 and t.shape[-1] != 1:
        raise ValueError(f"the last dimension of {what} must be contiguous")


def _ints(t, what, *shape):
    """A contiguous int32 tensor of this shape."""
    if t.dtype != torch.int32 or t.shape != shape or not t.is_contiguous():
        raise TypeError(f"{what} must be a contiguous int32 tensor of shape {tuple(shape)}")


_inline = contextlib.nullcontext()


def _on(stream, *tensors):
    """What to run under and the stream's handle.  A stream other than the current one keeps the inputs' memory until it is done."""
    if stream is None:
        return _inline, torch.cuda.current_stream().cuda_stream
    for t in tensors:
        if t is not None:
            t.record_stream(stream)
    return torch.cuda.stream(stream), stream.cuda_stream


class Rope:
    """A rotary table on the device (ngg_rope_table).  scaling: None, or a dict with `kind` ("linear", "base", "bands" or
    "ramp"), `factor` and, for the last two, `original`, `low` and `high`; `amplitude` with any."""

    def __init__(self, rotary_dim, n_positions, theta=10000.0, interleaved=False, scaling=None, device="cuda"):
        sc = None
        if scaling is not None:
            kind = scaling.get("kind")
            if kind not in _KINDS:
                raise ValueError(f"unknown scaling {kind!r}")
            sc = ngg_rope_scaling(_KINDS[kind], int(scaling.get("original", 0)), float(scaling["factor"]), float(scaling.get("low", 0.0)),
                                  float(scaling.get("high", 0.0)), float(scaling.get("amplitude", 0.0)))
        shape = (max(int(n_positions), 0), max(int(rotary_dim) // 2, 0))
        cos, sin = np.empty(shape, np.float32), np.empty(shape, np.float32)
        st = load_library().ngg_rope_table(theta, rotary_dim, n_positions, C.byref(sc) if sc is not None else None, cos.ctypes.data,
                                           sin.ctypes.data)
        if st != NGG_OK:
            _raise(st)
        self.cos, self.sin = torch.from_numpy(cos).to(device), torch.from_numpy(sin).to(device)
        self.rotary_dim, self.n_positions, self.interleaved = rotary_dim, n_positions, bool(interleaved)
        self._c = ngg_rope(self.cos.data_ptr(), self.sin.data_ptr(), n_positions, rotary_dim, int(self.interleaved))


def rotary(rope, positions, q, k=None, inverse=False, out=None, k_out=None, stream=None):
    """ngg_rotary on q and, in the same launch, k: [tokens, heads, head_dim], any strides with contiguous heads; positions int32
    [tokens].  out and k_out may be q and k themselves.  Returns the rotated q, or both."""
    n, _, hd = q.shape
    dt = _dtype(q, "q")
    _on_gpu(q, k, positions, rope.cos, out, k_out)
    _ints(positions, "positions", n)
    with_k = k is not None
    if with_k and (k.shape[0] != n or k.shape[2] != hd or k.dtype != q.dtype or k.dim() != 3):
        raise ValueError("q and k must agree in tokens, head_dim and dtype")
    on, s = _on(stream, q, k, positions, out, k_out)
    with on:
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        if with_k and k_out is None:
            k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device)
    rows = []
    for x, o in ((q, out), (k, k_out)) if with_k else ((q, out),):
        _inner(x, "q and k")
        _inner(o, "the output")
        if o.shape != x.shape or o.dtype != x.dtype:
            raise ValueError("an output must have its input's shape and dtype")
        i, j = x.stride(), o.stride()
        rows.append(ngg_rotary_rows(x.data_ptr(), o.data_ptr(), i[0], i[1], j[0], j[1], x.shape[1]))
    st = load_library().ngg_rotary(rope._c, positions.data_ptr(), n, hd, dt, rows[0], rows[1] if with_k else None, int(inverse), s)
    if st != NGG_OK:
        _raise(st)
    return (out, k_out) if with_k else out


class KVPages:
    """A pool of pages of keys and values (ngg_kv_pages) in memory of its own.  cache: "f32", "bf16", or "fp8" for 8 bits an
    element with a power of two for every position and head."""

    def __init__(self, n_pages, page_size, n_kv_heads, head_dim, cache="bf16", device="cuda"):
        if cache not in _CACHES:
            raise ValueError(f"unknown cache type {cache!r}")
        self.lib = load_library()
        self.n_pages, self.page_size, self.n_kv_heads, self.head_dim, self.cache = n_pages, page_size, n_kv_heads, head_dim, cache
        self._c = ngg_kv_pages(None, None, None, None, n_pages, page_size, n_kv_heads, head_dim, _CACHES[cache])
        values, exps = C.c_int64(0), C.c_int64(0)
        st = self.lib.ngg_kv_bytes(self._c, values, exps)
        if st != NGG_OK:
            _raise(st)
        if not torch.cuda.is_available():
            raise RuntimeError("ngg needs a GPU: there is no CPU fallback")
        self.k_bytes, self.v_bytes = (torch.zeros(values.value, dtype=torch.uint8, device=device) for _ in range(2))
        self._c.k, self._c.v = self.k_bytes.data_ptr(), self.v_bytes.data_ptr()
        self.k_exps = self.v_exps = None
        if exps.value:
            self.k_exps, self.v_exps = (torch.full((exps.value,), 127, dtype=torch.uint8, device=device) for _ in range(2))
            self._c.k_exp, self._c.v_exp = self.k_exps.data_ptr(), self.v_exps.data_ptr()

    def _tokens(self, x, n, what):
        if x.dim() != 3 or x.shape != (n, self.n_kv_heads, self.head_dim):
            raise ValueError(f"{what} must have the shape {(n, self.n_kv_heads, self.head_dim)}")
        _inner(x, what)

    def write(self, k, v, slots, rope=None, positions=None, stream=None):
        """ngg_kv_write: k and v [tokens, kv heads, head_dim], any strides with contiguous heads, to slots (int32 [tokens]); with a
        Rope the keys are rotated to positions (int32 [tokens]) on the way."""
        n = slots.shape[0]
        _on_gpu(self.k_bytes, k, v, slots, positions)
        _ints(slots, "slots", n)
        self._tokens(k, n, "k")
        self._tokens(v, n, "v")
        dt = _dtype(k, "k")
        if v.dtype != k.dtype:
            raise TypeError("k and v must have one dtype")
        rp = pp = None
        if rope is not None:
            if positions is None:
                raise ValueError("rope needs positions")
            _ints(positions, "positions", n)
            rp, pp = rope._c, positions.data_ptr()
        _, s = _on(stream, k, v, slots, positions)
        a, b = k.stride(), v.stride()
        st = self.lib.ngg_kv_write(self._c, k.data_ptr(), v.data_ptr(), dt, (C.c_int64 * 4)(a[0], a[1], b[0], b[1]), slots.data_ptr(), n, rp, pp, s)
        if st != NGG_OK:
            _raise(st)

    def read(self, slots, dtype=None, stream=None):
        """ngg_kv_read: the keys and values of slots (int32 [tokens]), [tokens, kv heads, head_dim] each, in dtype (default: the
        pool's, bfloat16 for 8 bits)."""
        n = slots.shape[0]
        _on_gpu(self.k_bytes, slots)
        _ints(slots, "slots", n)
        if dtype is None:
            dtype = torch.float32 if self.cache == "f32" else torch.bfloat16
        if dtype not in _DTYPES:
            raise TypeError(f"dtype must be float32 or bfloat16, not {dtype}")
        on, s = _on(stream, slots)
        with on:
            out = torch.empty((2, n, self.n_kv_heads, self.head_dim), dtype=dtype, device=slots.device)
        k, v = out[0], out[1]
        t, h = self.n_kv_heads * self.head_dim, self.head_dim
        st = self.lib.ngg_kv_read(self._c, slots.data_ptr(), n, _DTYPES[dtype], k.data_ptr(), v.data_ptr(), (C.c_int64 * 4)(t, h, t, h), s)
        if st != NGG_OK:
            _raise(st)
        return k, v


def tree_mask(parents):
    """ngg_tree_mask on the host: parents (-1: follows the context) -> (mask int64 [n, words], depth int32 [n]) as numpy arrays."""
    p = np.ascontiguousarray(parents, dtype=np.int32)
    n = len(p)
    mask, depth = np.zeros((n, max(1, (n + 63) // 64)), np.int64), np.zeros(n, np.int32)
    st = load_library().ngg_tree_mask(p.ctypes.data, n, mask.ctypes.data, depth.ctypes.data)
    if st != NGG_OK:
        _raise(st)
    return mask, depth


def tree_attention(q, kv, pages, context_lens, mask=None, tree_lens=None, scale=None, out=None, want_lse=False, workspace=None, stream=None):
    """ngg_tree_attention: q [batch, tree, heads, head_dim] over kv (KVPages) through pages (int32 [batch, max_pages]) behind
    context_lens cached positions (int32 [batch]).  mask: int64 [tree, words] for all or [batch, tree, words], None for a chain; tree_lens: int32
    [batch] or None; scale: 1 / sqrt(head_dim) by default.  workspace: a uint8 tensor kept by the caller, or None to take one per
    call.  Returns out, or (out, lse) with lse float32 [batch, tree, heads]."""
    B, T, H, hd = q.shape
    dt = _dtype(q, "q")
    _on_gpu(kv.k_bytes, q, pages, context_lens, mask, tree_lens, out, workspace)
    if hd != kv.head_dim:
        raise ValueError(f"q has heads of {hd}, the cache of {kv.head_dim}")
    _inner(q, "q")
    if pages.dtype != torch.int32 or pages.dim() != 2 or pages.shape[0] != B:
        raise TypeError(f"pages must be an int32 tensor of shape ({B}, max_pages)")
    _inner(pages, "pages")
    _ints(context_lens, "context_lens", B)
    if tree_lens is not None:
        _ints(tree_lens, "tree_lens", B)
    mb = mt = 0
    if mask is not None:
        words = (T + 63) // 64
        if mask.dtype != torch.int64 or mask.shape not in ((T, words), (B, T, words)):
            raise TypeError(f"mask must be an int64 tensor of shape {(T, words)} or {(B, T, words)}")
        _inner(mask, "mask")
        mt, mb = mask.stride(-2), mask.stride(0) if mask.dim() == 3 else 0
    on, s = _on(stream, q, pages, context_lens, mask, tree_lens, out, workspace, kv.k_bytes, kv.v_bytes, kv.k_exps, kv.v_exps)
    lib = kv.lib
    lse = None
    with on:
        if out is None:
            out = torch.empty((B, T, H, hd), dtype=q.dtype, device=q.device)
        elif out.shape != q.shape or out.dtype != q.dtype:
            raise ValueError("out must have the shape and dtype of q")
        else:
            _inner(out, "out")
        if want_lse:
            lse = torch.empty((B, T, H), dtype=torch.float32, device=q.device)
        i, j = q.stride(), out.stride()
        a = ngg_tree_args(q.data_ptr(), out.data_ptr(), lse.data_ptr() if want_lse else None, i[0], i[1], i[2], j[0], j[1], j[2],
                          pages.data_ptr(), pages.stride(0), context_lens.data_ptr(), tree_lens.data_ptr() if tree_lens is not None else None,
                          mask.data_ptr() if mask is not None else None, mb, mt, pages.shape[1], B, T, H, dt,
                          1.0 / math.sqrt(hd) if scale is None else scale)
        if workspace is None:
            need = C.c_int64(0)
            st = lib.ngg_tree_attention_workspace(kv._c, a, need)
            if st != NGG_OK:
                _raise(st)
            workspace = torch.empty(max(need.value, 16), dtype=torch.uint8, device=q.device)
        elif workspace.dtype != torch.uint8 or not workspace.is_contiguous():
            raise TypeError("workspace must be a contiguous uint8 tensor")
        st = lib.ngg_tree_attention(kv._c, a, workspace.data_ptr(), workspace.numel(), s)
    if st != NGG_OK:
        _raise(st)
    return (out, lse) if want_lse else out


def token_logprobs(logits, targets=None, top_n=0, scale=1.0, stream=None):
    """ngg_token_logprobs on logits [rows, vocab] (any row stride): a TokenLogprobs of logprobs (float32 [rows, targets], or [rows]
    for targets of shape [rows]; None without), entropy and lse (float32 [rows]), top_ids (int32) and top_logprobs ([rows, top_n];
    None without)."""
    n, V = logits.shape
    dt = _dtype(logits, "logits")
    _on_gpu(logits, targets)
    _inner(logits, "logits")
    m = 0
    if targets is not None:
        if targets.dtype != torch.int32 or targets.dim() not in (1, 2) or targets.shape[0] != n or not targets.is_contiguous():
            raise TypeError(f"targets must be a contiguous int32 tensor of {n} rows")
        m = 1 if targets.dim() == 1 else targets.shape[1]
    on, s = _on(stream, logits, targets)
    lib = load_library()
    with on:
        f = torch.empty(n * (2 + m + top_n), dtype=torch.float32, device=logits.device)
        ids = torch.empty((n, top_n), dtype=torch.int32, device=logits.device) if top_n > 0 else None
        base = f.data_ptr()
        a = ngg_score_args(logits.data_ptr(), logits.stride(0), dt, n, V, scale, targets.data_ptr() if m else None, m, top_n,
                           base + 8 * n, base, base + 4 * n, base + 4 * n * (2 + m), ids.data_ptr() if ids is not None else None)
        need = C.c_int64(0)
        st = lib.ngg_token_logprobs_workspace(a, need)
        if st != NGG_OK:
            _raise(st)
        ws = torch.empty(need.value, dtype=torch.uint8, device=logits.device) if need.value else None
        st = lib.ngg_token_logprobs(a, ws.data_ptr() if ws is not None else None, need.value, s)
    if st != NGG_OK:
        _raise(st)
    return TokenLogprobs(f[2 * n:(2 + m) * n].view(targets.shape) if targets is not None else None, f[:n], f[n:2 * n], ids,
                         f[(2 + m) * n:].view(n, top_n) if top_n > 0 else None)
