"""The operators of a batched tree verification: rotary positions, a paged cache of 16 or 8 bits, tree attention and log
probabilities (ngg.h states what each computes; csrc/ngg_torch.cpp checks the tensors and makes the calls).

Outputs and workspaces come from torch's allocator on the stream that the call runs on: the current one, or `stream`, which
then has to have been made to wait for whatever wrote the inputs.  Nothing is synchronised.  No gradients are recorded: a call on
tensors that require them raises, unless gradients are off (`rotary` with inverse=True is the gradient of `rotary`).
"""
from __future__ import annotations

import collections
import ctypes as C

import numpy as np
import torch

from . import NGG_BF16, NGG_F32, NGG_FP8, NGG_OK, NggError, load_binding, load_library
from . import ngg_kv_pages, ngg_rope, ngg_rope_scaling

_binding = load_binding()
_KINDS = {"linear": 1, "base": 2, "bands": 3, "ramp": 4}
_CACHES = {"f32": NGG_F32, "bf16": NGG_BF16, "fp8": NGG_FP8}

TokenLogprobs = collections.namedtuple("TokenLogprobs", "logprobs entropy lse top_ids top_logprobs")


def _check(st):
    if st != NGG_OK:
        raise NggError(st, load_library().ngg_last_error(None).decode())


def _on(stream, call, *args, keep=()):
    """The call on another stream than the current one; the inputs' memory is kept until the stream is done with it."""
    for t in (*args, *keep):
        if isinstance(t, torch.Tensor) and t.is_cuda:
            t.record_stream(stream)
    with torch.cuda.stream(stream):
        return call(*args)


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
        _check(load_library().ngg_rope_table(theta, rotary_dim, n_positions, C.byref(sc) if sc is not None else None, cos.ctypes.data,
                                             sin.ctypes.data))
        self.cos, self.sin = torch.from_numpy(cos).to(device), torch.from_numpy(sin).to(device)
        self.rotary_dim, self.n_positions, self.interleaved = rotary_dim, n_positions, bool(interleaved)
        self._c = ngg_rope(self.cos.data_ptr(), self.sin.data_ptr(), n_positions, rotary_dim, int(self.interleaved))
        self._at = C.addressof(self._c)


def rotary(rope, positions, q, k=None, inverse=False, out=None, k_out=None, stream=None):
    """ngg_rotary on q and, in the same launch, k: [tokens, heads, head_dim], any strides with contiguous heads; positions int32
    [tokens].  out and k_out may be q and k themselves.  Returns the rotated q, or both."""
    if stream is not None:
        return _on(stream, _binding.rotary, rope._at, rope.cos, positions, q, k, inverse, out, k_out, keep=(rope.sin,))
    return _binding.rotary(rope._at, rope.cos, positions, q, k, inverse, out, k_out)


class KVPages:
    """A pool of pages of keys and values (ngg_kv_pages) in memory of its own.  cache: "f32", "bf16", or "fp8" for 8 bits an
    element with a power of two for every position and head."""

    def __init__(self, n_pages, page_size, n_kv_heads, head_dim, cache="bf16", device="cuda"):
        if cache not in _CACHES:
            raise ValueError(f"unknown cache type {cache!r}")
        self.n_pages, self.page_size, self.n_kv_heads, self.head_dim, self.cache = n_pages, page_size, n_kv_heads, head_dim, cache
        self._c = ngg_kv_pages(None, None, None, None, n_pages, page_size, n_kv_heads, head_dim, _CACHES[cache])
        values, exps = C.c_int64(0), C.c_int64(0)
        _check(load_library().ngg_kv_bytes(self._c, values, exps))
        if not torch.cuda.is_available():
            raise RuntimeError("ngg needs a GPU: there is no CPU fallback")
        self.k_bytes, self.v_bytes = (torch.zeros(values.value, dtype=torch.uint8, device=device) for _ in range(2))
        self._c.k, self._c.v = self.k_bytes.data_ptr(), self.v_bytes.data_ptr()
        self.k_exps = self.v_exps = None
        if exps.value:
            self.k_exps, self.v_exps = (torch.full((exps.value,), 127, dtype=torch.uint8, device=device) for _ in range(2))
            self._c.k_exp, self._c.v_exp = self.k_exps.data_ptr(), self.v_exps.data_ptr()
        self._at = C.addressof(self._c)
        self._own = torch.float32 if cache == "f32" else torch.bfloat16

    def _memory(self):
        return (self.k_bytes, self.v_bytes, self.k_exps, self.v_exps)

    def write(self, k, v, slots, rope=None, positions=None, stream=None):
        """ngg_kv_write: k and v [tokens, kv heads, head_dim], any strides with contiguous heads, to slots (int32 [tokens]); with a
        Rope the keys are rotated to positions (int32 [tokens]) on the way."""
        at, table = (rope._at, rope.cos) if rope is not None else (0, None)
        if stream is not None:
            sin = (rope.sin,) if rope is not None else ()
            return _on(stream, _binding.kv_write, self._at, self.k_bytes, k, v, slots, at, table, positions, keep=self._memory() + sin)
        _binding.kv_write(self._at, self.k_bytes, k, v, slots, at, table, positions)

    def read(self, slots, dtype=None, stream=None):
        """ngg_kv_read: the keys and values of slots (int32 [tokens]), [tokens, kv heads, head_dim] each, in dtype (default: the
        pool's, bfloat16 for 8 bits)."""
        if stream is not None:
            return _on(stream, _binding.kv_read, self._at, self.k_bytes, slots, dtype or self._own, keep=self._memory())
        return _binding.kv_read(self._at, self.k_bytes, slots, dtype or self._own)


def tree_mask(parents):
    """ngg_tree_mask on the host: parents (-1: follows the context) -> (mask int64 [n, words], depth int32 [n]) as numpy arrays."""
    p = np.ascontiguousarray(parents, dtype=np.int32)
    n = len(p)
    mask, depth = np.zeros((n, max(1, (n + 63) // 64)), np.int64), np.zeros(n, np.int32)
    _check(load_library().ngg_tree_mask(p.ctypes.data, n, mask.ctypes.data, depth.ctypes.data))
    return mask, depth


def tree_attention(q, kv, pages, context_lens, mask=None, tree_lens=None, scale=None, out=None, want_lse=False, workspace=None, stream=None):
    """ngg_tree_attention: q [batch, tree, heads, head_dim] over kv (KVPages) through pages (int32 [batch, max_pages]) behind
    context_lens cached positions (int32 [batch]); the launch is planned for all of pages, of which its first columns do where no
    sequence is longer.  mask: int64 [tree, words] for all or [batch, tree, words], None for a chain; tree_lens: int32
    [batch] or None; scale: 1 / sqrt(head_dim) by default.  workspace: a uint8 tensor kept by the caller, or None to take one per
    call.  Returns out, or (out, lse) with lse float32 [batch, tree, heads]."""
    if stream is not None:
        return _on(stream, _binding.tree_attention, kv._at, kv.k_bytes, q, pages, context_lens, mask, tree_lens, scale, out, want_lse, workspace,
                   keep=kv._memory())
    return _binding.tree_attention(kv._at, kv.k_bytes, q, pages, context_lens, mask, tree_lens, scale, out, want_lse, workspace)


def token_logprobs(logits, targets=None, top_n=0, scale=1.0, stream=None):
    """ngg_token_logprobs on logits [rows, vocab] (any row stride): a TokenLogprobs of logprobs (float32 [rows, targets], or [rows]
    for targets of shape [rows]; None without), entropy and lse (float32 [rows]), top_ids (int32) and top_logprobs ([rows, top_n];
    None without)."""
    if stream is not None:
        return TokenLogprobs(*_on(stream, _binding.token_logprobs, logits, targets, top_n, scale))
    return TokenLogprobs(*_binding.token_logprobs(logits, targets, top_n, scale))
