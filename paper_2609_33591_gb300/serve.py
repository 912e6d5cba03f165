"""Serving with K-interval attention: block tables, rotary positions, a paged cache that holds
keys and values in 4 bits, and attention over it (include/kint_serve.h).

The functions take torch tensors and run libkint's kernels on the current stream, or the one
given, to which the memory that a call allocates then belongs.  One step of a layer is

    plan = extend_blocks(...)                       # once a step
    q = append(k, v, plan.slots, pages, q=q, pos=plan.pos, table=rope)
    o = attention(q, pages, blocks, plan.lens, plan.cu, cfg, slots=plan.slots, ...)

Only ``rotary`` is differentiable.  The other calls' results raise where a gradient through them is asked for (keys and values
end in the cache, whose codes have none).

``PagedCache`` keeps the tables and lengths between steps, ``rotary`` is the differentiable
rotation for training, and ``KIntServingAttention`` is the GPT-2 block of ``attention`` with
rotary positions, a training forward and a serving step.
"""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import math
from typing import NamedTuple

import torch

from . import build as _build
from . import kint
from .attention import KIntSelfAttention, kint_attention

GROUP = 64  # channels that share one (scale, centre) pair
DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}

# Every symbol include/kint_serve.h declares.
EXPORTS = ("kint_cache_block_bytes", "kint_blocks_extend", "kint_rope_table", "kint_rope", "kint_cache_append",
           "kint_cache_read", "kint_cache_attn", "kint_cache_attn_step", "kint_cache_attn_workspace_bytes")


class kint_heads(ctypes.Structure):
    _fields_ = [("ptr", ctypes.c_void_p), ("stride_b", ctypes.c_longlong), ("stride_t", ctypes.c_longlong),
                ("stride_h", ctypes.c_longlong), ("heads", ctypes.c_int)]


class kint_cache(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_void_p), ("block_stride", ctypes.c_longlong), ("num_blocks", ctypes.c_int),
                ("block_size", ctypes.c_int), ("kv_heads", ctypes.c_int), ("d", ctypes.c_int)]


_lib = None


def load():
    """libkint with the serving entry points' types set."""
    global _lib
    if _lib is None:
        lib = kint.load()
        vp, i, f, ll, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_longlong, ctypes.c_size_t
        hp, cp = ctypes.POINTER(kint_heads), ctypes.POINTER(kint_cache)
        for name, args, res in (
                ("kint_cache_block_bytes", [i, i, i], sz),
                ("kint_blocks_extend", [vp, vp, vp, i, i, vp, i, vp, i, i, i] + [vp] * 8, i),
                ("kint_rope_table", [vp, i, i, ctypes.POINTER(ctypes.c_double), ctypes.c_double, vp], i),
                ("kint_rope", [hp, hp, hp, hp, vp, ll, vp, i, i, i, i, i, i, i, i, vp], i),
                ("kint_cache_append", [cp, hp, hp, vp, i, hp, hp, vp, vp, i, i, i, i, vp], i),
                ("kint_cache_read", [cp, vp, i, hp, hp, i, vp], i),
                ("kint_cache_attn", [hp, hp, cp, vp, i, i, vp, vp, i, i, i, i, i, i, f, i, i, i, i, vp, sz, vp], i),
                ("kint_cache_attn_step", [hp, hp, cp, vp, i, i, vp, vp, i, i, i, i, i, i, f, i, i, i, i, vp, i, vp, sz, vp], i),
                ("kint_cache_attn_workspace_bytes", [i] * 8, sz)):
            fn = getattr(lib, name)
            fn.argtypes, fn.restype = args, res
        _lib = lib
    return _lib


_mod = None


def _ext():
    """The marshalling module (csrc/serve_torch.cpp): checks, output allocation and the C call, one Python call deep."""
    global _mod
    if _mod is None:
        lib = load()
        loader = importlib.machinery.ExtensionFileLoader("_kint_serve", _build.EXT)
        mod = importlib.util.module_from_spec(importlib.util.spec_from_loader("_kint_serve", loader))
        loader.exec_module(mod)
        mod.bind(*(ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in (
            "kint_blocks_extend", "kint_rope", "kint_cache_append", "kint_cache_read", "kint_cache_attn_step",
            "kint_cache_attn_workspace_bytes")), kint.KintError)
        _mod = mod
    return _mod


def _handle(stream):
    return None if stream is None else stream.cuda_stream


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


# ---- block tables and slots -----------------------------------------------------------------------

class BlockPlan(NamedTuple):
    """One step's rows: lens [B] after it, cu [B + 1] row offsets, and for each new token its slot, position and request."""
    lens: torch.Tensor
    cu: torch.Tensor
    slots: torch.Tensor
    pos: torch.Tensor
    req: torch.Tensor
    n_free: torch.Tensor
    refused: torch.Tensor


def extend_blocks(lens, new, table, free, n_free, block_size: int, tokens: int, *, stream=None) -> BlockPlan:
    """Blocks and slots for new[b] more tokens of each request (int32 [B] both).  ``table`` [B, width] gets the blocks
    taken from the end of free[:n_free]; ``tokens`` is the number of places for new tokens (those left over are -1)."""
    return BlockPlan(*(_mod or _ext()).extend_blocks(lens, new, table, free, n_free, block_size, tokens, _handle(stream)))


# ---- rotary positions -----------------------------------------------------------------------------

def rope_frequencies(rot: int, base: float = 10000.0, *, scaling: str | None = None, factor: float = 1.0,
                     original_len: int = 4096, slow: float = 1.0, fast: float = 32.0) -> tuple[list[float], float]:
    """Angles a position of the rot / 2 pairs, base^(-2 i / rot), and the magnitude of the rotation.

    scaling, for contexts longer than those trained on (original_len tokens, longer by ``factor``):
      None      the plain angles;
      "linear"  every angle / factor (position interpolation, Chen et al. 2023);
      "base"    base * factor^(rot / (rot - 2)): the slowest pair turns 1 / factor as far, the fastest as before (known as
                NTK-aware scaling);
      "bands"   (YaRN, Peng et al. 2023) pairs that turn less than ``slow`` times over original_len are divided by factor, those that turn more
                than ``fast`` times are kept, a linear blend between; magnitude 0.1 ln(factor) + 1.
    """
    _need(rot >= 2 and rot % 2 == 0, "rot must be even and at least 2")
    _need(base > 0 and factor > 0, "base and factor must be positive")
    _need(scaling in (None, "linear", "base", "bands"), f"unknown scaling {scaling!r}")
    if scaling == "base" and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    freq = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    mag = 1.0
    if scaling == "linear":
        freq = [w / factor for w in freq]
    elif scaling == "bands":
        _need(fast > slow, "fast must exceed slow")
        keep = [min(max((original_len * w / (2 * math.pi) - slow) / (fast - slow), 0.0), 1.0) for w in freq]
        freq = [w * k + w / factor * (1 - k) for w, k in zip(freq, keep)]
        mag = 0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0
    return freq, mag


def rope_table(max_pos: int, rot: int, base: float = 10000.0, *, device="cuda", stream=None, **scaling) -> torch.Tensor:
    """(cos, sin) pairs [max_pos, rot / 2, 2], fp32 (angles and functions in fp64); keywords as rope_frequencies."""
    freq, mag = rope_frequencies(rot, base, **scaling)
    with torch.cuda.stream(stream):  # (None: the current one)
        table = torch.empty(max_pos, rot // 2, 2, dtype=torch.float32, device=device)
        handle = torch.cuda.current_stream().cuda_stream
        rc = load().kint_rope_table(table.data_ptr(), max_pos, rot, (ctypes.c_double * len(freq))(*freq), mag, handle)
    if rc:
        raise kint.KintError(rc, "kint_rope_table")
    return table


def rope(q, k, pos, table, *, interleaved: bool = False, inverse: bool = False, out=None, stream=None):
    """q [B, T, heads, d] and k (or None) rotated to positions pos [B, T] or [T] (int32; -1: left as it is).
    inverse: the opposite rotation, the gradient's way back.  out: (q', k') to write, which may be q and k."""
    qo, ko = (None, None) if out is None else out
    return (_mod or _ext()).rope(q, k, pos, table, interleaved, inverse, qo, ko, _handle(stream))


class RotaryFn(torch.autograd.Function):
    """rope as a differentiable op: gradients are turned back by the inverse rotation, which is this op again, so derivatives of
    every order follow."""

    @staticmethod
    def forward(ctx, q, k, pos, table, interleaved: bool, inverse: bool = False):
        ctx.save_for_backward(pos, table)
        ctx.interleaved, ctx.inverse = interleaved, inverse
        return rope(q, k, pos, table, interleaved=interleaved, inverse=inverse)

    @staticmethod
    def backward(ctx, dq, dk):
        pos, table = ctx.saved_tensors
        dq, dk = (x if x is None or x.stride(-1) == 1 else x.contiguous() for x in (dq, dk))
        dq, dk = RotaryFn.apply(dq, dk, pos, table, ctx.interleaved, not ctx.inverse)
        return dq, dk, None, None, None, None


def rotary(q, k, pos, table, interleaved: bool = False):
    """Differentiable rotary positions of q and k (or None) [B, T, heads, d]."""
    return RotaryFn.apply(q, k, pos, table, interleaved)


# ---- the cache --------------------------------------------------------------------------------------

def cache_pages(num_blocks: int, block_size: int, kv_heads: int, d: int, *, device="cuda") -> torch.Tensor:
    """An empty pool of pages [num_blocks, kv_heads, block_size / 16, 18 d] (uint8)."""
    if load().kint_cache_block_bytes(block_size, kv_heads, d) == 0:
        raise kint.KintError(-2, "cache_pages: block_size must be a power of two from 16 to 4096, d 64 or 128")
    return torch.zeros(num_blocks, kv_heads, block_size // 16, 18 * d, dtype=torch.uint8, device=device)


def append(k, v, slots, pages, *, q=None, pos=None, table=None, interleaved: bool = False, q_out=None, stream=None):
    """New tokens' k and v [tokens, kv_heads, d] into the cache at slots [tokens] (int64; -1: skipped), the keys rotated
    to pos [tokens] where a table is given.  Returns q [tokens, heads, d] rotated likewise, in q_out if given (without a table
    q itself, without q None)."""
    return (_mod or _ext()).append(k, v, slots, pages, q, pos, table, interleaved, q_out, _handle(stream))


def read(pages, slots, *, dtype=torch.float32, stream=None):
    """Cached keys and values of slots [tokens] as numbers: k, v [tokens, kv_heads, d]; slot -1 gives zeros."""
    return (_mod or _ext()).read(pages, slots, DTYPES[dtype], _handle(stream))


def attention(q, pages, table, lens, cu, cfg: kint.Config, *, window: int = 0, sinks: int = 0, max_new: int | None = None,
              max_len: int | None = None, slots=None, out=None, ws=None, stream=None):
    """K-interval attention of new tokens over the cache: q [rows, heads, d], request b's rows cu[b] .. cu[b + 1] - 1 at
    the last positions of its lens[b] cached tokens, whose blocks are table[b].  window > 0: a row sees its last
    ``window`` keys and the first ``sinks``.  max_new and max_len bound the rows a request has and lens (host numbers
    that size the launch and its scratch; by default rows and what the table can hold, so give max_new = 1 when every request has one
    token: for 64 of them, 32 heads over 8 and a table of 32768 tokens, 0.3 GB of scratch and not 18.3).  ``slots``: the plan's, so that requests it refused
    get zeros (without them their rows are taken for the last positions of what is cached).  Rows that are no request's, or left out for
    their bounds, are zero in a new output and left as they are in ``out``."""
    return (_mod or _ext()).attention(q, pages, table, lens, cu, cfg.Kint, cfg.calib, cfg.tau, cfg.recon, window, sinks, max_new,
                                      max_len, out, ws, slots, _handle(stream))


def attention_workspace(B: int, heads: int, kv_heads: int, d: int, *, window: int = 0, sinks: int = 0, max_new: int = 1,
                        max_len: int, device="cuda") -> torch.Tensor:
    """Scratch of one ``attention`` call of these sizes (reusable, one call at a time)."""
    n = load().kint_cache_attn_workspace_bytes(B, heads, kv_heads, d, window, sinks, max_new, max_len)
    return torch.empty(max(n, 16), dtype=torch.uint8, device=device)


# ---- state between steps, and a layer on top ----------------------------------------------------------

class PagedCache:
    """The pages of `layers` layers and the tables of up to `requests` requests of up to `max_len` tokens, all on the GPU."""

    def __init__(self, layers: int, requests: int, max_len: int, num_blocks: int, kv_heads: int, d: int, *,
                 block_size: int = 32, device="cuda"):
        self.block_size, self.max_len = block_size, max_len
        self.pages = cache_pages(layers * num_blocks, block_size, kv_heads, d, device=device).unflatten(0, (layers, num_blocks))
        width = -(-max_len // block_size)
        i32 = dict(dtype=torch.int32, device=device)
        self.table = torch.full((requests, width), -1, **i32)
        self.lens = torch.zeros(requests, **i32)
        self.free = torch.arange(num_blocks, **i32)
        self.n_free = torch.tensor([num_blocks], **i32)

    def extend(self, new, tokens: int, *, stream=None) -> BlockPlan:
        """Places for new[b] more tokens of every request (int32 [requests]), `tokens` rows in all."""
        plan = extend_blocks(self.lens, new, self.table, self.free, self.n_free, self.block_size, tokens, stream=stream)
        self.lens, self.n_free = plan.lens, plan.n_free
        return plan

    def release(self, request: int) -> None:
        """Ends a request: its blocks return to the free list.  Waits for the GPU."""
        held, n = -(-int(self.lens[request]) // self.block_size), int(self.n_free)
        self.free[n:n + held] = self.table[request, :held]
        self.table[request] = -1
        self.lens[request] = 0
        self.n_free += held


class KIntServingAttention(KIntSelfAttention):
    """The GPT-2 K-interval attention block with rotary positions: ``forward`` as in training (whole sequences, rotation
    and attention differentiable), ``step`` for new tokens over a 4-bit paged cache.  The cache has as many kv heads as
    the block has heads; weights are KIntSelfAttention's.  Sequences and the bound on a step's lengths have to lie within max_pos."""

    def __init__(self, n_embd: int = 768, n_head: int = 12, cfg: kint.Config | None = None, *, max_pos: int = 4096,
                 rot: int | None = None, base: float = 10000.0, interleaved: bool = False, window: int = 0, sinks: int = 0,
                 prec: int = kint.PREC_TF32, bias: bool = True, device="cuda", **scaling):
        super().__init__(n_embd, n_head, cfg, prec, bias)
        self.interleaved, self.window, self.sinks = interleaved, window, sinks
        self.to(device)
        self.register_buffer("rope", rope_table(max_pos, rot or n_embd // n_head, base, device=device, **scaling),
                             persistent=False)

    def _apply(self, fn, recurse=True):
        rope = self.rope if "rope" in self._buffers else None
        super()._apply(fn, recurse)
        if rope is not None and self.rope.dtype != rope.dtype:  # a cast of the layer is not one of its angles' cosines and sines
            self.rope = rope.to(self.rope.device)
        return self

    def forward(self, x, pos=None):
        B, T, C = x.shape
        H, D = self.n_head, C // self.n_head
        if self.window and self.window < T:
            raise ValueError("the training forward is full causal attention: T may not exceed the window")
        if pos is None:
            _need(T <= self.rope.size(0), f"T = {T} is past the layer's max_pos, {self.rope.size(0)}")
        q, k, v = (t.view(B, T, H, D) for t in self.c_attn(x).split(C, dim=2))
        pos = torch.arange(T, dtype=torch.int32, device=x.device) if pos is None else pos
        q, k = rotary(q, k, pos, self.rope, self.interleaved)
        q, k, v = (t.transpose(1, 2).float().contiguous() for t in (q, k, v))
        y = kint_attention(q, k, v, self.cfg, self.prec)
        return self.c_proj(y.to(x.dtype).transpose(1, 2).contiguous().view(B, T, C))

    @torch.no_grad()
    def step(self, x, cache: PagedCache, plan: BlockPlan, layer: int = 0, *, max_new: int | None = None,
             max_len: int | None = None):
        """x [rows, C]: the new tokens of every request in the plan's order (cache.extend).  Places left over and requests that
        the plan refused get the projection of zeros.  max_new and max_len as in ``attention``: by default all rows, and
        what the cache's table holds."""
        rows, C = x.shape
        D = C // self.n_head
        most = self.rope.size(0)
        _need((max_len or cache.max_len) <= most, f"requests of up to {max_len or cache.max_len} tokens are past the layer's max_pos, {most}")
        # (by default what the table's blocks hold: the cache lets a request fill its last one)
        max_len = max_len or min(cache.table.size(1) * cache.block_size, most)
        q, k, v = (t.view(rows, self.n_head, D) for t in self.c_attn(x).split(C, dim=1))
        pages = cache.pages[layer]
        q = append(k, v, plan.slots, pages, q=q, pos=plan.pos, table=self.rope, interleaved=self.interleaved)
        y = attention(q, pages, cache.table, plan.lens, plan.cu, self.cfg, window=self.window, sinks=self.sinks,
                      max_new=max_new, max_len=max_len, slots=plan.slots)
        return self.c_proj(y.view(rows, C))
