"""Serving with K-interval attention: block tables, rotary positions, a paged cache that holds
keys and values in 4 bits, and attention over it (include/kint_serve.h).

The functions take torch tensors and run libkint's kernels on the current stream (or the one
given); torch supplies the memory.  One step of a layer is

    plan = extend_blocks(...)                       # once a step
    q = append(k, v, plan.slots, pages, q=q, pos=plan.pos, table=rope)
    o = attention(q, pages, blocks, plan.lens, plan.cu, cfg, ...)

``PagedCache`` keeps the tables and lengths between steps, ``rotary`` is the differentiable
rotation for training, and ``KIntServingAttention`` is the GPT-2 block of ``attention`` with
rotary positions, a training forward and a serving step.
"""
from __future__ import annotations

import ctypes
import math
from dataclasses import dataclass

import torch

from . import kint
from .attention import KIntSelfAttention, kint_attention

GROUP = 64  # channels that share one (scale, centre) pair
DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}

# Every symbol include/kint_serve.h declares.
EXPORTS = ("kint_cache_block_bytes", "kint_blocks_extend", "kint_rope_table", "kint_rope", "kint_cache_append",
           "kint_cache_read", "kint_cache_attn", "kint_cache_attn_workspace_bytes")


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
                ("kint_cache_attn", [hp, hp, cp, vp, i, i, vp, vp, i, i, i, i, i, f, i, i, i, i, vp, sz, vp], i),
                ("kint_cache_attn_workspace_bytes", [i] * 8, sz)):
            fn = getattr(lib, name)
            fn.argtypes, fn.restype = args, res
        _lib = lib
    return _lib


# ---- arguments ----------------------------------------------------------------------------------

def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _heads(x, what: str, dims: int) -> kint_heads:
    """[..., heads, d] with contiguous channels on the GPU: (batch,) time, heads, d."""
    if not (x.is_cuda and x.dim() == dims and x.dtype in DTYPES and (x.stride(-1) == 1 or x.size(-1) == 1)):
        raise ValueError(f"{what}: expected a CUDA tensor of fp32, bf16 or fp16 with {dims} dimensions and contiguous channels")
    st = x.stride()
    return kint_heads(x.data_ptr(), st[0] if dims == 4 else 0, st[-3], st[-2], x.size(-2))


def _ints(x, what: str, dtype=torch.int32):
    if not (x.is_cuda and x.dtype == dtype and (x.dim() == 0 or x.stride(-1) == 1 or x.size(-1) <= 1)):
        raise ValueError(f"{what}: expected a contiguous CUDA tensor of {dtype}")
    return x.data_ptr()


def _pool(pages) -> kint_cache:
    """pages [num_blocks, kv_heads, block_size / 16, 18 d], uint8; blocks may be strided."""
    _need(pages.is_cuda and pages.dtype == torch.uint8 and pages.dim() == 4, "pages: expected a 4-D uint8 CUDA tensor")
    n, kv, slabs, size = pages.shape
    _need(size % 18 == 0 and pages.stride()[1:] == (slabs * size, size, 1),
          "pages: expected [num_blocks, kv_heads, block_size / 16, 18 d], contiguous within a block")
    return kint_cache(pages.data_ptr(), pages.stride(0), n, 16 * slabs, kv, size // 18)


def _stream(stream) -> int:
    return (torch.cuda.current_stream() if stream is None else stream).cuda_stream


def _run(rc: int, what: str):
    if rc:
        raise kint.KintError(rc, what)


# ---- block tables and slots -----------------------------------------------------------------------

@dataclass
class BlockPlan:
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
    B = lens.shape[0]
    _need(new.shape == lens.shape and table.dim() == 2 and table.size(0) == B, "lens, new and table disagree on the requests")
    args = [_ints(x, n) for x, n in ((lens, "lens"), (new, "new"), (table, "table"), (free, "free"), (n_free, "n_free"))]
    small = torch.empty(2 * B + 3 + 2 * tokens, dtype=torch.int32, device=lens.device)
    slots = torch.empty(tokens, dtype=torch.int64, device=lens.device)
    lens_o, cu, n_free_o, refused, pos, req = small.split((B, B + 1, 1, 1, tokens, tokens))
    at = small.data_ptr()
    _run(load().kint_blocks_extend(args[0], args[1], args[2], table.stride(0), table.size(1), args[3], free.numel(), args[4], B,
                                   block_size, tokens, at, at + 4 * (2 * B + 1), at + 4 * B, slots.data_ptr() or 8,
                                   at + 4 * (2 * B + 3), at + 4 * (2 * B + 3 + tokens), at + 4 * (2 * B + 2), _stream(stream)),
         "kint_blocks_extend")
    return BlockPlan(lens_o, cu, slots, pos, req, n_free_o, refused)


# ---- rotary positions -----------------------------------------------------------------------------

def rope_frequencies(rot: int, base: float = 10000.0, *, scaling: str | None = None, factor: float = 1.0,
                     original_len: int = 4096, slow: float = 1.0, fast: float = 32.0) -> tuple[list[float], float]:
    """Angles a position of the rot / 2 pairs, base^(-2 i / rot), and the magnitude of the rotation.

    scaling, for contexts longer than those trained on (original_len tokens, longer by ``factor``):
      None      the plain angles;
      "linear"  every angle / factor (positions interpolated);
      "base"    base * factor^(rot / (rot - 2)): the slowest pair turns 1 / factor as far, the fastest as before;
      "bands"   pairs that turn less than ``slow`` times over original_len are divided by factor, those that turn more
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
    table = torch.empty(max_pos, rot // 2, 2, dtype=torch.float32, device=device)
    _run(load().kint_rope_table(table.data_ptr(), max_pos, rot, (ctypes.c_double * len(freq))(*freq), mag, _stream(stream)),
         "kint_rope_table")
    return table


def _table(table):
    _need(table.is_cuda and table.dtype == torch.float32 and table.dim() == 3 and table.size(2) == 2 and table.is_contiguous(),
          "table: expected a contiguous fp32 CUDA tensor [max_pos, rot / 2, 2]")
    return table.data_ptr(), table.size(0), 2 * table.size(1)


_NO_HEADS = kint_heads(None, 0, 0, 0, 0)


def rope(q, k, pos, table, *, interleaved: bool = False, inverse: bool = False, out=None, stream=None):
    """q [B, T, heads, d] and k (or None) rotated to positions pos [B, T] or [T] (int32; -1: left as it is).
    inverse: the opposite rotation, the gradient's way back.  out: (q', k') to write, which may be q and k."""
    hq = _heads(q, "q", 4)
    _need(k is None or (k.dtype == q.dtype and k.shape[:2] == q.shape[:2] and k.size(3) == q.size(3)),
          "q and k disagree on type, batch, time or channels")
    _need(pos.shape == q.shape[:2] or pos.shape == q.shape[1:2], "pos: expected [B, T] or [T]")
    tab, max_pos, rot = _table(table)
    qo, ko = out if out is not None else (torch.empty_like(q), None if k is None else torch.empty_like(k))
    _need(qo.shape == q.shape and qo.dtype == q.dtype and (k is None or (ko.shape == k.shape and ko.dtype == k.dtype)),
          "out disagrees with q and k")
    B, T = q.shape[:2]
    if q.numel():
        _run(load().kint_rope(hq, _heads(qo, "out", 4), _NO_HEADS if k is None else _heads(k, "k", 4),
                              _NO_HEADS if k is None else _heads(ko, "out", 4), _ints(pos, "pos"),
                              pos.stride(0) if pos.dim() == 2 else 0, tab, max_pos, B, T, q.size(3), rot, interleaved, inverse,
                              DTYPES[q.dtype], _stream(stream)), "kint_rope")
    return qo, ko


class RotaryFn(torch.autograd.Function):
    """rope as a differentiable op: the gradients are turned back by the inverse rotation."""

    @staticmethod
    def forward(ctx, q, k, pos, table, interleaved: bool):
        ctx.save_for_backward(pos, table)
        ctx.interleaved = interleaved
        return rope(q, k, pos, table, interleaved=interleaved)

    @staticmethod
    def backward(ctx, dq, dk):
        pos, table = ctx.saved_tensors
        dq, dk = (x if x.stride(-1) == 1 else x.contiguous() for x in (dq, dk))
        dq, dk = rope(dq, dk, pos, table, interleaved=ctx.interleaved, inverse=True)
        return dq, dk, None, None, None


def rotary(q, k, pos, table, interleaved: bool = False):
    """Differentiable rotary positions of q and k [B, T, heads, d]."""
    return RotaryFn.apply(q, k, pos, table, interleaved)


# ---- the cache --------------------------------------------------------------------------------------

def cache_pages(num_blocks: int, block_size: int, kv_heads: int, d: int, *, device="cuda") -> torch.Tensor:
    """An empty pool of pages [num_blocks, kv_heads, block_size / 16, 18 d] (uint8)."""
    if load().kint_cache_block_bytes(block_size, kv_heads, d) == 0:
        raise kint.KintError(-2, "cache_pages: block_size must be a power of two from 16 to 4096, d 64 or 128")
    return torch.zeros(num_blocks, kv_heads, block_size // 16, 18 * d, dtype=torch.uint8, device=device)


def append(k, v, slots, pages, *, q=None, pos=None, table=None, interleaved: bool = False, q_out=None, stream=None):
    """New tokens' k and v [tokens, kv_heads, d] into the cache at slots [tokens] (int64; -1: skipped), the keys rotated
    to pos [tokens] where a table is given.  Returns q [tokens, heads, d] rotated likewise (None without q)."""
    hk, hv = _heads(k, "k", 3), _heads(v, "v", 3)
    pool = _pool(pages)
    n = k.size(0)
    _need(k.shape == v.shape and k.dtype == v.dtype and k.size(2) == pool.d and slots.shape == (n,),
          "k, v, slots and the pages disagree")
    _need(table is None or (pos is not None and pos.shape == (n,)), "a rotation needs pos [tokens]")
    turn = q is not None and table is not None
    if q is not None:
        _need(q.dim() == 3 and q.size(0) == n and q.size(2) == pool.d and q.dtype == k.dtype, "q and k disagree")
        if turn and q_out is None:
            q_out = torch.empty_like(q)
    tab, max_pos, rot = _table(table) if table is not None else (None, 0, 0)
    if n:
        _run(load().kint_cache_append(pool, hk, hv, _ints(slots, "slots", torch.int64), n, _heads(q, "q", 3) if turn else None,
                                      _heads(q_out, "q_out", 3) if turn else None, None if table is None else _ints(pos, "pos"),
                                      tab, max_pos, rot, interleaved, DTYPES[k.dtype], _stream(stream)), "kint_cache_append")
    return q_out if turn else q


def read(pages, slots, *, dtype=torch.float32, stream=None):
    """Cached keys and values of slots [tokens] as numbers: k, v [tokens, kv_heads, d]; slot -1 gives zeros."""
    pool = _pool(pages)
    n = slots.numel()
    kv = torch.empty(2, n, pool.kv_heads, pool.d, dtype=dtype, device=pages.device)
    k, v = kv.unbind(0)
    if n:
        _run(load().kint_cache_read(pool, _ints(slots, "slots", torch.int64), n, _heads(k, "k", 3), _heads(v, "v", 3),
                                    DTYPES[dtype], _stream(stream)), "kint_cache_read")
    return k, v


def attention(q, pages, table, lens, cu, cfg: kint.Config, *, window: int = 0, sinks: int = 0, max_new: int | None = None,
              max_len: int | None = None, out=None, ws=None, stream=None):
    """K-interval attention of new tokens over the cache: q [rows, heads, d], request b's rows cu[b] .. cu[b + 1] - 1 at
    the last positions of its lens[b] cached tokens, whose blocks are table[b].  window > 0: a row sees its last
    ``window`` keys and the first ``sinks``.  max_new and max_len bound the rows a request has and lens (host numbers
    that size the launch; by default rows and what the table can hold)."""
    hq = _heads(q, "q", 3)
    pool = _pool(pages)
    B = lens.size(0)
    _need(q.size(2) == pool.d and table.dim() == 2 and table.size(0) == B and cu.shape == (B + 1,),
          "q, pages, table, lens and cu disagree")
    out = torch.empty_like(q) if out is None else out
    _need(out.shape == q.shape and out.dtype == q.dtype, "out disagrees with q")
    if q.numel() == 0:
        return out
    width = table.size(1)
    max_new = q.size(0) if max_new is None else max_new
    max_len = width * pool.block_size if max_len is None else max_len
    lib = load()
    if ws is None:
        ws = attention_workspace(B, q.size(1), pool.kv_heads, pool.d, window=window, sinks=sinks, max_new=max_new,
                                 max_len=max_len, device=q.device)
    _run(lib.kint_cache_attn(hq, _heads(out, "out", 3), pool, _ints(table, "table"), table.stride(0), width, _ints(lens, "lens"),
                             _ints(cu, "cu"), B, window, sinks, cfg.Kint, cfg.calib, cfg.tau, cfg.recon, max_new, max_len,
                             DTYPES[q.dtype], ws.data_ptr(), ws.numel(), _stream(stream)), "kint_cache_attn")
    return out


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
        self.pages = torch.stack([cache_pages(num_blocks, block_size, kv_heads, d, device=device) for _ in range(layers)])
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
    the block has heads; weights are KIntSelfAttention's."""

    def __init__(self, n_embd: int = 768, n_head: int = 12, cfg: kint.Config | None = None, *, max_pos: int = 4096,
                 rot: int | None = None, base: float = 10000.0, interleaved: bool = False, window: int = 0, sinks: int = 0,
                 prec: int = kint.PREC_TF32, bias: bool = True, device="cuda", **scaling):
        super().__init__(n_embd, n_head, cfg, prec, bias)
        self.interleaved, self.window, self.sinks = interleaved, window, sinks
        self.to(device)
        self.register_buffer("rope", rope_table(max_pos, rot or n_embd // n_head, base, device=device, **scaling),
                             persistent=False)

    def forward(self, x, pos=None):
        B, T, C = x.shape
        H, D = self.n_head, C // self.n_head
        if self.window and self.window < T:
            raise ValueError("the training forward is full causal attention: T may not exceed the window")
        q, k, v = (t.view(B, T, H, D) for t in self.c_attn(x).split(C, dim=2))
        pos = torch.arange(T, dtype=torch.int32, device=x.device) if pos is None else pos
        q, k = rotary(q, k, pos, self.rope, self.interleaved)
        q, k, v = (t.transpose(1, 2).float().contiguous() for t in (q, k, v))
        y = kint_attention(q, k, v, self.cfg, self.prec)
        return self.c_proj(y.to(x.dtype).transpose(1, 2).contiguous().view(B, T, C))

    @torch.no_grad()
    def step(self, x, cache: PagedCache, plan: BlockPlan, layer: int = 0, *, max_new: int | None = None,
             max_len: int | None = None):
        """x [rows, C]: the new tokens of every request in the plan's order (cache.extend)."""
        rows, C = x.shape
        D = C // self.n_head
        q, k, v = (t.view(rows, self.n_head, D) for t in self.c_attn(x).split(C, dim=1))
        pages = cache.pages[layer]
        q = append(k, v, plan.slots, pages, q=q, pos=plan.pos, table=self.rope, interleaved=self.interleaved)
        y = attention(q, pages, cache.table, plan.lens, plan.cu, self.cfg, window=self.window, sinks=self.sinks,
                      max_new=max_new, max_len=max_len or cache.max_len)
        return self.c_proj(y.view(rows, C))
