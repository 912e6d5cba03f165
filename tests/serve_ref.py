"""Plain 64-bit forms of the serving operators (test infrastructure), on the CPU, from the definitions in
include/kint_serve.h."""
import math

import numpy as np
import torch

from paper_2609_33591_gb300 import kint


# ---- the cache's numbers ---------------------------------------------------------------------------

def quantise(x):
    """Codes 0..15, s, c (fp32 values of fp16 numbers) of fp32 x [..., d]; fp32 arithmetic, as the format defines it."""
    g = x.float().unflatten(-1, (-1, 64))
    bad = ~torch.isfinite(g).all(-1, keepdim=True)
    lo, hi = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    s = ((hi - lo) * torch.tensor(1.0 / 15.0)).clamp(max=65504).half().float()
    c = (lo + 8 * s).clamp(-65504, 65504).half().float()
    inv = torch.where(s > 0, 1 / s, torch.zeros_like(s))
    code = ((g - c) * inv).round().clamp(-8, 7) + 8
    code = torch.where(bad, torch.full_like(code, 8), code)
    c = torch.where(bad, torch.full_like(c, math.nan), c)
    return code.flatten(-2).to(torch.int64), s[..., 0], c[..., 0]


def dequantise(code, s, c):
    return (code.unflatten(-1, (-1, 64)).double() - 8) * s[..., None].double() + c[..., None].double()


def held(x):
    """The numbers the cache keeps of x, fp64."""
    return dequantise(*quantise(x)).flatten(-2)


def pack(k, v):
    """Slabs [..., 18 d] of k and v [..., 16, d] (fp32)."""
    d = k.shape[-1]
    lead = k.shape[:-2]
    out = np.zeros(lead + (18 * d,), np.uint8)
    for x, is_v in ((k, False), (v, True)):
        code, s, c = quantise(x)
        code = code.numpy().astype(np.uint8)
        sc = torch.stack([s, c], -1).half().contiguous().numpy().view(np.uint8).reshape(lead + (16 * d // 16,))
        base = 9 * d if is_v else 0
        out[..., base + 8 * d: base + 9 * d] = sc
        for j in range(16):
            for e in range(d):
                if is_v:
                    r, g, h = e // 64, e // 8 % 8, e // 4 % 2
                    at = 9 * d + ((8 * (j // 2) + g) * (d // 32) + 2 * r + h) * 4 + 2 * (j % 2) + e % 4 // 2
                else:
                    at = j * d // 2 + (e // 8 % 4) * d // 8 + 4 * (e // 32) + e % 8 // 2
                out[..., at] |= code[..., j, e] << (4 * (e % 2))
    return torch.from_numpy(out)


class Pool:
    """A pool filled through `pack`: request b's tokens of k[b], v[b] [len, kv, d] in scattered blocks."""

    def __init__(self, k, v, block, d, kv, seed=0, spare=3, garbage=None, width=None):
        rng = np.random.default_rng(seed)
        lens = [x.shape[0] for x in k]
        need = [-(-n // block) for n in lens]
        total = sum(need) + spare
        self.pages = torch.randint(0, 256, (total, kv, block // 16, 18 * d), dtype=torch.uint8,
                                   generator=torch.Generator().manual_seed(seed))
        fill = 0.0 if garbage is None else garbage
        for at in (8 * d, 17 * d):
            self.pages[..., at:at + d] = torch.full((d // 2,), fill, dtype=torch.half).view(torch.uint8)
        ids = rng.permutation(total)
        width = max(need + [1]) if width is None else width
        self.table = torch.full((len(k), width), -1, dtype=torch.int32)
        self.lens = torch.tensor(lens, dtype=torch.int32)
        self.k, self.v = [], []
        at = 0
        for b, n in enumerate(lens):
            self.table[b, :need[b]] = torch.from_numpy(ids[at:at + need[b]].astype(np.int32))
            pad = torch.zeros(need[b] * block, kv, d)
            kk, vv = pad.clone(), pad.clone()
            kk[:n], vv[:n] = k[b], v[b]
            slabs = pack(*(x.view(-1, 16, kv, d).permute(0, 2, 1, 3).contiguous() for x in (kk, vv)))  # [slabs, kv, 18 d]
            slabs = slabs.view(need[b], block // 16, kv, 18 * d).transpose(1, 2)
            if garbage is not None and n % 16 and need[b]:  # scales of the places behind the last token
                i, s = (n - 1) // block, (n - 1) % block // 16
                for off in (8 * d, 17 * d):
                    sc = slabs[i, :, s, off:off + d].contiguous().view(torch.half).view(kv, 16, -1)
                    sc[:, n % 16:] = garbage
                    slabs[i, :, s, off:off + d] = sc.view(kv, -1).view(torch.uint8)
                slabs[i, :, s + 1:, 8 * d:9 * d] = torch.full((d // 2,), garbage, dtype=torch.half).view(torch.uint8)
                slabs[i, :, s + 1:, 17 * d:] = torch.full((d // 2,), garbage, dtype=torch.half).view(torch.uint8)
            self.pages[self.table[b, :need[b]].long()] = slabs
            self.k.append(held(k[b]))
            self.v.append(held(v[b]))
            at += need[b]


# ---- attention ---------------------------------------------------------------------------------------

def weights(z, cfg: kint.Config):
    """Weights at z = s - M of one row's visible keys (fp64)."""
    K = cfg.Kint
    if cfg.calib == kint.CALIB_SOFTMAX:
        return z.exp()
    if cfg.calib == kint.CALIB_EXP_FP8:
        return z.exp().float().to(torch.float8_e4m3fn).double()
    if cfg.calib == kint.CALIB_EXP_BF16:
        return z.float().bfloat16().double().exp().float().bfloat16().double()
    low = z.min() if cfg.calib == kint.CALIB_MINMAX else torch.tensor(-float(cfg.tau), dtype=torch.float64)
    if -low <= 1e-12:
        return torch.ones_like(z)
    h = -low / K
    u = (z - low) / h
    r = u.floor().clamp(max=K - 1)
    if cfg.calib != kint.CALIB_FWM_RESOLVED:
        r = r.clamp(min=0)
    t = u - r
    e0, e1 = (low + r * h).exp(), (low + (r + 1) * h).exp()
    w = torch.where(t >= 0.5, e1, e0) if cfg.recon == kint.RECON_NEAREST else e0 + t * (e1 - e0)
    return torch.where(z < low, torch.zeros_like(w), w) if cfg.calib == kint.CALIB_FWM else w


def seen(p, n, window, sinks):
    """The keys of n that position p sees."""
    j = torch.arange(n)
    m = j <= p
    return m if window == 0 else m & ((j > p - window) | (j < sinks))


DELTA = 1e-5  # scores of the kernel are within this of exact ones (fp32 sums of up to 128 products of size O(1))


def attention(q, k, v, lens, new, cfg, window=0, sinks=0):
    """O [rows, heads, d] in fp64, and whether each (row, head) is free of a rounding decision within DELTA (a weight
    that jumps there).  q: fp64 rows; k, v: lists of [len, kv, d]."""
    out = torch.zeros(q.shape, dtype=torch.float64)
    safe = torch.ones(q.shape[:2], dtype=torch.bool)
    row = 0
    for b, n in enumerate(new):
        kv = k[b].shape[1]
        G = q.shape[1] // kv
        for t in range(n):
            p = lens[b] - n + t
            see = seen(p, lens[b], window, sinks)
            for h in range(q.shape[1]):
                if not see.any():
                    continue
                s = k[b][see, h // G] @ q[row, h] / math.sqrt(q.shape[2])
                z = s - s.max()
                w = weights(z, cfg)
                out[row, h] = w @ v[b][see, h // G] / w.sum()
                lo, hi = weights(torch.clamp(z - DELTA, min=z.min().item()), cfg), weights(torch.clamp(z + DELTA, max=0.0), cfg)
                safe[row, h] = bool(((hi - lo).abs() <= 10 * DELTA).all())
            row += 1
    return out, safe


# ---- rotation and blocks --------------------------------------------------------------------------------

def rotate(x, pos, table, rot, interleaved, inverse=False):
    """x [B, T, heads, d] in fp64; table fp64 [max_pos, rot / 2, 2]; pos [B, T] (-1: as it is)."""
    y = x.double().clone()
    half = rot // 2
    for b in range(x.shape[0]):
        for t in range(x.shape[1]):
            if pos[b, t] < 0:
                continue
            c, s = table[pos[b, t], :, 0].double(), table[pos[b, t], :, 1].double() * (-1 if inverse else 1)
            i = torch.arange(half)
            ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
            a, bb = x[b, t, :, ia].double(), x[b, t, :, ib].double()
            y[b, t, :, ia], y[b, t, :, ib] = a * c - bb * s, bb * c + a * s
    return y


def extend(lens, new, table, free, n_free, block, tokens):
    """Block tables and slots, one request and token at a time."""
    table = table.clone()
    width = table.shape[1]
    B = len(lens)
    taken = refused = 0
    want_sum = 0
    cu, slots, pos, req, out = [0], [], [], [], []
    for b in range(B):
        have, need_all = -(-lens[b] // block), -(-(lens[b] + new[b]) // block)
        fits = need_all <= width
        need = need_all - have if fits else 0
        want_sum += need
        ok = fits and (need == 0 or want_sum <= n_free)
        if ok:
            for i in range(need):
                table[b, have + i] = free[n_free - 1 - taken - i]
            taken += need
        else:
            refused += 1
        out.append(lens[b] + new[b] if ok else lens[b])
        for j in range(new[b]):
            p = lens[b] + j
            slots.append(int(table[b, p // block]) * block + p % block if ok else -1)
            pos.append(p)
            req.append(b)
        cu.append(cu[-1] + new[b])
    pad = [-1] * max(0, tokens - len(slots))
    return dict(lens=out, cu=cu, slots=(slots + pad)[:tokens], pos=(pos + pad)[:tokens], req=(req + pad)[:tokens],
                n_free=[n_free - taken], refused=[refused], table=table)
