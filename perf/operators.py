"""Measured cases of the serving operators: block tables, rotary positions, the 4-bit cache's
append, and attention over the 4-bit cache.

``run`` computes an operator in its plain form (elementary torch operations in 32 bits), or, where
``own`` is true, through the package's entry points.  ``exact`` gives the same outputs in 64 bits,
request by request.  All inputs come from the case and the seed alone.

A slab of the cache holds 16 keys of one kv head in 18 d bytes: K codes (8 d), K scales (d),
V codes (8 d), V scales (d); a value is s * (code - 8) + c with one (s, c) pair of halves for each
64 channels of a key.  K codes: the 32-bit word of channels 32 i + 8 t + 0..7 of key j at
j d / 2 + t d / 8 + 4 i.  V codes: keys 2 p and 2 p + 1 share the word of channels
64 gr + 8 g + 4 h + 0..3, at ((8 p + g) (d / 32) + 2 gr + h) * 4, the even key in its low half.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
CALIBS = {"minmax": 0, "fwm": 1, "softmax": 2}
RECONS = {"lerp": 0, "nearest": 1}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}


# ---- cases ------------------------------------------------------------------------------------

def listed():
    att = dict(op="attention", block=32, new=1, K=4, tau=8.0, window=0, sinks=0)
    return [
        # one user, a short answer under way: 24 heads of 64 (a 1B-scale layer), latency counts
        dict(att, name="attend_one_short", batch=1, q_heads=24, kv_heads=24, d=64, ctx_lo=333, ctx_hi=333,
             dtype="bf16", calib="softmax", recon="lerp"),
        # the GPT-2 layer's heads (12 of 64) in fp32 as it trains, eight users at ragged lengths up to 1024
        dict(att, name="attend_gpt2_fp32", batch=8, q_heads=12, kv_heads=12, d=64, ctx_lo=1, ctx_hi=1024,
             dtype="fp32", calib="fwm", recon="lerp"),
        # a full server: 64 users, grouped heads of 128, the window calibration with hard rounding
        dict(att, name="attend_batch", batch=64, q_heads=32, kv_heads=8, d=128, ctx_lo=1021, ctx_hi=8192,
             dtype="bf16", calib="fwm", recon="nearest"),
        # one user with a long document: few rows, one long axis
        dict(att, name="attend_long", batch=1, q_heads=32, kv_heads=8, d=128, ctx_lo=131071, ctx_hi=131071,
             dtype="bf16", calib="minmax", recon="lerp", K=16),
        # four drafted tokens a user, a sliding window of 1024 keys and four first tokens that stay visible
        dict(att, name="attend_window_draft", batch=32, q_heads=16, kv_heads=4, d=128, ctx_lo=0, ctx_hi=16384, new=4,
             dtype="fp16", calib="softmax", recon="lerp", window=1024, sinks=4, block=16),
        # one step's tokens of 64 users into the cache, keys rotated on the way
        dict(op="append", name="append_step", tokens=64, q_heads=32, kv_heads=8, d=128, rot=128, interleaved=False,
             dtype="bf16", block=32),
        # long prompts into the cache, heads of 64, half of each head rotated
        dict(op="append", name="append_prompt", tokens=16381, q_heads=24, kv_heads=24, d=64, rot=32, interleaved=True,
             dtype="bf16", block=16),
        # one step's queries and keys rotated
        dict(op="rope", name="rope_step", batch=64, length=1, q_heads=32, kv_heads=8, d=128, rot=128, interleaved=False,
             inverse=False, heads_first=False, dtype="bf16", scaling="bands"),
        # the gradient's way back through the rotation in a training step at the GPT-2 layer's shape (fp32)
        dict(op="rope", name="rope_train_back", batch=8, length=1024, q_heads=12, kv_heads=12, d=64, rot=64,
             interleaved=True, inverse=True, heads_first=True, dtype="fp32", scaling="none"),
        # long prompts rotated
        dict(op="rope", name="rope_prompt", batch=4, length=8191, q_heads=32, kv_heads=8, d=128, rot=96, interleaved=False,
             inverse=False, heads_first=False, dtype="bf16", scaling="linear"),
        # one step's blocks and slots for 256 users
        dict(op="blocks", name="blocks_step", batch=256, len_lo=0, len_hi=8192, new_lo=1, new_hi=1, block=32),
        # a thousand prompts and running answers admitted together
        dict(op="blocks", name="blocks_prompts", batch=1024, len_lo=0, len_hi=2048, new_lo=0, new_hi=1999, block=16),
    ]


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    n = min(max(n, lo), hi)
    return n - 1 if n == 3072 else n


def draw(rng):
    op = rng.choice(["attention", "attention", "attention", "append", "rope", "blocks"])
    if op == "blocks":
        batch, new_hi = _log(rng, 1, 2048), _log(rng, 1, 2000)
        return dict(op=op, batch=batch, len_lo=0, len_hi=_log(rng, 1, 8192), new_lo=rng.choice([0, 1]),
                    new_hi=min(new_hi, max(1, 2000000 // batch)), block=rng.choice([16, 32, 64, 128]))
    d = rng.choice([64, 128])
    kv = rng.choice([1, 2, 3, 4, 8, 12])
    group = rng.choice([1, 1, 2, 3, 4, 8])
    dtype = rng.choice(["fp32", "bf16", "bf16", "fp16"])
    if op == "append":
        return dict(op=op, tokens=_log(rng, 1, 393216 // (kv * (group + 2)) // (d // 64)), q_heads=kv * group, kv_heads=kv, d=d,
                    rot=rng.choice([0, d // 4, d // 2, d]), interleaved=rng.random() < 0.5, dtype=dtype,
                    block=rng.choice([16, 32, 64]))
    if op == "rope":
        length = _log(rng, 1, 8192)
        return dict(op=op, batch=_log(rng, 1, max(1, 650000 // (length * kv * (group + 1)))), length=length, q_heads=kv * group,
                    kv_heads=kv, d=d, rot=rng.choice([d // 4, d // 2, 3 * d // 4, d]), interleaved=rng.random() < 0.5,
                    inverse=rng.random() < 0.5, heads_first=rng.random() < 0.5, dtype=dtype,
                    scaling=rng.choice(["none", "linear", "bands"]))
    batch = _log(rng, 1, 64)
    ctx = _log(rng, 1, min(131072, max(64, 2000000 // (batch * kv * (d // 64)))))
    window = rng.choice([0, 0, 0, _log(rng, 16, 4096)])
    return dict(op=op, batch=batch, q_heads=kv * group, kv_heads=kv, d=d, ctx_lo=rng.choice([0, 1, ctx]), ctx_hi=ctx,
                new=rng.choice([1, 1, 1, 2, 4, 7]), dtype=dtype, calib=rng.choice(["softmax", "fwm", "minmax"]),
                recon="lerp" if dtype == "fp32" else rng.choice(["lerp", "nearest"]), K=rng.choice([1, 4, 8, 16, 32]),
                tau=rng.choice([6.0, 8.0]), window=window, sinks=rng.choice([0, 1, 4, 17]) if window else 0,
                block=rng.choice([16, 32, 64, 128]))


def _spread(lo, hi, n):
    """n whole numbers over [lo, hi], out of order, hi first."""
    return [lo + (hi - lo) * (((n - 1 - i) * 7919) % n if n % 7919 else n - 1 - i) // max(1, n - 1) if i else hi for i in range(n)]


def _attention_sizes(case):
    lens = _spread(case["ctx_lo"], case["ctx_hi"], case["batch"])
    new = [min(case["new"], n) for n in lens]
    return lens, new


def _visible(case, lens, new):
    """Keys that some new token of each request sees, and (row, key) pairs, summed over requests."""
    keys = pairs = 0
    for n, t in zip(lens, new):
        if not t:
            continue
        w, s = case["window"], case["sinks"]
        first = max(0, n - t - w + 1) if w else 0
        keys += n - first + min(s, first)
        for p in range(n - t, n):
            low = max(0, p - w + 1) if w else 0
            pairs += p + 1 - low + min(s, low)
    return keys, pairs


def work(case):
    op = case["op"]
    if op == "blocks":
        lens, new = _spread(case["len_lo"], case["len_hi"], case["batch"]), _spread(case["new_lo"], case["new_hi"], case["batch"])
        need = sum(-(-(n + t) // case["block"]) - -(-n // case["block"]) for n, t in zip(lens, new))
        # lens and new read, the prefix offsets and new lengths written; 16 bytes a token; 8 a block taken
        return {"bytes": 16 * case["batch"] + 16 * sum(new) + 8 * need, "flops": 0}
    size, d = BYTES[case["dtype"]], case["d"]
    if op == "rope":
        n = case["batch"] * case["length"] * (case["q_heads"] + case["kv_heads"])
        table = 4 * case["rot"] * case["length"]
        return {"bytes": 2 * n * d * size + table, "flops": 3 * n * case["rot"]}
    if op == "append":
        n, kv = case["tokens"], case["kv_heads"]
        # k, v, q read, q written, the pages written and read back as values
        return {"bytes": n * d * size * (2 * kv + 2 * case["q_heads"] + 2 * kv) + 2 * n * kv * 18 * d // 16 + 4 * case["rot"] * n,
                "flops": 10 * n * d * 2 * kv}
    lens, new = _attention_sizes(case)
    keys, pairs = _visible(case, lens, new)
    return {"bytes": keys * case["kv_heads"] * 18 * d // 16 + 2 * sum(new) * case["q_heads"] * d * size,
            "flops": 4 * pairs * case["q_heads"] * d}


# ---- inputs -----------------------------------------------------------------------------------

def _rope_table(length, rot, scaling):
    """(cos, sin) pairs [length, rot / 2, 2] in fp32, formed in 64 bits; "linear" divides positions by four, "bands"
    divides the slow channels' frequencies by eight, blends the middle ones and scales the result's magnitude."""
    i = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    freq = 10000.0 ** (-2.0 * i / max(rot, 1))
    mag = 1.0
    if scaling == "linear":
        freq = freq / 4.0
    elif scaling == "bands":
        turns = 4096.0 * freq / (2 * math.pi)
        keep = ((turns - 1.0) / 31.0).clamp(0, 1)
        freq = freq * keep + freq / 8.0 * (1 - keep)
        mag = 0.1 * math.log(8.0) + 1.0
    angle = torch.arange(length, dtype=torch.float64, device="cuda")[:, None] * freq
    return (torch.stack([angle.cos(), angle.sin()], -1) * mag).float().contiguous()


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _pages(blocks, kv, block, d, gen):
    """A filled pool: uniform codes, steps near 0.22 and centres near 0, so that values have about unit variance.
    Block 0 belongs to nobody: its scales are NaN."""
    pages = torch.randint(0, 256, (blocks, kv, block // 16, 18 * d), dtype=torch.uint8, device="cuda", generator=gen)
    for at in (8 * d, 17 * d):
        sc = torch.rand(blocks, kv, block // 16, d // 2, device="cuda", generator=gen)
        sc[..., 0::2] = 0.15 + 0.14 * sc[..., 0::2]
        sc[..., 1::2] = 0.4 * sc[..., 1::2] - 0.1
        sc[0] = float("nan")
        pages[..., at:at + d] = sc.half().view(torch.uint8)
    return pages


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    s = {"case": dict(case)}
    if op == "blocks":
        B, bs = case["batch"], case["block"]
        lens, new = _spread(case["len_lo"], case["len_hi"], B), _spread(case["new_lo"], case["new_hi"], B)
        shift = torch.randperm(B, device="cuda", generator=gen)
        s["lens"], s["new"] = _ints(lens)[shift].contiguous(), _ints(new).contiguous()
        s["tokens"] = sum(new) + 5  # a few places are left over
        width = -(-(case["len_hi"] + case["new_hi"]) // bs)
        total = B * width
        ids = torch.randperm(total, device="cuda", generator=gen).int()
        held = (s["lens"] + bs - 1) // bs
        cols = torch.arange(width, device="cuda")[None]
        s["table"] = torch.where(cols < held[:, None], ids.view(B, width), -1).int().contiguous()
        free = ids.view(B, width)[cols >= held[:, None]]
        s["free"] = torch.cat([free, torch.full((total - free.numel() + 1,), -1, dtype=torch.int32, device="cuda")])
        s["n_free"] = _ints([free.numel()])
        return s
    dtype, d, qh, kv = DTYPES[case["dtype"]], case["d"], case["q_heads"], case["kv_heads"]

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen).to(dtype)

    if op == "rope":
        B, L = case["batch"], case["length"]
        start = torch.randint(0, 64, (B, 1), device="cuda", generator=gen)
        s["pos"] = (start + torch.arange(L, device="cuda")).int().contiguous()
        s["table"] = _rope_table(L + 64, case["rot"], case["scaling"])
        if case["heads_first"]:  # gradients as attention hands them back
            s["q"], s["k"] = normal(B, qh, L, d).transpose(1, 2), normal(B, kv, L, d).transpose(1, 2)
        else:  # slices of one projection
            qkv = normal(B, L, qh + 2 * kv, d)
            s["q"], s["k"] = qkv[:, :, :qh], qkv[:, :, qh:qh + kv]
        return s
    bs = case["block"]
    if op == "append":
        n = case["tokens"]
        x = normal(n, qh + 2 * kv, d)
        x[:, qh:, 3] += 2.0  # a channel with an offset, as keys have them
        s["q"], s["k"], s["v"] = x[:, :qh], x[:, qh:qh + kv], x[:, qh + kv:]
        blocks = -(-n // bs) + 8
        s["pages"] = _pages(blocks, kv, bs, d, gen)
        slots = torch.randperm(blocks, device="cuda", generator=gen)[:, None] * bs + torch.arange(bs, device="cuda")
        s["slots"] = slots.reshape(-1)[:n].long().contiguous()
        s["slots"][n // 2] = -1 if n > 4 else s["slots"][n // 2]  # a token that found no block
        s["pos"] = torch.randint(0, 8192, (n,), device="cuda", generator=gen).int()
        s["rope"] = _rope_table(8192, case["rot"], "none") if case["rot"] else None
        return s
    lens, new = _attention_sizes(case)
    B = case["batch"]
    s["lens"] = _ints(lens)
    s["cu"] = _ints([sum(new[:i]) for i in range(B + 1)])
    width = -(-max(lens + [1]) // bs)
    held = [-(-n // bs) for n in lens]
    ids = 1 + torch.randperm(sum(held) + 3, device="cuda", generator=gen).int()
    s["table"] = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    cols = torch.arange(width, device="cuda")[None] < _ints(held)[:, None]
    s["table"][cols] = ids[:sum(held)]
    s["pages"] = _pages(sum(held) + 4, kv, bs, d, gen)
    s["q"] = normal(max(1, sum(new)), qh, d)[:sum(new)] * 1.5
    s["max_new"], s["max_len"] = max(new + [1]), max(lens + [1])
    return s


# ---- one pass -----------------------------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    if own:
        return _OWN[op](state)
    return _PLAIN[op](state)


def _own_blocks(s):
    from paper_2609_33591_gb300 import serve
    p = serve.extend_blocks(s["lens"], s["new"], s["table"], s["free"], s["n_free"], s["case"]["block"], s["tokens"])
    return {"cu": p.cu, "slots": p.slots, "pos": p.pos, "req": p.req, "lens": p.lens, "n_free": p.n_free, "refused": p.refused,
            "table": s["table"]}


def _own_rope(s):
    from paper_2609_33591_gb300 import serve
    c = s["case"]
    q, k = serve.rope(s["q"], s["k"], s["pos"], s["table"], interleaved=c["interleaved"], inverse=c["inverse"])
    return {"q": q, "k": k}


def _own_append(s):
    from paper_2609_33591_gb300 import serve
    c = s["case"]
    q = serve.append(s["k"], s["v"], s["slots"], s["pages"], q=s["q"], pos=s["pos"], table=s["rope"], interleaved=c["interleaved"])
    k, v = serve.read(s["pages"], s["slots"], dtype=s["k"].dtype)
    return {"q": q, "k": k, "v": v}


def _own_attention(s):
    from paper_2609_33591_gb300 import kint, serve
    c = s["case"]
    cfg = kint.Config(Kint=c["K"], calib=CALIBS[c["calib"]], tau=c["tau"], recon=RECONS[c["recon"]])
    return serve.attention(s["q"], s["pages"], s["table"], s["lens"], s["cu"], cfg, window=c["window"], sinks=c["sinks"],
                           max_new=s["max_new"], max_len=s["max_len"])


def _plain_blocks(s):
    lens, new, table, free, bs = s["lens"].long(), s["new"].long(), s["table"], s["free"], s["case"]["block"]
    B, width = table.shape
    end = lens + new
    held, want = (lens + bs - 1) // bs, (end + bs - 1) // bs
    fits = want <= width
    need = torch.where(fits, want - held, 0)
    last = need.cumsum(0)
    ok = fits & ((need == 0) | (last <= s["n_free"].long()))
    got = torch.where(ok, need, 0)
    first = last - need
    cu = torch.cat([torch.zeros_like(end[:1]), new.cumsum(0)])
    cols = torch.arange(width, device=table.device)[None]
    taken = (cols >= held[:, None]) & (cols < (held + got)[:, None])
    at = s["n_free"].long() - 1 - (first[:, None] + cols - held[:, None])
    table = torch.where(taken, free[at.clamp(0, free.numel() - 1)], table)
    i = torch.arange(s["tokens"], device=table.device)
    req = torch.searchsorted(cu[1:], i, right=True)
    live = req < B
    r = req.clamp(max=B - 1)
    pos = lens[r] + i - cu[r]
    block = table[r, (pos // bs).clamp(0, width - 1)].long()
    slots = torch.where(live & ok[r], block * bs + pos % bs, -1)
    return {"cu": cu.int(), "slots": slots, "pos": torch.where(live, pos, -1).int(), "req": torch.where(live, req, -1).int(),
            "lens": torch.where(ok, end, lens).int(), "n_free": (s["n_free"] - got.sum()).int(),
            "refused": (~ok).sum().int().reshape(1), "table": table}


def _turn(x, c, sn, rot, interleaved):
    """The rotation of x [..., heads, d] in 32 bits, c and sn broadcast over the heads."""
    y = x.float()
    if interleaved:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        return torch.cat([torch.stack([a * c - b * sn, b * c + a * sn], -1).flatten(-2), y[..., rot:]], -1)
    a, b = y[..., :rot // 2], y[..., rot // 2:rot]
    return torch.cat([a * c - b * sn, b * c + a * sn, y[..., rot:]], -1)


def _plain_rope(s):
    c = s["case"]
    cs = s["table"][s["pos"].long()][:, :, None]
    cos, sin = cs[..., 0], cs[..., 1] * (-1.0 if c["inverse"] else 1.0)
    return {n: _turn(s[n], cos, sin, c["rot"], c["interleaved"]).to(s[n].dtype) for n in ("q", "k")}


def _held(x):
    """What 4 bits keep of x [..., d] (32 bits in, 32 bits out)."""
    g = x.unflatten(-1, (-1, 64))
    lo, hi = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    step = ((hi - lo) * (1.0 / 15.0)).half().float()
    mid = (lo + 8.0 * step).half().float()
    inv = torch.where(step > 0, 1.0 / step, torch.zeros_like(step))
    code = ((g - mid) * inv).round().clamp(-8, 7)
    return (step * code + mid).flatten(-2)


def _plain_append(s):
    c = s["case"]
    q, k = s["q"].float(), s["k"].float()
    if c["rot"]:
        cs = s["rope"][s["pos"].long()][:, None]
        q, k = (_turn(x, cs[..., 0], cs[..., 1], c["rot"], c["interleaved"]) for x in (s["q"], s["k"]))
    live = (s["slots"] >= 0)[:, None, None]
    dt = s["k"].dtype
    return {"q": q.to(dt), "k": torch.where(live, _held(k), 0.0).to(dt), "v": torch.where(live, _held(s["v"].float()), 0.0).to(dt)}


def _values(slabs, d):
    """K and V [..., 16 keys, d] in fp32 of slabs [..., 18 d] bytes."""
    def nibbles(b):
        return torch.stack([b & 15, b >> 4], -1)

    def pairs(b):
        return b.contiguous().view(torch.float16).float().unflatten(-1, (16, d // 64, 2))

    lead = slabs.dim() - 1
    lay = tuple(range(lead))
    k = nibbles(slabs[..., :8 * d].unflatten(-1, (16, 4, d // 32, 4)))  # key, t, i, byte, nibble
    k = k.permute(*lay, lead, lead + 2, lead + 1, lead + 3, lead + 4).flatten(lead + 1).float() - 8.0
    v = nibbles(slabs[..., 9 * d:17 * d].unflatten(-1, (8, 8, d // 64, 2, 2, 2)))  # pair, g, gr, h, parity, byte, nibble
    v = v.permute(*lay, lead, lead + 4, lead + 2, lead + 1, lead + 3, lead + 5, lead + 6).flatten(lead, lead + 1)
    v = v.flatten(lead + 1).float() - 8.0
    ks, vs = pairs(slabs[..., 8 * d:9 * d]), pairs(slabs[..., 17 * d:])
    k = k.unflatten(-1, (-1, 64)) * ks[..., :1] + ks[..., 1:]
    v = v.unflatten(-1, (-1, 64)) * vs[..., :1] + vs[..., 1:]
    return k.flatten(-2), v.flatten(-2)


def _weights(sc, seen, c):
    """Unnormalised weights of scores sc, zero where not seen."""
    top = torch.where(seen, sc, -math.inf).amax(-1, keepdim=True)
    z = torch.where(seen, sc - top, 0.0)
    if c["calib"] == "softmax":
        return torch.where(seen, z.exp(), 0.0)
    K = c["K"]
    if c["calib"] == "fwm":
        low, width = -c["tau"], c["tau"] / K
        flat = torch.zeros_like(top, dtype=torch.bool)
    else:
        low = torch.where(seen, z, 0.0).amin(-1, keepdim=True)
        flat = low >= -1e-12
        width = torch.where(flat, 1.0, -low / K)
    u = (z - low) / width
    r = u.clamp(0, K).floor().clamp(max=K - 1)
    t = u.clamp(0, K) - r
    if c["recon"] == "nearest":
        w = (low + (r + (t >= 0.5).float()) * width).exp()
    else:
        e = (low + r * width).exp()
        w = e + t * ((low + (r + 1) * width).exp() - e)
    if c["calib"] == "fwm":
        w = torch.where(u < 0, 0.0, w)
    return torch.where(seen, torch.where(flat, 1.0, w), 0.0)


def _plain_attention(s):
    c, q = s["case"], s["q"]
    d, kv, bs = c["d"], c["kv_heads"], c["block"]
    B, width = s["table"].shape
    new = (s["cu"][1:] - s["cu"][:-1]).long()
    slabs = s["pages"][s["table"].clamp(min=0).long()]  # [B, blocks, kv, slabs, bytes]
    keys = torch.arange(width * bs, device=q.device)
    there = (keys[None] < s["lens"].long()[:, None])[:, None, :, None]
    k, v = (x.permute(0, 2, 1, 3, 4, 5).flatten(2, 4) for x in _values(slabs, d))  # [B, kv, keys, d]
    k, v = torch.where(there, k, 0.0), torch.where(there, v, 0.0)
    t = torch.arange(s["max_new"], device=q.device)
    rows = (s["cu"][:-1].long()[:, None] + t).clamp(max=max(0, q.shape[0] - 1))
    live = t[None] < new[:, None]
    p = (s["lens"].long() - new)[:, None] + t  # positions of the new tokens
    x = q.float()[rows].unflatten(2, (kv, -1)).permute(0, 2, 1, 3, 4).flatten(2, 3)  # [B, kv, new * group, d]
    sc = torch.matmul(x, k.transpose(2, 3)) / math.sqrt(d)
    seen = (keys <= p[..., None]) & live[..., None]
    if c["window"]:
        seen &= (keys > p[..., None] - c["window"]) | (keys < c["sinks"])
    seen = seen[:, None, :, None].expand(-1, -1, -1, c["q_heads"] // kv, -1).flatten(2, 3)
    w = _weights(sc, seen, c)
    total = w.sum(-1, keepdim=True)
    o = torch.matmul(w, v) / torch.where(total > 0, total, 1.0)
    o = o.unflatten(2, (s["max_new"], -1)).permute(0, 2, 1, 3, 4).flatten(2, 3)  # [B, new, heads, d]
    i = torch.arange(q.shape[0], device=q.device)
    req = torch.searchsorted(s["cu"][1:].contiguous(), i, right=True)
    return o[req, i - s["cu"].long()[req]].to(q.dtype)


_OWN = {"blocks": _own_blocks, "rope": _own_rope, "append": _own_append, "attention": _own_attention}
_PLAIN = {"blocks": _plain_blocks, "rope": _plain_rope, "append": _plain_append, "attention": _plain_attention}


# ---- the definitions in 64 bits -----------------------------------------------------------------

def exact(case, seed):
    if case["op"] == "blocks":
        return None  # whole numbers
    s = prepare(case, seed)
    if case["op"] == "attention":
        return _exact_attention(s)
    table = s["table"] if case["op"] == "rope" else s["rope"]

    def spin(x, inverse=False):
        """The pair (a, b) as the complex number a + i b, times c + i s."""
        x = x.double().clone()
        if table is None:
            return x
        half = case["rot"] // 2
        ch = torch.arange(half, device=x.device)
        a, b = (2 * ch, 2 * ch + 1) if case["interleaved"] else (ch, ch + half)
        turn = torch.view_as_complex(table.double()[s["pos"].long()]).unsqueeze(-2)
        z = torch.complex(x[..., a], x[..., b]) * (turn.conj() if inverse else turn)
        x[..., a], x[..., b] = z.real, z.imag
        return x

    if case["op"] == "rope":
        return {"q": spin(s["q"], case["inverse"]), "k": spin(s["k"], case["inverse"])}

    def kept(x):
        out = torch.zeros_like(x)
        for g in range(0, case["d"], 64):
            part = x[..., g:g + 64]
            least, most = part.min(-1, keepdim=True).values, part.max(-1, keepdim=True).values
            step = ((most - least) / 15).half().double()
            mid = (least + 8 * step).half().double()
            out[..., g:g + 64] = mid + step * torch.clamp(torch.round((part - mid) / step.clamp(min=1e-30)), -8, 7)
        out[s["slots"] < 0] = 0
        return out

    return {"q": spin(s["q"]), "k": kept(spin(s["k"])), "v": kept(s["v"].double())}


def _exact_attention(s):
    c = s["case"]
    d, kv, bs = c["d"], c["kv_heads"], c["block"]
    G = c["q_heads"] // kv
    ch = torch.arange(d, device="cuda")
    key = torch.arange(16, device="cuda")[:, None]
    # byte and nibble of every (key, channel) of a slab
    kb = key * (d // 2) + (ch // 8 % 4) * (d // 8) + 4 * (ch // 32) + ch % 8 // 2
    vb = 9 * d + ((key // 2 * 8 + ch // 8 % 8) * (d // 32) + 2 * (ch // 64) + ch // 4 % 2) * 4 + 2 * (key % 2) + ch % 4 // 2
    gb = (key * (d // 64) + ch // 64) * 4

    def decode(slabs, at, scales):
        code = (slabs[..., at] >> (4 * (ch % 2)).to(torch.uint8)) & 15
        sc = torch.stack([slabs[..., scales + gb + i] for i in range(4)], -1).view(torch.float16).double()
        return (code.double() - 8) * sc[..., 0] + sc[..., 1]

    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lens, cu, table = s["lens"].tolist(), s["cu"].tolist(), s["table"]
    for b in range(c["batch"]):
        T, n = lens[b], cu[b + 1] - cu[b]
        if not n:
            continue
        slabs = s["pages"][table[b, :-(-T // bs)].long()].transpose(0, 1).flatten(1, 2)  # [kv, slabs, bytes]
        k = decode(slabs, kb, 8 * d).flatten(1, 2)[:, :T]
        v = decode(slabs, vb, 17 * d).flatten(1, 2)[:, :T]
        j = torch.arange(T, device="cuda")
        for t in range(n):
            p = T - n + t
            see = j <= p
            if c["window"]:
                see &= (p - j < c["window"]) | (j < c["sinks"])
            see = see.nonzero()[:, 0]
            x = s["q"][cu[b] + t].double().view(kv, G, d)
            z = torch.einsum("hgd,hkd->hgk", x, k[:, see]) * d ** -0.5
            z = z - z.amax(-1, keepdim=True)
            out[cu[b] + t] = torch.einsum("hgk,hkd->hgd", _exact_probabilities(z, c), v[:, see]).reshape(-1, d)
    return out


def _exact_probabilities(z, c):
    """z = s - max s over the visible keys."""
    if c["calib"] == "softmax":
        return torch.softmax(z, -1)
    K = c["K"]
    span = torch.full_like(z[..., :1], c["tau"]) if c["calib"] == "fwm" else -z.amin(-1, keepdim=True)
    h = span / K
    grid = torch.exp(-span + torch.arange(K + 1, device=z.device, dtype=z.dtype) * h)
    x = torch.where(h > 0, (z + span) / h, torch.zeros_like(z)).clamp(0, K)
    if c["recon"] == "nearest":
        w = torch.gather(grid, -1, torch.floor(x + 0.5).long())
    else:
        r = x.long().clamp(max=K - 1)
        w = torch.gather(grid, -1, r) * (1 - (x - r)) + torch.gather(grid, -1, r + 1) * (x - r)
    w = torch.where(z < -span, torch.zeros_like(w), w) if c["calib"] == "fwm" else torch.where(span <= 1e-12, torch.ones_like(w), w)
    return w / w.sum(-1, keepdim=True)
