"""GPU: the serving operators against plain 64-bit forms (tests/serve_ref.py).

Tolerances, set from the arithmetic before the first run:
- attention: a row's output is a convex combination of its values, so errors are measured against the largest value V the
  row sees.  Scores are fp32 sums (error below 1e-5, serve_ref.DELTA), which moves a weight by at most 1e-5 of itself for
  the exponential and by at most 10 DELTA where no rounding decision lies within DELTA; weights times scales are split
  to 2^-17 (2^-24 for fp32 outputs).  All told 3e-5 V, and half a unit of the output's type on top.  The rare forms keep
  decisions smaller than 10 DELTA: 2e-4 V.
- rotation: two products and a sum in fp32, 3 * 2^-24 of |a| + |b|, and half a unit of the type.
- the cache, block tables: equal.
"""
import math

import numpy as np
import pytest
import torch

from paper_2609_33591_gb300 import kint, serve
from tests import serve_ref as ref

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
HALF_UNIT = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}  # of 24, 8 and 11 significant bits
SOFT, FWM, MM = kint.CALIB_SOFTMAX, kint.CALIB_FWM, kint.CALIB_MINMAX
LERP, NEAR = kint.RECON_LERP, kint.RECON_NEAREST


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    serve.load()


@pytest.fixture(autouse=True)
def _clean():
    kint.kint_get_status()
    yield
    assert kint.kint_get_status() == (0, 0)


def gpu(x, dtype=None):
    return x.to("cuda", dtype)


def ints(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


def filled(lens, kv, d, block, seed, **kw):
    g = torch.Generator().manual_seed(seed)
    k = [torch.randn(n, kv, d, generator=g) for n in lens]
    v = [torch.randn(n, kv, d, generator=g) for n in lens]
    return ref.Pool(k, v, block, d, kv, seed=seed, **kw)


def run_attention(pool, q, new, cfg, **kw):
    cu = ints(np.concatenate([[0], np.cumsum(new)]).tolist())
    return serve.attention(q, gpu(pool.pages), gpu(pool.table), gpu(pool.lens), cu, cfg, **kw)


def check_attention(lens, new, heads, kv, d, cfg, dtype, *, block=32, window=0, sinks=0, seed=0, rare=False, scale=1.0, **kw):
    pool = filled(lens, kv, d, block, seed)
    g = torch.Generator().manual_seed(seed + 1)
    q = (scale * torch.randn(sum(new), heads, d, generator=g)).to(dtype)
    o = run_attention(pool, gpu(q), new, cfg, window=window, sinks=sinks, max_new=max(new + [1]), **kw)
    assert o.dtype == dtype and o.shape == q.shape
    want, safe = ref.attention(q.double(), pool.k, pool.v, lens, new, cfg, window, sinks)
    top = max([float(x.abs().max()) for x in pool.v if x.numel()] + [0.0])
    err = (o.cpu().double() - want).abs()
    tol = HALF_UNIT[dtype] * want.abs() + (2e-4 if rare else 3e-5) * top
    bad = (err > tol).any(-1) & safe
    assert not bad.any(), (err[bad].max(), bad.sum(), bad.numel())
    assert safe.float().mean() > 0.4
    return pool, q, o


LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 300]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("calib,recon", [(SOFT, LERP), (FWM, LERP), (FWM, NEAR), (MM, LERP), (MM, NEAR)])
def test_single_tokens_at_every_kind_of_length(dtype, d, calib, recon):
    cfg = kint.Config(Kint=4, calib=calib, tau=3.0, recon=recon)
    check_attention(LENS, [min(1, n) for n in LENS], 4, 2, d, cfg, dtype, seed=1)


@pytest.mark.parametrize("heads,kv,new", [(1, 1, 1), (5, 1, 1), (8, 1, 1), (9, 1, 1), (16, 2, 1), (12, 12, 1), (6, 2, 3),
                                          (8, 2, 7), (24, 1, 2), (3, 3, 20)])
@pytest.mark.parametrize("d,dtype", [(64, F32), (128, BF16)])
def test_head_layouts_and_several_new_tokens(heads, kv, new, d, dtype):
    lens = [20, 33, 70]
    cfg = kint.Config(Kint=8, calib=FWM, tau=6.0, recon=LERP)
    check_attention(lens, [new, max(1, new - 1), new], heads, kv, d, cfg, dtype, seed=2)


@pytest.mark.parametrize("calib", [kint.CALIB_FWM_RESOLVED, kint.CALIB_EXP_FP8, kint.CALIB_EXP_BF16])
@pytest.mark.parametrize("recon", [LERP, NEAR])
def test_rare_weights(calib, recon):
    cfg = kint.Config(Kint=4, calib=calib, tau=3.0, recon=recon)
    for d, dtype in ((64, F32), (128, BF16)):
        check_attention([7, 30, 45], [1, 2, 1], 4, 2, d, cfg, dtype, seed=3, rare=True)


@pytest.mark.parametrize("K", [1, 2, 16, 32, 64])
@pytest.mark.parametrize("calib", [FWM, MM])
def test_intervals(K, calib):
    check_attention([129, 64], [1, 1], 8, 2, 128, kint.Config(Kint=K, calib=calib, tau=8.0, recon=LERP), F32, seed=4)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 0), (17, 4), (40, 16), (40, 17), (100, 64), (33, 1000), (1000, 4)])
@pytest.mark.parametrize("new", [1, 5])
def test_window_and_first_tokens(window, sinks, new):
    lens = [1, 5, 40, 57, 200, 333]
    cfg = kint.Config(Kint=4, calib=SOFT)
    check_attention(lens, [min(new, n) for n in lens], 4, 2, 64, cfg, F32, window=window, sinks=sinks, block=16, seed=5)
    check_attention(lens, [min(new, n) for n in lens], 4, 1, 128, kint.Config(Kint=4, calib=MM), BF16, window=window, sinks=sinks,
                    block=64, seed=6)


@pytest.mark.parametrize("block", [16, 32, 64, 128, 512])
def test_block_sizes(block):
    check_attention([block - 1, block, block + 1, 3 * block + 5], [1] * 4, 2, 2, 64, kint.Config(calib=FWM, recon=LERP), F32,
                    block=block, seed=7)


@pytest.mark.parametrize("calib", [SOFT, FWM, MM])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_long_context_joined_from_many_parts(calib, dtype):
    """One short and one long request: ranges of 8 to 64 slabs, joined in order."""
    check_attention([9001, 40], [1, 1], 4, 1, 64, kint.Config(Kint=16, calib=calib, tau=8.0), dtype, block=128, seed=8, scale=2.0)


@pytest.mark.parametrize("heads,new,d", [(2, 1, 128), (8, 1, 64), (16, 1, 128), (5, 3, 64)])
def test_few_units_with_long_lists(heads, new, d):
    """One request on many thread blocks at once (a cooperative launch): tiles of 4, 8 and 16 rows, an empty request beside it."""
    cfg = kint.Config(Kint=8, calib=MM, recon=LERP)
    check_attention([4100, 0, 3], [new, 0, min(new, 3)], heads, 1, d, cfg, F32, block=64, seed=15)


@pytest.mark.parametrize("blocks", range(1, 9))
@pytest.mark.parametrize("heads,d,dtype", [(4, 64, F32), (7, 128, BF16), (13, 64, BF16)])
def test_every_number_of_blocks_a_unit(blocks, heads, d, dtype):
    """Eight slabs a thread block: clusters of one to eight; a request too short for all of them and an empty one beside it."""
    cfg = kint.Config(Kint=8, calib=MM, recon=LERP)
    check_attention([128 * blocks + 5, 19, 0], [1, 1, 0], heads, 1, d, cfg, dtype, seed=17 + blocks)


@pytest.mark.parametrize("requests", [110, 128, 129])
@pytest.mark.parametrize("lo", [0, 600])
def test_more_blocks_than_run_at_once(requests, lo):
    """Many ragged requests (up to 128: the longest first) with equal lengths and empty ones among them, and nearly equal ones."""
    lens = [lo + 50 * (i * 37 % 29 * (700 - lo) // 29 // 50) for i in range(requests)]
    check_attention(lens, [min(n, 1) for n in lens], 6, 6, 64, kint.Config(Kint=4, calib=FWM, recon=LERP), BF16, seed=30)


def test_many_tiles_with_long_lists():
    """Scores too many for shared memory: two launches, joined by the last block of each tile."""
    check_attention([8500], [150], 16, 1, 64, kint.Config(calib=SOFT), F32, block=256, seed=16)


def test_rows_that_see_nothing_are_zero():
    """More new tokens than cached ones (the first rows lie before position 0), and an empty request between others."""
    cfg = kint.Config(Kint=4, calib=MM)
    _, _, o = check_attention([2, 0, 3], [4, 2, 1], 4, 2, 64, cfg, F32, seed=9)
    assert (o[:2] == 0).all() and (o[4:6] == 0).all() and (o[2:4] != 0).any()


@pytest.mark.parametrize("garbage", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("calib", [SOFT, FWM, MM, kint.CALIB_EXP_BF16])
def test_what_is_not_seen_does_not_matter(garbage, calib):
    """Scales of the places behind a request's last token, and whole unowned blocks, hold NaN or infinities: same bits."""
    lens, new = [3, 17, 50, 0], [1, 2, 1, 0]
    cfg = kint.Config(Kint=4, calib=calib, tau=3.0)
    q = torch.randn(sum(new), 8, 64, generator=torch.Generator().manual_seed(1)).cuda()
    outs = []
    for g in (None, garbage):
        pool = filled(lens, 4, 64, 64, 10, garbage=g, width=4)
        outs.append(run_attention(pool, q, new, cfg, window=20, sinks=2, max_new=2))
    assert torch.isfinite(outs[1]).all() and torch.equal(*outs)


def test_a_nan_that_is_seen_shows():
    pool = filled([40, 40], 2, 64, 32, 11)
    k = torch.randn(40, 2, 64)
    k[17, 1, 5] = math.inf
    pages, slots = gpu(pool.pages), (gpu(pool.table[1]).long()[:, None] * 32 + torch.arange(32, device="cuda")).flatten()[:40]
    serve.append(gpu(k), gpu(k), slots, pages)
    q = torch.randn(2, 4, 64, device="cuda")
    for calib in (SOFT, FWM, MM):
        o = serve.attention(q, pages, gpu(pool.table), gpu(pool.lens), ints([0, 1, 2]), kint.Config(calib=calib))
        assert torch.isfinite(o[0]).all() and torch.isfinite(o[1, :2]).all() and torch.isnan(o[1, 2:]).all()


@pytest.mark.parametrize("dtype,scale", [(F32, 1e-30), (F32, 1e4), (BF16, 1e-20), (BF16, 3e3)])
def test_scale_of_the_queries(dtype, scale):
    """Tiny queries (equal weights) and huge ones (one key takes all)."""
    check_attention([50], [1], 2, 1, 64, kint.Config(calib=SOFT), F32, seed=12, scale=1e-30)
    pool = filled([50], 1, 64, 32, 12)
    q = (scale * torch.randn(1, 2, 64, generator=torch.Generator().manual_seed(0))).to(dtype)
    o = run_attention(pool, gpu(q), [1], kint.Config(calib=SOFT), max_new=1).cpu().double()
    s = torch.einsum("hd,kd->hk", q[0].double(), pool.k[0][:, 0]) / 8
    want = torch.softmax(s, -1) @ pool.v[0][:, 0]
    # scores of size S carry relative error 2^-20 (sums of 64 products), so weights e^(2 S 2^-20)
    slack = min(1.0, 2 * float(s.abs().max()) * 2.0 ** -20 + 3e-5)
    assert ((o[0] - want).abs() <= HALF_UNIT[dtype] * want.abs() + slack * pool.v[0].abs().max()).all()
    z = torch.zeros(1, 2, 64, dtype=dtype, device="cuda")
    o = run_attention(pool, z, [1], kint.Config(calib=MM), max_new=1).cpu().double()
    assert ((o[0] - pool.v[0][:, 0].mean(0)).abs() <= HALF_UNIT[dtype] * 4 + 1e-4).all()


def test_strides_layers_streams_and_graphs():
    """q a slice of a projection, out a strided view, pages one layer of several, table a slice of a wider one, a side
    stream, a captured graph: the same bits as the plain call, and run to run."""
    lens, new, H, kv, d = [100, 37, 9], [2, 1, 3], 8, 2, 128
    cfg = kint.Config(Kint=8, calib=FWM, tau=8.0, recon=NEAR)
    pool = filled(lens, kv, d, 32, 13)
    pages, table, lens_g, cu = gpu(pool.pages), gpu(pool.table), gpu(pool.lens), ints([0, 2, 3, 6])
    q = torch.randn(6, H, d, device="cuda").bfloat16()
    kw = dict(max_new=3, max_len=128)
    want = serve.attention(q, pages, table, lens_g, cu, cfg, **kw)
    assert torch.equal(want, serve.attention(q, pages, table, lens_g, cu, cfg, **kw))
    wide = torch.randn(6, H + 3, d + 8, device="cuda").bfloat16()
    wide[:, 1:H + 1, 3:d + 3] = q  # rows at odd addresses
    out = torch.zeros(6, H, 2 * d, device="cuda").bfloat16()
    layers = torch.randint(0, 256, (3, *pages.shape), dtype=torch.uint8, device="cuda").transpose(0, 1).contiguous()
    layers[:, 1] = pages
    tables = torch.full((3, table.size(1) + 5), -7, dtype=torch.int32, device="cuda")
    tables[:, 2:2 + table.size(1)] = table
    got = serve.attention(wide[:, 1:H + 1, 3:d + 3], layers[:, 1], tables[:, 2:2 + table.size(1)], lens_g, cu, cfg,
                          out=out[:, :, 5:d + 5], **kw)
    assert torch.equal(got, want) and (out[:, :, :5] == 0).all() and (out[:, :, d + 5:] == 0).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = serve.attention(q, pages, table, lens_g, cu, cfg, **kw)
    side.synchronize()
    assert torch.equal(other, want)
    other = serve.attention(q, pages, table, lens_g, cu, cfg, stream=side, **kw)
    side.synchronize()
    assert torch.equal(other, want)
    ws = serve.attention_workspace(3, H, kv, d, **kw)
    res = torch.zeros_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        serve.attention(q, pages, table, lens_g, cu, cfg, out=res, ws=ws, **kw)
    for _ in range(2):
        res.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(res, want)


@pytest.mark.parametrize("lens,new,heads", [([6000], [1], 4), ([8300], [130], 16)])
def test_captured_long_lists(lens, new, heads):
    """The cooperative launch and the two launches in a captured graph: the plain call's bits, replay after replay."""
    pool = filled(lens, 1, 64, 128, 17)
    pages, table, lens_g, cu = gpu(pool.pages), gpu(pool.table), gpu(pool.lens), ints([0] + new)
    q, cfg = torch.randn(new[0], heads, 64, device="cuda").bfloat16(), kint.Config(calib=FWM, recon=LERP)
    kw = dict(max_new=new[0], max_len=lens[0])
    want = serve.attention(q, pages, table, lens_g, cu, cfg, **kw)
    ws = serve.attention_workspace(1, heads, 1, 64, **kw)
    res = torch.zeros_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        serve.attention(q, pages, table, lens_g, cu, cfg, out=res, ws=ws, **kw)
    for _ in range(2):
        res.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(res, want)


def test_offsets_past_32_bits():
    """A pool of over 4 GiB, its blocks at the far end."""
    kv, d, block = 8, 128, 512
    size = kv * block // 16 * 18 * d
    blocks = (1 << 32) // size + 40
    pages = torch.empty(blocks, kv, block // 16, 18 * d, dtype=torch.uint8, device="cuda")
    n = 700
    table = ints([[blocks - 1, blocks - 3]])
    slots = (table.long().flatten()[:, None] * block + torch.arange(block, device="cuda")).flatten()[:n]
    k, v = torch.randn(n, kv, d, device="cuda"), torch.randn(n, kv, d, device="cuda")
    serve.append(k, v, slots, pages)
    got_k, got_v = serve.read(pages, slots)
    assert torch.equal(got_k.cpu().double(), ref.held(k.cpu()).float().double())
    q = torch.randn(1, kv, d, device="cuda")
    o = serve.attention(q, pages, table, ints([n]), ints([0, 1]), kint.Config(calib=SOFT))
    s = torch.einsum("hd,khd->hk", q[0].double(), got_k.double()) / math.sqrt(d)
    want = torch.einsum("hk,khd->hd", torch.softmax(s, -1), got_v.double())
    assert ((o[0].double() - want).abs() <= 3e-5 * got_v.abs().max()).all()


def expect_flag():
    rc, detail = kint.kint_get_status()
    assert rc == -6 and detail == 8, (rc, detail)


def test_index_data_out_of_range_is_flagged_not_followed():
    pool = filled([40], 2, 64, 32, 14)
    pages, cfg = gpu(pool.pages), kint.Config(calib=SOFT)
    q = torch.randn(1, 2, 64, device="cuda")
    for bad in (-1, pages.size(0), 1 << 30):
        t = gpu(pool.table).clone()
        t[0, 1] = bad
        serve.attention(q, pages, t, gpu(pool.lens), ints([0, 1]), cfg)
        expect_flag()
    serve.attention(q, pages, gpu(pool.table), ints([70]), ints([0, 1]), cfg)  # a length past the table
    expect_flag()
    for cu in ([-1, 0], [0, 2], [1, 2], [3, 2]):  # rows that q does not have
        out = torch.full_like(q, 7.0)
        serve.attention(q, pages, gpu(pool.table), gpu(pool.lens), ints(cu), cfg, max_new=4, out=out)
        expect_flag()
        assert (out == 7.0).all()
    before = pages.clone()
    x = torch.randn(3, 2, 64, device="cuda")
    serve.append(x, x, ints([-1, -2, pages.size(0) * 32], torch.int64), pages)
    expect_flag()
    assert torch.equal(before, pages)
    k, v = serve.read(pages, ints([-1, -2, pages.size(0) * 32], torch.int64))
    expect_flag()
    assert not k.any() and not v.any()
    table = serve.rope_table(8, 64)
    y, _ = serve.rope(x[None], None, ints([3, 8, -2]), table)
    expect_flag()
    assert torch.equal(y[0, 1:], x[1:]) and not torch.equal(y[0, 0], x[0])


# ---- rotation ---------------------------------------------------------------------------------------

def check_rope(dtype, B, T, hq, hk, d, rot, interleaved, inverse=False, view=lambda x: x, **kw):
    table = serve.rope_table(T + 9, rot, **kw)
    g = torch.Generator().manual_seed(d + rot)
    q, k = (view(gpu(torch.randn(B, T, h, d, generator=g), dtype)) for h in (hq, max(hk, 1)))
    k = k if hk else None
    pos = gpu(torch.randint(0, T + 9, (B, T), generator=g).int())
    pos[0, 0] = -1
    got = serve.rope(q, k, pos, table, interleaved=interleaved, inverse=inverse)
    for x, y in ((q, got[0]), (k, got[1])):
        if x is None:
            assert y is None
            continue
        want = ref.rotate(x.cpu(), pos.cpu(), table.cpu(), rot, interleaved, inverse)
        size = x.cpu().double().abs().amax(-1, keepdim=True) * 2
        assert ((y.cpu().double() - want).abs() <= HALF_UNIT[dtype] * want.abs() + 3 * 2.0 ** -24 * size + 2.0 ** -25 * 0).all()
        assert torch.equal(y[..., rot:], x[..., rot:]) and torch.equal(y[0, 0], x[0, 0])


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 64), (64, 32), (128, 96), (128, 2), (80, 20), (2, 2), (256, 256), (66, 34)])
def test_rope(dtype, interleaved, d, rot):
    check_rope(dtype, 2, 5, 3, 2, d, rot, interleaved)
    check_rope(dtype, 1, 1, 1, 0, d, rot, interleaved, inverse=True)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_of_strided_and_odd_views(interleaved):
    def odd(x):
        y = torch.zeros(*x.shape[:-1], x.shape[-1] + 3, dtype=x.dtype, device=x.device)
        y[..., 1:-2] = x
        return y[..., 1:-2]
    check_rope(BF16, 2, 7, 4, 2, 64, 64, interleaved, view=odd)
    check_rope(F32, 2, 7, 4, 2, 64, 32, interleaved, view=lambda x: x.transpose(1, 2).contiguous().transpose(1, 2))
    check_rope(F16, 3, 33, 40, 8, 128, 128, interleaved, scaling="bands", factor=4.0)


def test_rope_in_place_and_there_and_back():
    table = serve.rope_table(50, 64)
    pos = torch.arange(50, dtype=torch.int32, device="cuda")
    for interleaved in (False, True):
        q, k = torch.randn(2, 50, 4, 64, device="cuda"), torch.randn(2, 50, 2, 64, device="cuda")
        a, b = serve.rope(q, k, pos, table, interleaved=interleaved)
        x, y = q.clone(), k.clone()
        serve.rope(x, y, pos, table, interleaved=interleaved, out=(x, y))
        assert torch.equal(x, a) and torch.equal(y, b)
        serve.rope(x, y, pos, table, interleaved=interleaved, inverse=True, out=(x, y))
        # cos^2 + sin^2 of fp32 numbers, and two roundings each way
        assert ((x - q).abs() <= 8 * 2.0 ** -24 * 2 * q.abs().amax(-1, keepdim=True)).all()


def test_rope_table_against_64_bits():
    for kw in ({}, dict(scaling="linear", factor=4.0), dict(scaling="base", factor=2.0), dict(scaling="bands", factor=8.0)):
        freq, mag = serve.rope_frequencies(48, 5000.0, **kw)
        t = serve.rope_table(3000, 48, 5000.0, **kw).cpu().double().numpy()
        a = np.arange(3000)[:, None] * np.array(freq)
        # fp64 angles up to 3000 (2^-53 * 3000 of error), rounded to fp32
        assert np.abs(t[..., 0] - mag * np.cos(a)).max() <= mag * 2.0 ** -24
        assert np.abs(t[..., 1] - mag * np.sin(a)).max() <= mag * 2.0 ** -24


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_gradient_against_the_formula_and_differences(interleaved):
    """L = sum c * rotary(x): the gradient is the transposed rotation of c, and, the map being linear, differences of
    any step give it too (in fp32: two rounded sums of 2 * 6 * 3 * 64 terms)."""
    table = serve.rope_table(40, 48)
    pos = torch.randint(0, 40, (2, 6), device="cuda").int()
    q, k = torch.randn(2, 6, 3, 64, device="cuda", requires_grad=True), torch.randn(2, 6, 1, 64, device="cuda", requires_grad=True)
    cq, ck = torch.randn(2, 6, 3, 64, device="cuda"), torch.randn(2, 6, 1, 64, device="cuda")
    a, b = serve.rotary(q, k, pos, table, interleaved)
    ((a * cq).sum() + (b * ck).sum()).backward()
    for x, c in ((q, cq), (k, ck)):
        want = ref.rotate(c.cpu(), pos.cpu(), table.cpu(), 48, interleaved, inverse=True)
        assert ((x.grad.cpu().double() - want).abs() <= 2.0 ** -22 * c.abs().max().item()).all()
    d = torch.randn_like(q)
    with torch.no_grad():
        hi, lo = (serve.rotary(q + s * d, k, pos, table, interleaved)[0].double() for s in (0.5, -0.5))
    diff, grad = ((hi - lo) * cq.double()).sum().item(), (q.grad.double() * d.double()).sum().item()
    assert abs(diff - grad) <= 1e-5 * (cq.abs().double() * (hi.abs() + lo.abs())).sum().item()


# ---- the cache ---------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("d,kv,block", [(64, 1, 16), (64, 3, 32), (128, 2, 64)])
def test_append_writes_the_documented_bytes(dtype, d, kv, block):
    n = 45
    g = torch.Generator().manual_seed(d)
    k, v = (torch.randn(n, kv, d, generator=g).to(dtype) for _ in range(2))
    k[:, :, 7] += 5.0
    k[3] = 0.25          # a constant group
    v[4] = 0.0
    slots = torch.randperm(4 * block, generator=g)[:n]
    pages = serve.cache_pages(4, block, kv, d)
    serve.append(gpu(k), gpu(v), gpu(slots), pages)
    want = torch.zeros(4 * block, kv, d), torch.zeros(4 * block, kv, d)
    want[0][slots], want[1][slots] = k.float(), v.float()
    code_ok = ref.pack(*(x.view(4, block // 16, 16, kv, d).permute(0, 3, 1, 2, 4).contiguous() for x in want))
    # places that no token was written to still hold the pool's zeros
    live = torch.zeros(4 * block, dtype=torch.bool)
    live[slots] = True
    got_k, got_v = serve.read(pages, gpu(slots), dtype=F32)
    assert torch.equal(got_k.cpu().double(), ref.held(k).float().double())
    assert torch.equal(got_v.cpu().double(), ref.held(v).float().double())
    for at in (8 * d, 17 * d):
        a, b = (x[..., at:at + d].contiguous().view(torch.half).view(4, kv, block // 16, 16, -1) for x in (pages.cpu(), code_ok))
        m = live.view(4, 1, block // 16, 16, 1)
        assert torch.equal(torch.where(m, a, 0), torch.where(m, b, 0))
    # K codes of a token are whole bytes: equal where the token is live
    a, b = (x[..., :8 * d].reshape(4, kv, block // 16, 16, d // 2) for x in (pages.cpu(), code_ok))
    m = live.view(4, 1, block // 16, 16, 1)
    assert torch.equal(torch.where(m, a, 0), torch.where(m, b, 0))
    r16 = serve.read(pages, gpu(slots), dtype=dtype)
    assert torch.equal(r16[0].cpu(), ref.held(k).float().to(dtype)) and torch.equal(r16[1].cpu(), ref.held(v).float().to(dtype))


def test_append_of_odd_numbers():
    """Infinities and NaN make their group NaN and no other; values past fp16 saturate; a slot of -1 is left out."""
    k = torch.randn(6, 2, 128)
    k[0, 0, 3], k[1, 1, 70], k[2, 0, 64] = math.inf, math.nan, -math.inf
    k[3, 1, :64] = torch.linspace(-3e6, 3e6, 64)
    k[4, 0, :64] = 1e-12
    pages = serve.cache_pages(2, 16, 2, 128)
    slots = ints([5, 6, 7, 8, 9, -1], torch.int64)
    serve.append(gpu(k), gpu(k), slots, pages)
    for x in serve.read(pages, slots):
        x = x.cpu()
        odd = torch.isnan(x).view(6, 2, 2, 64)
        want = torch.zeros(6, 2, 2, dtype=torch.bool)
        want[0, 0, 0] = want[1, 1, 1] = want[2, 0, 1] = True
        assert torch.equal(odd.all(-1), want) and torch.equal(odd.any(-1), want)
        fine = ~want[:5].repeat_interleave(64, -1).view(5, 2, 128)
        assert torch.equal(x[:5][fine], ref.held(k)[:5][fine].float()) and not x[5].any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 64), (64, 16), (128, 128), (128, 96), (128, 6), (64, 34)])
def test_append_rotates_keys_and_queries(dtype, interleaved, d, rot):
    n, kv, H = 21, 2, 6
    x = torch.randn(n, H + 2 * kv, d + 1, generator=torch.Generator().manual_seed(rot)).to(dtype)
    for view in (x[..., :d].contiguous(), x[..., 1:]):  # aligned and odd rows
        xg = torch.empty(n, H + 2 * kv, d + (0 if view.is_contiguous() else 1), dtype=dtype, device="cuda")
        xg = xg if view.is_contiguous() else xg[..., 1:]
        xg.copy_(view)
        q, k, v = xg[:, :H], xg[:, H:H + kv], xg[:, H + kv:]
        pos = torch.randint(0, 100, (n,), device="cuda").int()
        table = serve.rope_table(100, rot)
        pages = serve.cache_pages(3, 16, kv, d)
        slots = torch.randperm(48, device="cuda")[:n]
        got = serve.append(k, v, slots, pages, q=q, pos=pos, table=table, interleaved=interleaved)
        want_q, want_k = (serve.rope(t[None], None, pos[None], table, interleaved=interleaved)[0][0] for t in (q, k.float()))
        assert torch.equal(got, want_q)  # the same bits as the rotation by itself
        gk, gv = serve.read(pages, slots)
        assert torch.equal(gk.cpu().double(), ref.held(want_k.cpu()).float().double())
        assert torch.equal(gv.cpu().double(), ref.held(v.cpu()).float().double())
        inplace = q.clone()
        serve.append(k, v, slots, pages, q=inplace, q_out=inplace, pos=pos, table=table, interleaved=interleaved)
        assert torch.equal(inplace, want_q)


# ---- block tables ------------------------------------------------------------------------------------

def check_blocks(lens, new, width, block, n_free, tokens, seed=0, spare=0):
    rng = np.random.default_rng(seed)
    B = len(lens)
    held = [-(-n // block) for n in lens]
    ids = rng.permutation(sum(held) + n_free + 2).astype(np.int32)
    table = np.full((B, width), -1, np.int32)
    at = 0
    for b in range(B):
        table[b, :min(held[b], width)] = ids[at:at + held[b]][:width]
        at += held[b]
    free = torch.from_numpy(np.concatenate([ids[at:at + n_free], np.full(spare, -1, np.int32)]))
    want = ref.extend(lens, new, torch.from_numpy(table), free, n_free, block, tokens)
    t = gpu(torch.from_numpy(table))
    a, b, f, nf = ints(lens), ints(new), gpu(free), ints([n_free])
    for _ in range(2):  # the call can be repeated
        p = serve.extend_blocks(a, b, t, f, nf, block, tokens)
        for name in ("lens", "cu", "slots", "pos", "req", "n_free", "refused"):
            assert getattr(p, name).tolist() == want[name], name
        assert torch.equal(t.cpu(), want["table"])


@pytest.mark.parametrize("B", [1, 2, 31, 257, 1024, 1025, 3000])
@pytest.mark.parametrize("block", [16, 64])
def test_blocks(B, block):
    rng = np.random.default_rng(B)
    lens, new = rng.integers(0, 200, B).tolist(), rng.integers(0, 50, B).tolist()
    lens[0], new[-1] = 0, 0
    check_blocks(lens, new, 20, block, B * 5, sum(new) + 3, seed=B, spare=4)


def test_blocks_that_run_out():
    check_blocks([16, 31, 5, 40, 16], [1, 1, 20, 3, 0], 4, 16, 2, 30)     # the third finds none
    check_blocks([16, 31, 5, 40, 16], [1, 5, 20, 3, 1], 3, 16, 10, 40)    # one row is too short
    check_blocks([0, 0, 0], [1, 1, 1], 2, 16, 0, 3)                       # nothing free at all
    check_blocks([0], [0], 1, 16, 0, 0)                                   # and nothing to do
    check_blocks([7] * 40, [0] * 40, 1, 16, 3, 5)


def test_blocks_with_too_few_places_are_flagged():
    t = torch.full((2, 4), -1, dtype=torch.int32, device="cuda")
    p = serve.extend_blocks(ints([0, 0]), ints([20, 20]), t, torch.arange(8, dtype=torch.int32, device="cuda"), ints([8]), 16, 30)
    expect_flag()
    assert p.cu.tolist() == [0, 20, 40] and p.req.tolist() == [0] * 20 + [1] * 10


# ---- together ----------------------------------------------------------------------------------------

def test_a_layer_answers_step_by_step():
    """Prompts of three requests, then single tokens, through the layer's step: each output is the plain attention, in
    64 bits, over the numbers the cache holds; and near the training forward of the same tokens, but for 4-bit noise."""
    torch.manual_seed(0)
    cfg = kint.Config(Kint=8, calib=FWM, tau=8.0, recon=LERP)
    layer = serve.KIntServingAttention(256, 4, cfg, max_pos=128, rot=32, prec=kint.PREC_3XTF32)
    cache = serve.PagedCache(1, 3, 100, 16, 4, 64, block_size=16)
    x = torch.randn(3, 40, 256, device="cuda")
    with torch.no_grad():
        whole = layer(x)
    prompt = [17, 5, 32]
    plan = cache.extend(ints(prompt), sum(prompt))
    rows = torch.cat([x[b, :n] for b, n in enumerate(prompt)])
    y = layer.step(rows, cache, plan)
    at = list(prompt)
    outs = {b: [y[sum(prompt[:b]):sum(prompt[:b]) + n]] for b, n in enumerate(prompt)}
    for _ in range(4):
        plan = cache.extend(ints([1, 1, 1]), 3)
        y = layer.step(torch.stack([x[b, at[b]] for b in range(3)]), cache, plan, max_new=1)
        for b in range(3):
            outs[b].append(y[b:b + 1])
            at[b] += 1
    assert cache.lens.tolist() == at and int(plan.refused) == 0
    for b in range(3):
        got = torch.cat(outs[b])
        slots = (cache.table[b].long().clamp(min=0)[:, None] * 16 + torch.arange(16, device="cuda")).flatten()[:at[b]]
        k, v = (t.cpu().double() for t in serve.read(cache.pages[0], slots))
        q = layer.c_attn(x[b, :at[b]]).split(256, dim=-1)[0].view(1, at[b], 4, 64).detach()
        q = serve.rope(q, None, torch.arange(at[b], dtype=torch.int32, device="cuda"), layer.rope)[0][0]
        o, safe = ref.attention(q.cpu().double(), [k], [v], [at[b]], [at[b]], cfg)
        want = layer.c_proj(o.float().cuda().view(at[b], 256)).detach()
        ok = safe.all(-1).cuda()
        assert ok.float().mean() > 0.4
        # the attention's bar through a projection of 256 inputs of weights below 1/16
        assert ((got - want).abs().amax(-1)[ok] <= 3e-5 * v.abs().max().item() * 16 + 1e-5).all()
        near = whole[b, :at[b]]
        assert (got - near).norm() / near.norm() < 0.2  # steps of about 0.3 of a key's spread
    cache.release(1)
    assert int(cache.n_free) == 16 - sum(-(-at[b] // 16) for b in (0, 2)) and cache.lens.tolist() == [at[0], 0, at[2]]
    plan = cache.extend(ints([0, 30, 0]), 30)
    assert int(plan.refused) == 0 and len(set(plan.slots.tolist())) == 30


def test_the_layer_trains():
    """Gradients of the serving block's training forward against the same block with torch's rotation around the op."""
    torch.manual_seed(1)
    cfg = kint.Config(Kint=4, calib=SOFT)
    layer = serve.KIntServingAttention(128, 2, cfg, max_pos=64, prec=kint.PREC_3XTF32)
    x = torch.randn(2, 33, 128, device="cuda", requires_grad=True)
    dy = torch.randn(2, 33, 128, device="cuda")
    layer(x).backward(dy)
    got = [x.grad.clone()] + [p.grad.clone() for p in layer.parameters()]
    x.grad = None
    layer.zero_grad()
    q, k, v = (t.view(2, 33, 2, 64) for t in layer.c_attn(x).split(128, dim=2))
    cs = layer.rope[:33, None]
    turn = lambda t: torch.cat([t[..., :32] * cs[..., 0] - t[..., 32:] * cs[..., 1],  # noqa: E731
                                t[..., 32:] * cs[..., 0] + t[..., :32] * cs[..., 1]], -1)
    q, k, v = (t.transpose(1, 2).contiguous() for t in (turn(q), turn(k), v))
    s = (q @ k.transpose(2, 3)) / 8
    s = s.masked_fill(torch.ones(33, 33, device="cuda").triu(1).bool(), -math.inf)
    layer.c_proj((torch.softmax(s, -1) @ v).transpose(1, 2).reshape(2, 33, 128)).backward(dy)
    for a, b in zip(got, [x.grad] + [p.grad for p in layer.parameters()]):
        assert (a - b).abs().max() <= 1e-4 * b.abs().max()
