"""GPU: every way in which attention over the cache is launched, against the plain 64-bit forms.

Which way a call takes is read off the launch callback (the kernels' names) and the workspace's size (a cluster launch
needs none), so a change of the launch rules cannot quietly empty these tests.  Tolerances: test_gpu_serve.py.
"""
import pytest
import torch

from paper_2609_33591_gb300 import kint, serve
from tests import serve_ref as ref
from tests.test_gpu_serve import BF16, F16, F32, FWM, HALF_UNIT, LERP, MM, SOFT, _clean, _lib, filled, gpu, ints  # noqa: F401

pytestmark = pytest.mark.gpu

CLUSTER, TOGETHER, TWO = ["k_attn"], ["k_attn", "together"], ["k_attn_scores", "k_attn_values"]
FALLBACK = TWO  # blocks planned to run together that do not fit at once
RESOLVED = kint.CALIB_FWM_RESOLVED


def launched(call, *sizes, **bounds):
    """The call's result and the way it took; sizes: B, heads, kv heads, d."""
    names = []
    kint.kint_set_launch_callback(lambda name, phase, stream: names.append(name) if phase == 0 else None)
    try:
        out = call()
    finally:
        kint.kint_set_launch_callback(None)
    if names == ["k_attn"] and serve.attention_workspace(*sizes, **bounds).numel() > 256:
        names.append("together")
    return out, names


def check(way, long, requests, heads, kv, new, d, calib, dtype, K=8, max_len=None, seed=50):
    """`requests` requests on one list of `long` tokens: the first holds all of it, the second a little less, the others a few."""
    lens = ([long, long - 37] + [3 + 5 * (b % 7) for b in range(requests)])[:requests]
    new = [min(new, n) for n in lens]
    pool = filled([long], kv, d, 64, seed)
    table = pool.table.repeat(requests, 1)
    max_len = max_len or table.size(1) * 64
    table = torch.nn.functional.pad(table, (0, -(-max_len // 64) - table.size(1)), value=-1)
    q = torch.randn(sum(new), heads, d, generator=torch.Generator().manual_seed(seed + 1)).to(dtype)
    cu = torch.tensor([0] + new).cumsum(0).int()
    cfg, bounds = kint.Config(Kint=K, calib=calib, tau=6.0, recon=LERP), dict(max_new=max(new), max_len=max_len)
    args = gpu(q), gpu(pool.pages), gpu(table), ints(lens), gpu(cu)
    o, names = launched(lambda: serve.attention(*args, cfg, **bounds), requests, heads, kv, d, **bounds)
    assert names == way
    k, v = ([x[0][:n] for n in lens] for x in (pool.k, pool.v))
    want, safe = ref.attention(q.double(), k, v, lens, new, cfg)
    rare = calib not in (SOFT, FWM, MM)
    bad = ((o.cpu().double() - want).abs() > HALF_UNIT[dtype] * want.abs() + (2e-4 if rare else 3e-5) * pool.v[0].abs().max()).any(-1) & safe
    assert not bad.any() and safe.float().mean() > 0.4
    return args, cfg, bounds, o


# heads and new tokens of one kv head: tiles of 4, 8 and 16 rows
TILES = [(4, 1), (1, 4), (8, 1), (2, 3), (16, 1), (5, 4)]


@pytest.mark.parametrize("calib,dtype", [(SOFT, F32), (SOFT, BF16), (FWM, BF16), (FWM, F32), (MM, F16), (RESOLVED, F32)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,new", TILES)
def test_blocks_that_run_together(heads, new, d, calib, dtype):
    check(TOGETHER, 9100, 3, heads, 1, new, d, calib, dtype)


@pytest.mark.parametrize("calib,dtype", [(SOFT, F32), (SOFT, BF16), (FWM, BF16), (FWM, F32), (MM, F16), (RESOLVED, F32)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,new", TILES)
def test_two_launches(heads, new, d, calib, dtype):
    check(TWO, 8700 if heads * new > 8 else 16500, 39, heads, 1, new, d, calib, dtype)


@pytest.mark.parametrize("heads,new", TILES)
def test_clusters_with_the_larger_share_of_shared_memory(heads, new):
    """As long as clusters go: 32 KB of scores a block (tiles of four rows), 48 and 56 KB."""
    check(CLUSTER, 16000 if heads * new <= 4 else 12000 if heads * new <= 8 else 7000, 40, heads, 1, new, 64, MM, F32, K=64)


@pytest.mark.parametrize("heads,new", [(4, 1), (1, 3)])
def test_blocks_that_do_not_fit_at_once(heads, new):
    """MinMax with many intervals: its tables leave room for fewer blocks than the launch was planned with."""
    check(FALLBACK, 9000, 19, heads, 1, new, 128, MM, BF16, K=64, max_len=65536)


@pytest.mark.parametrize("way,requests,heads,calib,K,max_len", [(TOGETHER, 2, 4, FWM, 8, None), (TOGETHER, 2, 16, MM, 8, None),
                                                               (TWO, 39, 16, FWM, 8, None), (FALLBACK, 19, 4, MM, 64, 65536)])
def test_captured(way, requests, heads, calib, K, max_len):
    """In a captured graph, replay after replay: the plain call's bits."""
    args, cfg, bounds, want = check(way, 9100, requests, heads, 1, 1, 128, calib, BF16, K=K, max_len=max_len)
    ws = serve.attention_workspace(requests, heads, 1, 128, **bounds)
    res = torch.zeros_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        serve.attention(*args, cfg, out=res, ws=ws, **bounds)
    for _ in range(2):
        res.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(res, want)


@pytest.mark.parametrize("heads", [4, 8, 16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("calib", [SOFT, MM])
def test_rounding_of_long_sums(calib, d, heads):
    """Over 131071 keys the values average out to a hundredth of themselves.  The result in fp16 is then off by its own rounding and
    no more: within a tenth of the error of the 64-bit result rounded once (fp32 sums add some 2^-24 of the values, a hundredth of
    an fp16 unit of such a result, to each)."""
    n, g = 131071, torch.Generator(device="cuda").manual_seed(d + heads)
    pages, slots = serve.cache_pages(128, 1024, 1, d), torch.arange(n, device="cuda")
    k, v, q = (torch.randn(m, h, d, device="cuda", generator=g).half() for m, h in ((n, 1), (n, 1), (1, heads)))
    serve.append(k, v, slots, pages)
    cfg = kint.Config(Kint=8, calib=calib, recon=LERP)
    table = torch.arange(128, dtype=torch.int32, device="cuda")[None]
    o = serve.attention(q, pages, table, ints([n]), ints([0, 1]), cfg, max_new=1, max_len=n)[0].double()
    k, v = (x[:, 0].double() for x in serve.read(pages, slots))
    s = q[0].double() @ k.T / d ** 0.5
    w = torch.stack([ref.weights((x - x.max()).cpu(), cfg) for x in s]).cuda()
    want = w @ v / w.sum(-1, keepdim=True)
    assert (o - want).norm() <= 1.1 * (want.half().double() - want).norm()
