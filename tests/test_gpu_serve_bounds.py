"""GPU: what the serving operators do at and past the bounds that a caller states, and with rows, blocks and memory that
belong to nobody.  Tolerances are those of test_gpu_serve.py; the rest is equality."""
import math
import threading

import numpy as np
import pytest
import torch

from paper_2609_33591_gb300 import kint, serve
from tests import serve_ref as ref
from tests.test_gpu_serve import (BF16, F32, FWM, HALF_UNIT, LERP, MM, SOFT, _clean, _lib, expect_flag, filled,  # noqa: F401
                                  gpu, ints)

pytestmark = pytest.mark.gpu


def offsets(new):
    return np.concatenate([[0], np.cumsum(new)]).tolist()


@pytest.mark.parametrize("requests", [6110, 6111, 6144, 6145, 16384, 6111])
def test_blocks_of_many_requests(requests):
    """Prefix sums at and past 48 KB of shared memory (6111 to 6144 requests reach it with what the kernel holds besides), up to
    the largest number of requests."""
    from tests.test_gpu_serve import check_blocks
    rng = np.random.default_rng(requests)
    lens, new = rng.integers(0, 60, requests).tolist(), rng.integers(0, 4, requests).tolist()
    check_blocks(lens, new, 4, 16, requests, sum(new) + 3, seed=requests)


def test_blocks_from_several_host_threads():
    """Calls of very different sizes at once: no thread's shared memory is taken back by another's."""
    rcs = []

    def work(requests):
        i32 = dict(dtype=torch.int32, device="cuda")
        lens, new = torch.zeros(requests, **i32), torch.ones(requests, **i32)
        table, free, n_free = torch.zeros(requests, 1, **i32), torch.arange(requests, **i32), ints([requests])
        out = torch.empty(8 * requests + 8, **i32)
        slots = torch.empty(requests, dtype=torch.int64, device="cuda")
        at = [x.data_ptr() for x in (out, out[8 * requests:], out[2 * requests:], slots, out[4 * requests:], out[5 * requests:],
                                     out[8 * requests + 4:])]
        torch.cuda.synchronize()
        for _ in range(300):
            rcs.append(serve.load().kint_blocks_extend(lens.data_ptr(), new.data_ptr(), table.data_ptr(), 1, 1, free.data_ptr(), requests,
                                                       n_free.data_ptr(), requests, 16, requests, *at, None))

    threads = [threading.Thread(target=work, args=(n,)) for n in (16384, 7000, 12000, 9000)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert len(rcs) == 1200 and not any(rcs)


@pytest.mark.parametrize("calib", [SOFT, FWM, MM])
@pytest.mark.parametrize("heads,kv,bound,d,dtype", [(4, 1, 1, 128, BF16), (1, 1, 3, 64, F32), (6, 2, 1, 64, BF16), (8, 1, 1, 64, F32),
                                                    (5, 1, 1, 128, BF16), (12, 1, 1, 64, BF16), (16, 2, 4, 128, F32)])
@pytest.mark.parametrize("lens", [[40, 0, 33, 300], [9000]])
def test_rows_past_the_stated_bound_are_left_out(calib, heads, kv, bound, d, dtype, lens):
    """Requests with more new tokens than max_new says: their first max_new rows are answered at their own positions, the rest
    of `out` is not touched, and the call is flagged.  Tiles of 4, 8 and 16 rows, in one launch of clusters and (9000 keys) of
    blocks that run together."""
    new = [min(n, e) for n, e in zip(lens, (bound + 3, 0, bound, bound + 17))]
    pool = filled(lens, kv, d, 64, 40)
    q = torch.randn(sum(new), heads, d, generator=torch.Generator().manual_seed(41)).to(dtype)
    out = torch.full((sum(new), heads, d), 7.0, dtype=dtype, device="cuda")
    cfg = kint.Config(Kint=8, calib=calib, tau=6.0, recon=LERP)
    serve.attention(gpu(q), gpu(pool.pages), gpu(pool.table), gpu(pool.lens), ints(offsets(new)), cfg, max_new=bound, out=out)
    expect_flag()
    at = torch.tensor([j < bound for n in new for j in range(n)])
    got = out.cpu().double()
    assert (got[~at] == 7.0).all()
    want, safe = ref.attention(q.double(), pool.k, pool.v, lens, new, cfg)
    top = max(float(x.abs().max()) for x in pool.v if x.numel())
    bad = ((got - want).abs() > HALF_UNIT[dtype] * want.abs() + 3e-5 * top).any(-1) & safe
    assert not bad[at].any()


def test_as_many_places_as_an_index_holds():
    """2^31 - 1 places for 8 tokens (34 GB of slots, positions and requests)."""
    tokens = (1 << 31) - 1
    table = torch.full((2, 4), -1, dtype=torch.int32, device="cuda")
    p = serve.extend_blocks(ints([0, 20]), ints([5, 3]), table, torch.arange(8, dtype=torch.int32, device="cuda"), ints([8]), 16, tokens)
    # the second request's first two blocks are not in its table: its new tokens (places 20 to 22) have no slot
    expect_flag()
    assert p.slots[:10].tolist() == [112, 113, 114, 115, 116, -1, -1, -1, -1, -1]
    assert p.pos[:10].tolist() == [0, 1, 2, 3, 4, 20, 21, 22, -1, -1] and p.req[:9].tolist() == [0] * 5 + [1] * 3 + [-1]
    for x in (p.slots, p.pos, p.req):
        for at in (1 << 30, 3 << 29, tokens - 700000):
            assert (x[at:at + 700000] == -1).all()
        assert (x[tokens - 9:] == -1).all()


# the three ways in which attention is launched: lengths, heads of one kv head
WAYS = [([40, 3, 0, 300], 4), ([40, 3, 0, 300], 16), ([9000, 3, 0, 30], 4), ([8300, 3, 0, 30], 8)]


def poison(like):
    """Freed memory full of NaN, which an output of the same size is given next."""
    torch.cuda.synchronize()
    x = torch.full_like(like, float("nan"))
    torch.cuda.synchronize()
    del x


@pytest.mark.parametrize("before,behind", [(0, 5), (3, 0), (2, 700)])
@pytest.mark.parametrize("lens,heads", WAYS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_of_no_request_are_zero(dtype, lens, heads, before, behind):
    """Rows of q before the first request's and behind the last one's; in a given `out` they are left as they are."""
    max_new = 130 if heads == 8 else 2
    new = [min(n, e) for n, e in zip(lens, (max_new, 1, 0, 2))]
    pool = filled(lens, 1, 64, 64, 60)
    q = torch.randn(before + sum(new) + behind, heads, 64, device="cuda").to(dtype)
    cu = ints([before + x for x in offsets(new)])
    args, kw = (gpu(pool.pages), gpu(pool.table), gpu(pool.lens)), dict(max_new=max_new)
    cfg, inner = kint.Config(calib=FWM, recon=LERP), slice(before, before + sum(new))
    want = serve.attention(q[inner].contiguous(), *args, ints(offsets(new)), cfg, **kw)
    poison(q)
    got = serve.attention(q, *args, cu, cfg, **kw)
    assert torch.equal(got[inner], want)
    assert (got[:before] == 0).all() and (got[inner.stop:] == 0).all()
    out = torch.full_like(q, 7.0)
    serve.attention(q, *args, cu, cfg, out=out, **kw)
    assert torch.equal(out[inner], want) and (out[:before] == 7.0).all() and (out[inner.stop:] == 7.0).all()


@pytest.mark.parametrize("cu", [[-1, 0], [0, 2], [1, 2], [3, 2]])
def test_rows_that_q_does_not_have_leave_zeros(cu):
    """A request left out for its offsets: flagged, and a new output holds zeros."""
    pool = filled([40], 2, 64, 32, 14)
    q = torch.randn(1, 2, 64, device="cuda")
    poison(q)
    o = serve.attention(q, gpu(pool.pages), gpu(pool.table), gpu(pool.lens), ints(cu), kint.Config(calib=SOFT), max_new=4)
    expect_flag()
    assert (o == 0).all()


def test_rows_past_the_stated_bound_are_zero_in_a_new_output():
    pool = filled([40], 2, 64, 32, 14)
    q = torch.randn(9, 4, 64, device="cuda")
    poison(q)
    o = serve.attention(q, gpu(pool.pages), gpu(pool.table), gpu(pool.lens), ints([0, 9]), kint.Config(calib=SOFT), max_new=2)
    expect_flag()
    assert (o[:2] != 0).any() and (o[2:] == 0).all()


def test_a_step_with_places_left_over():
    """Places behind the last new token go through the layer as rows of zeros, not as what memory holds."""
    layer = serve.KIntServingAttention(256, 4, kint.Config(calib=FWM), max_pos=128)
    cache = serve.PagedCache(1, 2, 128, 16, 4, 64, block_size=16)
    x = torch.randn(9, 256, device="cuda")
    plan = cache.extend(ints([3, 2]), 9)
    poison(torch.empty(9, 4, 64, device="cuda"))
    y = layer.step(x, cache, plan, max_new=3)
    assert torch.isfinite(y).all() and torch.equal(y[5:], layer.c_proj(torch.zeros(4, 256, device="cuda")).detach())


@pytest.mark.parametrize("lens,heads", WAYS)
def test_refused_requests_get_zeros(lens, heads):
    """With the plan's slots, rows of a request that found no blocks are zero (their keys are not in the cache); the others'
    bits do not change.  Through a given `out` too."""
    max_new = 130 if heads == 8 else 2
    new = [min(n, e) for n, e in zip(lens, (max_new, 1, 0, 2))]
    pool = filled(lens, 1, 64, 64, 61)
    q = torch.randn(sum(new) + 2, heads, 64, device="cuda")
    args = gpu(pool.pages), gpu(pool.table), gpu(pool.lens), ints(offsets(new)), kint.Config(calib=FWM, recon=LERP)
    want = serve.attention(q, *args, max_new=max_new)
    for b in (0, 1, 3):
        slots = torch.arange(q.size(0), device="cuda")
        rows = slice(sum(new[:b]), sum(new[:b + 1]))
        slots[rows] = -1
        slots[sum(new):] = -1
        for out in (None, torch.full_like(q, 7.0)):
            poison(q)
            got = serve.attention(q, *args, max_new=max_new, slots=slots, out=out)
            assert (got[rows] == 0).all() and torch.equal(got[:rows.start], want[:rows.start])
            assert torch.equal(got[rows.stop:sum(new)], want[rows.stop:sum(new)])
            assert (got[sum(new):] == (0.0 if out is None else 7.0)).all()


def test_a_step_that_refuses_a_request():
    """Two blocks of 16 for two requests of 16 and 10 tokens: the third is refused, and later the first finds no block for its
    17th.  Their rows are the projection of zeros; the others' are what they are without them."""
    torch.manual_seed(2)
    layer = serve.KIntServingAttention(256, 4, kint.Config(calib=FWM), max_pos=64)
    cache, twin = (serve.PagedCache(1, 3, 64, n, 4, 64, block_size=16) for n in (2, 8))
    zero = layer.c_proj(torch.zeros(1, 256, device="cuda")).detach()
    x = torch.randn(33, 256, device="cuda")
    y = layer.step(x, cache, cache.extend(ints([16, 10, 7]), 33), max_new=16)
    z = layer.step(x, twin, twin.extend(ints([16, 10, 7]), 33), max_new=16)
    assert torch.equal(y[:26], z[:26]) and torch.equal(y[26:], zero.expand(7, -1)) and not torch.equal(z[26:], y[26:])
    x = torch.randn(2, 256, device="cuda")
    plan = cache.extend(ints([1, 1, 0]), 2)
    y = layer.step(x, cache, plan, max_new=1)
    z = layer.step(x, twin, twin.extend(ints([1, 1, 0]), 2), max_new=1)
    assert int(plan.refused) == 1 and cache.lens.tolist() == [16, 11, 0]
    assert torch.equal(y[:1], zero) and torch.equal(y[1], z[1])
    with pytest.raises(ValueError):
        serve.attention(torch.zeros(2, 4, 64, device="cuda"), cache.pages[0], cache.table, plan.lens, plan.cu, kint.Config(),
                        slots=plan.slots[:1])


@pytest.mark.parametrize("calib,recon", [(FWM, LERP), (FWM, kint.RECON_NEAREST), (kint.CALIB_EXP_FP8, LERP), (SOFT, LERP)])
@pytest.mark.parametrize("place", [3, 36])
def test_a_value_that_is_seen_with_no_weight_still_shows_its_nan(calib, recon, place):
    """0 times NaN is NaN whether the key's slab is seen in full or lies at the end of the list (40 keys: slabs 0 and 2), and
    only in the 64 channels that hold it; a key that is not seen stays out."""
    k, v = torch.randn(40, 1, 128), torch.randn(40, 1, 128)
    k[:, :, 0], q = 1.0, torch.zeros(1, 2, 128)
    q[..., 0] = 3000.0
    k[place, 0, 0] = -1.0   # a score some 500 below the others': weight 0 (under softmax below the smallest number)
    v[place, 0, 70] = math.nan
    pages, table = serve.cache_pages(2, 64, 1, 128), ints([[1]])
    serve.append(gpu(k), gpu(v), 64 + torch.arange(40, device="cuda"), pages)
    cfg = kint.Config(Kint=4, calib=calib, tau=3.0, recon=recon)
    for n, shows in ((40, True), (place, False)):
        o = serve.attention(gpu(q), pages, table, ints([n]), ints([0, 1]), cfg)
        assert torch.isfinite(o[..., :64]).all()
        assert torch.isnan(o[..., 64:]).all() if shows else torch.isfinite(o[..., 64:]).all()


def test_a_free_list_of_rows_is_refused():
    """Only its last dimension's stride is looked at, so rows further apart (or on top of each other) would be read as one list."""
    lens, new, table, n_free = ints([0]), ints([3]), ints([[-1]]), ints([4])
    for free in (ints([[4, 5], [6, 7]]), ints([[4, 5, 0], [6, 7, 0]])[:, :2], ints([1]).expand(4, 1)):
        with pytest.raises(ValueError, match="free"):
            serve.extend_blocks(lens, new, table, free, n_free, 16, 3)
    assert table.tolist() == [[-1]]


def test_sizes_past_31_bits_are_refused():
    """Not taken modulo 2^32 (here 2^32 + 2 heads on top of each other as 2)."""
    x = torch.ones(1, 1, 1, 64, device="cuda")
    many = x.expand(1, 1, (1 << 32) + 2, 64)
    with pytest.raises(ValueError, match="past 2"):
        serve.rope(many, None, ints([1]), serve.rope_table(4, 64), out=(many, None))
    assert (x == 1).all()
