"""GPU: the serving layer, the cache that it keeps, and the smaller calls at their edges."""
import pytest
import torch

from paper_2609_33591_gb300 import kint, serve
from tests.test_gpu_serve import BF16, F16, F32, FWM, _clean, _lib, expect_flag, ints  # noqa: F401

pytestmark = pytest.mark.gpu


def test_positions_that_the_table_does_not_hold_are_refused():
    """Sequences and caches longer than the layer's rotations: an error, not rows without a rotation."""
    layer = serve.KIntServingAttention(256, 4, kint.Config(), max_pos=32)
    assert layer(torch.randn(1, 32, 256, device="cuda")).shape == (1, 32, 256)
    with pytest.raises(ValueError, match="max_pos"):
        layer(torch.randn(1, 33, 256, device="cuda"))
    cache = serve.PagedCache(1, 1, 64, 8, 4, 64, block_size=16)
    x = torch.randn(4, 256, device="cuda")
    plan = cache.extend(ints([4]), 4)
    with pytest.raises(ValueError, match="max_pos"):
        layer.step(x, cache, plan)
    with pytest.raises(ValueError, match="max_pos"):
        layer.step(x, cache, plan, max_len=33)
    assert not cache.pages.any()
    assert layer.step(x, cache, plan, max_len=32).shape == x.shape  # a shorter bound than the cache's


def test_a_buffer_for_queries_that_are_not_rotated_is_refused():
    x, buf = torch.randn(3, 2, 64, device="cuda"), torch.full((3, 2, 64), 7.0, device="cuda")
    pages, slots = serve.cache_pages(1, 16, 2, 64), ints([0, 1, 2], torch.int64)
    for kw in (dict(q=x), dict(), dict(table=serve.rope_table(4, 64), pos=ints([0, 1, 2]))):
        with pytest.raises(ValueError, match="q_out"):
            serve.append(x, x, slots, pages, q_out=buf, **kw)
    assert not pages.any() and (buf == 7.0).all()
    assert serve.append(x, x, slots, pages, q=x) is x and serve.append(x, x, slots, pages) is None


@pytest.mark.parametrize("hq,hk", [(0, 2), (2, 0)])
@pytest.mark.parametrize("place", [False, True])
def test_rope_of_one_of_two(hq, hk, place):
    """Queries or keys of no heads: the other is rotated."""
    table, pos = serve.rope_table(8, 64), ints([0, 1, 5])
    q, k = torch.randn(2, 3, hq, 64, device="cuda"), torch.randn(2, 3, hk, 64, device="cuda")
    x = q if hq else k
    want = serve.rope(x, None, pos, table)[0]
    a, b = serve.rope(q, k, pos, table, out=(q, k) if place else None)
    assert torch.equal(a if hq else b, want) and a.shape == q.shape and b.shape == k.shape


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_the_layer_in_another_type(dtype):
    """Casting the layer casts its weights; the rotations stay fp32, the same numbers, and follow it to a device.  (Numbers
    kept in 4 bits are off by a tenth of their spread, as scores and as values: 0.3 of the output is twice both.)"""
    torch.manual_seed(3)
    layer = serve.KIntServingAttention(256, 4, kint.Config(Kint=8, calib=FWM, tau=8.0, recon=kint.RECON_LERP), max_pos=64)
    table = layer.rope.clone()
    x = torch.randn(1, 20, 256, device="cuda")
    want = layer(x).detach()
    for cast in (lambda m: m.to(dtype), lambda m: m.cpu().cuda(), lambda m: m.to("cpu", torch.float64).to("cuda", dtype)):
        layer = cast(layer)
        assert layer.rope.dtype == F32 and layer.rope.is_cuda and torch.equal(layer.rope, table) and layer.c_proj.weight.dtype == dtype
        assert "rope" not in layer.state_dict()
        y = layer(x.to(dtype))
        assert y.dtype == dtype and (y.float() - want).norm() <= 0.05 * want.norm()
        cache = serve.PagedCache(1, 1, 64, 4, 4, 64, block_size=16)
        s = layer.step(x[0].to(dtype), cache, cache.extend(ints([20]), 20), max_new=20)
        assert s.dtype == dtype and (s.float() - want[0]).norm() <= 0.3 * want.norm()


def owner(t):
    """The stream that t's memory belongs to."""
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]


def test_memory_belongs_to_the_stream_that_is_given():
    """On another stream than the current one nothing orders the current stream's use of a block of memory and the call's."""
    side = torch.cuda.Stream()
    table = serve.rope_table(16, 64, stream=side)
    pages = serve.cache_pages(2, 16, 2, 64)
    x, slots, pos = torch.randn(3, 2, 64, device="cuda"), ints([0, 1, 2], torch.int64), ints([0, 1, 2])
    torch.cuda.synchronize()
    made = [table, serve.rope(x[None], None, pos, table, stream=side)[0], serve.read(pages, slots, stream=side)[0],
            serve.append(x, x, slots, pages, q=x, pos=pos, table=table, stream=side),
            serve.attention(x, pages, ints([[0, 1]]), ints([3]), ints([0, 3]), kint.Config(), stream=side),
            serve.extend_blocks(ints([0]), ints([3]), ints([[-1]]), ints([0]), ints([1]), 16, 3, stream=side).slots]
    side.synchronize()
    assert [owner(t) for t in made] == [side.cuda_stream] * len(made)
    assert torch.equal(table, serve.rope_table(16, 64))


def test_a_cache_takes_its_own_size_of_memory():
    """Not its layers' pools twice over."""
    torch.cuda.empty_cache()
    before = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    cache = serve.PagedCache(8, 4, 4096, 2048, 8, 128, block_size=32)
    assert torch.cuda.max_memory_allocated() - before <= 1.1 * cache.pages.numel()
    assert cache.pages.shape == (8, 2048, 8, 2, 18 * 128) and not cache.pages.any()
    for bad in (dict(block_size=24), dict(block_size=8)):
        with pytest.raises(kint.KintError):
            serve.PagedCache(1, 1, 64, 4, 4, 64, **bad)
    with pytest.raises(kint.KintError):
        serve.PagedCache(1, 1, 64, 4, 4, 96)


def test_a_request_may_fill_its_last_block():
    """A table of blocks holds more than a max_len that is no multiple of them, and extend hands the rest out: every key is seen."""
    torch.manual_seed(4)
    layer = serve.KIntServingAttention(256, 4, kint.Config(Kint=8, calib=FWM, recon=kint.RECON_LERP), max_pos=128)
    x = torch.randn(120, 256, device="cuda")
    short, long = (serve.PagedCache(1, 1, n, 2, 4, 64, block_size=64) for n in (100, 128))
    got, want = (torch.cat([layer.step(x[a:b], c, c.extend(ints([b - a]), b - a), max_new=b - a) for a, b in ((0, 90), (90, 119), (119, 120))])
                 for c in (short, long))
    assert short.lens.tolist() == [120] and torch.equal(got, want)
