"""Sizes past what the serving operators' indices hold are refused on the host (no GPU needed)."""
import pytest

from paper_2609_33591_gb300 import serve
from tests.test_serve_host import ATTN, P, cache, heads


@pytest.mark.parametrize("sizes", [
    dict(B=1, heads=512, kv=1, max_new=1 << 24),              # 2^33 rows a kv head
    dict(B=1, heads=129, kv=1, max_new=(1 << 23) + 1),        # one group of heads past 2^30
    dict(B=1 << 20, heads=1 << 24, kv=1 << 12, max_new=1 << 24),  # requests x kv heads x tiles = 2^64
    dict(B=(1 << 31) - 1, heads=1 << 16, kv=1 << 16, max_new=1 << 24),
    dict(B=(1 << 31) - 1, heads=2, kv=1, max_new=1),
])
def test_more_rows_or_units_than_an_index_holds(sizes):
    f = serve.load().kint_cache_attn_workspace_bytes
    assert f(sizes["B"], sizes["heads"], sizes["kv"], 64, 0, 0, sizes["max_new"], 256) == 0
    if sizes["heads"] <= 1 << 16:
        q = heads(sizes["heads"])
        pool = cache(kv_heads=sizes["kv"], block_stride=2 * 18 * 64 * sizes["kv"], pages=P)
        assert serve.load().kint_cache_attn(*{**ATTN, "q": q, "out": q, "cache": pool, "B": sizes["B"], "max_new": sizes["max_new"]}.values()) == -2


def test_the_most_rows_that_an_index_holds():
    f = serve.load().kint_cache_attn_workspace_bytes
    assert f(1, 64, 1, 64, 0, 0, 1 << 24, 256) > 0


ROPE = dict(q=heads(), qo=heads(), k=heads(0), ko=heads(0), pos=P, sb=0, table=P, max_pos=8, B=1, T=8, d=64, rot=64, il=0, inv=0, dtype=1,
            stream=None)
MOST = (1 << 31) - 1


@pytest.mark.parametrize("kw", [
    dict(q=heads(MOST - 2), qo=heads(MOST - 2)),                                          # groups of 8 heads past 2^31
    dict(q=heads(1 << 30), qo=heads(1 << 30), k=heads(1 << 30), ko=heads(1 << 30)),       # heads of both past 2^31
    dict(B=MOST, T=MOST, q=heads(1 << 24), qo=heads(1 << 24)),                            # work items past 2^63
    dict(B=1 << 16, T=1 << 15),
])
def test_rotations_of_more_items_than_an_index_holds(kw):
    assert serve.load().kint_rope(*{**ROPE, **kw}.values()) == -2


@pytest.mark.parametrize("tokens", [MOST, MOST - 6])
def test_more_cached_tokens_than_an_index_holds(tokens):
    """A warp a token: the last block's warps are numbered past the last token."""
    lib = serve.load()
    assert lib.kint_cache_append(cache(), heads(), heads(), P, tokens, None, None, None, None, 0, 0, 0, 0, None) == -2
    assert lib.kint_cache_read(cache(), P, tokens, heads(), None, 0, None) == -2
