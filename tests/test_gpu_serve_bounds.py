"""GPU: what the serving operators do at and past the bounds that a caller states, and with rows, blocks and memory that
belong to nobody.  Tolerances are those of test_gpu_serve.py; the rest is equality."""
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
