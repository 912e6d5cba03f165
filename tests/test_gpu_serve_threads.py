"""GPU: attention over the cache called from several host threads at once (the C calls hold no Python lock)."""
import threading

import pytest
import torch

from paper_2609_33591_gb300 import kint, serve
from tests.test_gpu_serve import BF16, F32, MM, SOFT, _clean, _lib, ints  # noqa: F401

pytestmark = pytest.mark.gpu
RESOLVED = kint.CALIB_FWM_RESOLVED


@pytest.mark.parametrize("d,heads", [(64, 4), (64, 8), (64, 16), (128, 4), (128, 8), (128, 16)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("calib", [SOFT, MM, RESOLVED])
def test_several_host_threads(d, heads, dtype, calib):
    """Calls that need different amounts of shared memory at once: no thread's is taken back by another's."""
    B, code = 160, {F32: 0, BF16: 1}[dtype]
    pages = serve.cache_pages(4, 4096, 1, d)
    pool = serve.kint_cache(pages.data_ptr(), pages.stride(0), 4, 4096, 1, d)
    lens, cu, table = ints([0] * B), ints(list(range(B + 1))), torch.zeros(B, 8, dtype=torch.int32, device="cuda")
    q = torch.zeros(B, heads, d, dtype=dtype, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    rcs = []
    start = threading.Barrier(4)

    def work(turn):
        o = torch.empty_like(q)
        hq, ho = (serve.kint_heads(x.data_ptr(), 0, heads * d, d, heads) for x in (q, o))
        start.wait()
        for i in range(24):
            max_len = 512 + 256 * ((7 * i + 6 * turn) % 24)
            rcs.append(serve.load().kint_cache_attn(hq, ho, pool, table.data_ptr(), 8, 8, lens.data_ptr(), cu.data_ptr(), B, B, 0, 0,
                                                    1 + (5 * i + 16 * turn) % 64, calib, 8.0, 0, 1, max_len, code, ws.data_ptr(),
                                                    ws.numel(), None))

    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(t,)) for t in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert len(rcs) == 96 and not any(rcs)
