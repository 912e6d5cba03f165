"""A K-interval attention block answering from the 4-bit paged cache: prompts of three requests, then single tokens.

    python examples/serve_step.py

Random weights and inputs (the block is the GPT-2 attention layer with rotary positions); prints how far each step's output
is from the block's own full-precision forward over the same tokens, which is what 4 bits a channel cost.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_33591_gb300 import kint, serve  # noqa: E402


def main():
    torch.manual_seed(0)
    n_embd, n_head, max_len, steps = 768, 12, 256, 8
    cfg = kint.Config(Kint=4, calib=kint.CALIB_FWM, tau=8.0, recon=kint.RECON_NEAREST)
    layer = serve.KIntServingAttention(n_embd, n_head, cfg, max_pos=max_len)
    cache = serve.PagedCache(layers=1, requests=3, max_len=max_len, num_blocks=64, kv_heads=n_head, d=n_embd // n_head)
    x = torch.randn(3, max_len, n_embd, device="cuda")
    at = [100, 17, 60]  # prompt lengths

    plan = cache.extend(torch.tensor(at, dtype=torch.int32, device="cuda"), sum(at))
    layer.step(torch.cat([x[b, :n] for b, n in enumerate(at)]), cache, plan, max_new=max(at))
    one = torch.ones(3, dtype=torch.int32, device="cuda")
    for _ in range(steps):
        plan = cache.extend(one, 3)
        y = layer.step(torch.stack([x[b, n] for b, n in enumerate(at)]), cache, plan, max_new=1)
        at = [n + 1 for n in at]
        off = []
        for b, n in enumerate(at):
            with torch.no_grad():
                want = layer(x[b:b + 1, :n])[0, -1]
            off.append(float((y[b] - want).norm() / want.norm()))
        print("lengths %s: relative difference %s" % (cache.lens.tolist(), ", ".join("%.3f" % v for v in off)))
    cache.release(1)
    kint.check_status()
    print("blocks free after request 1 ended: %d of %d" % (int(cache.n_free), 64))


if __name__ == "__main__":
    main()
