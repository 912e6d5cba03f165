"""Host-side checks of the serving operators (no GPU needed): the ABI, its refusals, the rotation's angles, and the
plain forms that the GPU tests compare with."""
import ctypes
import math
import os
import re

import numpy as np
import pytest
import torch

from paper_2609_33591_gb300 import kint, serve
from tests import serve_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 256  # a pointer that is never followed: the checks come first


def test_header_declares_the_binding_exports():
    text = open(os.path.join(ROOT, "include", "kint_serve.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    assert sorted(set(re.findall(r"\b(kint_[a-z_]+)\s*\(", text))) == sorted(serve.EXPORTS)
    for name in serve.EXPORTS:
        assert hasattr(serve.load(), name), name


def heads(n=4, ptr=P):
    return serve.kint_heads(ptr, 0, n * 64, 64, n)


def cache(**kw):
    a = dict(pages=P, block_stride=2 * 4 * 18 * 64, num_blocks=8, block_size=32, kv_heads=4, d=64)
    a.update(kw)
    return serve.kint_cache(*a.values())


ATTN = dict(q=heads(), out=heads(), cache=cache(), table=P, stride=8, width=8, lens=P, cu=P, rows=2, B=2, window=0, sinks=0, Kint=4,
            calib=1, tau=8.0, recon=0, max_new=1, max_len=256, dtype=0, ws=P, bytes=1 << 40, stream=None)


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), -1), (dict(table=None), -1), (dict(stride=7), -1), (dict(width=0), -1), (dict(Kint=0), -1), (dict(Kint=65), -1),
    (dict(tau=0.0), -1), (dict(tau=math.inf), -1), (dict(calib=6), -1), (dict(recon=2), -1), (dict(dtype=3), -1),
    (dict(window=-1), -1), (dict(sinks=-1), -1), (dict(max_new=0), -1), (dict(rows=-1), -1), (dict(max_len=0), -1), (dict(max_len=257), -1),
    (dict(q=heads(6), out=heads(6)), -1), (dict(out=heads(8)), -1), (dict(q=heads(ptr=None)), -1), (dict(q=heads(ptr=P + 2)), -3),
    (dict(lens=P + 2), -3), (dict(cache=cache(d=96)), -2), (dict(cache=cache(block_size=48)), -2), (dict(cache=cache(block_size=8)), -2),
    (dict(cache=cache(num_blocks=0)), -1), (dict(cache=cache(block_stride=9200)), -1), (dict(cache=cache(block_stride=9224)), -3),
    (dict(cache=cache(pages=P + 8)), -3), (dict(bytes=64), -4), (dict(ws=None), -4), (dict(ws=P + 8), -3),
])
def test_attention_refusals(kw, code):
    assert serve.load().kint_cache_attn(*{**ATTN, **kw}.values()) == code


def test_attention_workspace():
    f = serve.load().kint_cache_attn_workspace_bytes
    assert f(2, 4, 4, 64, 0, 0, 1, 256) > 0
    assert f(2, 4, 4, 64, 0, 0, 1, 1 << 20) > f(2, 4, 4, 64, 0, 0, 1, 256)
    # a window bounds the scratch whatever the length
    assert f(2, 4, 4, 64, 128, 4, 1, 1 << 20) == f(2, 4, 4, 64, 128, 4, 1, 1 << 21)
    for bad in ((0, 4, 4, 64, 0, 0, 1, 256), (2, 6, 4, 64, 0, 0, 1, 256), (2, 4, 4, 96, 0, 0, 1, 256), (2, 4, 4, 64, 0, 0, 0, 256),
                (2, 4, 4, 64, -1, 0, 1, 256)):
        assert f(*bad) == 0


APPEND = dict(cache=cache(), k=heads(), v=heads(), slots=P, n=3, q=None, qo=None, pos=P, table=P, max_pos=64, rot=64, il=0, dtype=0,
              stream=None)


@pytest.mark.parametrize("kw,code", [
    (dict(k=heads(3)), -1), (dict(v=heads(3)), -1), (dict(slots=None), -1), (dict(slots=P + 4), -3), (dict(n=-1), -1),
    (dict(rot=63), -1), (dict(rot=66), -1), (dict(rot=0), -1), (dict(max_pos=0), -1), (dict(pos=None), -1), (dict(table=P + 4), -3),
    (dict(q=heads(8), qo=heads(4)), -1), (dict(q=heads(8), qo=heads(8), table=None), -1), (dict(dtype=-1), -1),
    (dict(cache=cache(kv_heads=0)), -1), (dict(cache=cache(d=80)), -2), (dict(k=heads(ptr=P + 2)), -3),
])
def test_append_refusals(kw, code):
    a = {**APPEND, **kw}
    assert serve.load().kint_cache_append(*a.values()) == code


def test_read_rope_and_block_refusals():
    lib = serve.load()
    assert lib.kint_cache_read(cache(), P, 3, None, None, 0, None) == -1
    assert lib.kint_cache_read(cache(), P, 3, heads(3), None, 0, None) == -1
    assert lib.kint_cache_read(cache(), P + 4, 3, heads(), None, 0, None) == -3
    rope = dict(q=heads(), qo=heads(), k=heads(), ko=heads(), pos=P, sb=0, table=P, max_pos=8, B=1, T=8, d=64, rot=64, il=0, inv=0,
                dtype=1, stream=None)
    for kw, code in ((dict(d=63), -1), (dict(d=258), -2), (dict(rot=65), -1), (dict(rot=128), -1), (dict(qo=heads(3)), -1),
                     (dict(ko=heads(3)), -1), (dict(T=-1), -1), (dict(dtype=5), -1), (dict(table=None), -1),
                     (dict(q=heads(0), qo=heads(0), k=heads(0), ko=heads(0)), -1), (dict(q=heads(ptr=P + 1)), -3)):
        assert lib.kint_rope(*{**rope, **kw}.values()) == code, kw
    freq = (ctypes.c_double * 32)()
    assert lib.kint_rope_table(P, 0, 64, freq, 1.0, None) == -1
    assert lib.kint_rope_table(P, 8, 63, freq, 1.0, None) == -1
    assert lib.kint_rope_table(P, 8, 64, freq, math.nan, None) == -1
    assert lib.kint_rope_table(P, 8, 258, freq, 1.0, None) == -2
    blocks = [P, P, P, 8, 8, P, 4, P, 2, 32, 6] + [P] * 7 + [None]
    for i, bad, code in ((0, None, -1), (3, 7, -1), (4, 0, -1), (6, -1, -1), (8, 0, -1), (8, 20000, -2), (9, 33, -2), (10, -1, -1),
                         (13, None, -1), (14, P + 4, -3), (0, P + 2, -3)):
        a = list(blocks)
        a[i] = bad
        assert lib.kint_blocks_extend(*a) == code, (i, bad)
    assert lib.kint_cache_block_bytes(32, 4, 64) == 2 * 4 * 18 * 64
    assert lib.kint_cache_block_bytes(40, 4, 64) == 0 and lib.kint_cache_block_bytes(32, 4, 80) == 0


def test_torch_entry_points_refuse_host_tensors():
    q, i = torch.zeros(2, 4, 64), torch.zeros(2, dtype=torch.int32)
    pages = torch.zeros(4, 4, 2, 18 * 64, dtype=torch.uint8)
    slots = torch.zeros(2, dtype=torch.int64)
    table = torch.zeros(8, 32, 2)
    for call in (lambda: serve.attention(q, pages, i[:, None], i, torch.zeros(3, dtype=torch.int32), kint.Config()),
                 lambda: serve.append(q, q, slots, pages), lambda: serve.read(pages, slots),
                 lambda: serve.rope(q[None], q[None], i, table), lambda: serve.rotary(q[None], q[None], i, table),
                 lambda: serve.extend_blocks(i, i, i[:, None], i, i[:1], 32, 4)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(kint.KintError):
        serve.cache_pages(4, 24, 4, 64, device="cpu")


def test_rotation_angles():
    f, mag = serve.rope_frequencies(64, 10000.0)
    assert mag == 1.0 and f[0] == 1.0 and math.isclose(f[31], 10000.0 ** (-62 / 64), rel_tol=1e-12)
    lin, _ = serve.rope_frequencies(64, scaling="linear", factor=4.0)
    assert all(math.isclose(a, b / 4) for a, b in zip(lin, f))
    base, _ = serve.rope_frequencies(64, scaling="base", factor=4.0)
    assert base[0] == 1.0 and math.isclose(base[31], f[31] / 4, rel_tol=1e-9)
    bands, mag = serve.rope_frequencies(64, scaling="bands", factor=8.0, original_len=4096)
    assert bands[0] == f[0] and math.isclose(bands[31], f[31] / 8) and math.isclose(mag, 0.1 * math.log(8) + 1)
    assert all(a <= b for a, b in zip(bands, f)) and all(a >= b / 8 * (1 - 1e-12) for a, b in zip(bands, f))
    for bad in (dict(rot=7), dict(rot=0), dict(rot=8, scaling="other"), dict(rot=8, factor=0.0)):
        with pytest.raises(ValueError):
            serve.rope_frequencies(**bad)


@pytest.mark.parametrize("d", [64, 128])
def test_plain_pack_holds_what_quantise_says(d):
    """Each code sits in a nibble of its own: unpacking by the header's offsets gives the codes back."""
    g = torch.Generator().manual_seed(3)
    k, v = torch.randn(16, d, generator=g), torch.randn(16, d, generator=g)
    slab = ref.pack(k, v).numpy()
    used = np.zeros((18 * d, 2), int)
    for x, is_v in ((k, 0), (v, 1)):
        code, s, c = ref.quantise(x)
        for j in range(16):
            for e in range(d):
                at = (9 * d + ((8 * (j // 2) + e // 8 % 8) * (d // 32) + 2 * (e // 64) + e // 4 % 2) * 4 + 2 * (j % 2) + e % 4 // 2 if is_v
                      else j * d // 2 + (e // 8 % 4) * d // 8 + 4 * (e // 32) + e % 8 // 2)
                used[at, e % 2] += 1
                assert (slab[at] >> (4 * (e % 2))) & 15 == code[j, e]
        # the kept numbers are within half a step of x, but for the rounding of s and c to fp16 (relative 2^-11 each:
        # the step's on up to 8 steps, the centre's on its own size)
        step = s.repeat_interleave(64, -1)
        centre = c.abs().repeat_interleave(64, -1)
        err = (ref.held(x) - x.double()).abs()
        assert (err <= 0.5 * step + 8 * step * 2 ** -11 + (centre + 8 * step) * 2 ** -11).all()
    assert (used.reshape(-1) <= 1).all() and used.sum() == 2 * 16 * d


def test_plain_weights_agree_with_the_oracle_definitions():
    """The plain attention's causal rows against the fp64 oracle of the training operator."""
    import oracle
    from tests import parity
    from paper_2609_33591_gb300.inputs import make_qkvdo
    Q, K, V, _ = make_qkvdo(1, 2, 40, 64, seed=5)
    for calib in range(6):
        for recon in (0, 1):
            cfg = kint.Config(Kint=4, calib=calib, tau=3.0, recon=recon)
            o = oracle.forward(Q, K, V, parity.to_oracle_cfg(cfg))["O"]
            k, v = (torch.from_numpy(x[0]).double().transpose(0, 1) for x in (K, V))
            q = torch.from_numpy(Q[0]).double().transpose(0, 1)
            got, safe = ref.attention(q, [k], [v], [40], [40], cfg)
            want = torch.from_numpy(o[0]).transpose(0, 1)
            assert safe.float().mean() > 0.5
            assert ((got - want).abs().amax(-1)[safe] <= 1e-9).all(), (calib, recon)
