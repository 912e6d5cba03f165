"""GPU: the serving operators next to autograd: derivatives of the rotation of every order and type, and what is not
differentiable, or writes into its arguments, says so."""
import pytest
import torch

from paper_2609_33591_gb300 import kint, serve
from tests import serve_ref as ref
from tests.test_gpu_serve import BF16, F16, F32, HALF_UNIT, SOFT, _clean, _lib, filled, gpu, ints  # noqa: F401

pytestmark = pytest.mark.gpu


def plain(x, pos, table, interleaved):
    """The rotation in elementary torch operations, x and table in 64 bits, differentiable."""
    half = table.size(1)
    cs = table[pos.long()][:, :, None]
    i = torch.arange(half, device=x.device)
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    a, b = x[..., ia], x[..., ib]
    y = torch.empty_like(x)
    y[..., 2 * half:] = x[..., 2 * half:]
    y[..., ia], y[..., ib] = a * cs[..., 0] - b * cs[..., 1], b * cs[..., 0] + a * cs[..., 1]
    return y


@pytest.mark.parametrize("interleaved", [False, True])
def test_second_derivatives_of_the_rotation(interleaved):
    """L = sum c * dL1/dq with L1 = sum(a^3) + sum(a b): what goes through the rotation twice counts.  All fp32; each number is
    a sum of a few products of at most three rotated channels, so 2^-18 of the largest."""
    table = serve.rope_table(40, 48)
    pos = torch.randint(0, 40, (2, 6), device="cuda").int()
    q, k, c = (torch.randn(2, 6, 3, 64, device="cuda") for _ in range(3))

    def second(q, k, c, turn):
        q, k = q.clone().requires_grad_(), k.clone().requires_grad_()
        a, b = turn(q, k)
        g, = torch.autograd.grad((a ** 3).sum() + (a * b).sum(), q, create_graph=True)
        return torch.autograd.grad((g * c).sum(), (q, k))

    got = second(q, k, c, lambda q, k: serve.rotary(q, k, pos, table, interleaved))
    want = second(q.double(), k.double(), c.double(), lambda q, k: tuple(plain(x, pos, table.double(), interleaved) for x in (q, k)))
    for x, y in zip(got, want):
        assert (x.double() - y).abs().max() <= 2.0 ** -18 * y.abs().max()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("interleaved", [False, True])
def test_gradients_of_every_type(dtype, interleaved):
    table = serve.rope_table(40, 64)
    pos = torch.randint(0, 40, (1, 9), device="cuda").int()
    q, k = (torch.randn(1, 9, h, 64, device="cuda").to(dtype).requires_grad_() for h in (4, 2))
    c = [torch.randn_like(x) for x in (q, k)]
    grads = torch.autograd.grad(serve.rotary(q, k, pos, table, interleaved), (q, k), c)
    for g, x in zip(grads, c):
        want = ref.rotate(x.cpu(), pos.cpu(), table.cpu(), 64, interleaved, inverse=True)
        size = 2 * x.detach().cpu().double().abs().amax(-1, keepdim=True)
        assert g.dtype == dtype and ((g.cpu().double() - want).abs() <= HALF_UNIT[dtype] * want.abs() + 3 * 2.0 ** -24 * size).all()
    # a gradient that one number is spread from (no strides of its own)
    g, = torch.autograd.grad(serve.rotary(q, k, pos, table, interleaved)[0].sum(), q)
    want = ref.rotate(torch.ones(1, 9, 4, 64), pos.cpu(), table.cpu(), 64, interleaved, inverse=True)
    assert ((g.cpu().double() - want).abs() <= HALF_UNIT[dtype] * want.abs() + 6 * 2.0 ** -24).all()


@pytest.mark.parametrize("interleaved", [False, True])
def test_queries_alone(interleaved):
    """rotary without keys, forward and back."""
    table = serve.rope_table(40, 64)
    pos = torch.randint(0, 40, (7,), device="cuda").int()
    q = torch.randn(2, 7, 3, 64, device="cuda", requires_grad=True)
    c = torch.randn(2, 7, 3, 64, device="cuda")
    a, none = serve.rotary(q, None, pos, table, interleaved)
    assert none is None and torch.equal(a, serve.rope(q.detach(), None, pos, table, interleaved=interleaved)[0])
    a.backward(c)
    assert torch.equal(q.grad, serve.rope(c, None, pos, table, interleaved=interleaved, inverse=True)[0])


def test_writing_into_an_argument_counts_as_a_change_of_it():
    """Autograd notices that a tensor it saved was overwritten."""
    table, pos = serve.rope_table(8, 64), ints([0, 1, 2])
    pages, slots = serve.cache_pages(2, 16, 2, 64), ints([0, 1, 2], torch.int64)
    x = torch.randn(3, 2, 64, device="cuda")
    q, k, o = x.clone()[None], x.clone()[None], torch.empty_like(x)
    blocks, free = torch.full((1, 2), -1, dtype=torch.int32, device="cuda"), ints([0, 1])

    def changed(t, call):
        before = t._version
        call()
        return t._version > before

    assert changed(q, lambda: serve.rope(q, k, pos, table, out=(q, k)))
    assert changed(k, lambda: serve.rope(q, k, pos, table, out=(q, k)))
    assert changed(pages, lambda: serve.append(x, x, slots, pages))
    assert changed(o, lambda: serve.append(x, x, slots, pages, q=x, q_out=o, pos=pos, table=table))
    assert changed(o, lambda: serve.attention(x, pages, ints([[0, 1]]), ints([3]), ints([0, 3]), kint.Config(calib=SOFT), out=o))
    assert changed(blocks, lambda: serve.extend_blocks(ints([0]), ints([3]), blocks, free, ints([2]), 16, 3))
    assert not changed(x, lambda: serve.rope(x[None], None, pos, table))
    w = torch.randn_like(q).requires_grad_()
    y = w * q
    serve.rope(q, k, pos, table, out=(q, k))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    with torch.inference_mode():
        t = x.clone()
        assert torch.equal(serve.rope(t[None], None, pos, table, out=(t[None], None))[0][0],
                           serve.rope(x[None], None, pos, table)[0][0])


def test_what_is_not_differentiable_says_so():
    """Results of inputs that require gradients are the same numbers; asking for the gradient raises.  Without gradients asked
    for, nothing is recorded."""
    table, pos = serve.rope_table(8, 64), ints([0, 1, 2])
    pool = filled([16], 2, 64, 32, 3)
    pages, slots = gpu(pool.pages), ints([13, 14, 15], torch.int64)
    x = torch.randn(3, 2, 64, device="cuda")
    attend = lambda q, **kw: serve.attention(q, pages, gpu(pool.table), gpu(pool.lens), ints([0, 3]), kint.Config(), **kw)  # noqa: E731
    turn = lambda q, **kw: serve.rope(q[None], None, pos, table, **kw)[0]  # noqa: E731
    turn_k = lambda k: serve.rope(x[None], k[None], pos, table)[1]  # noqa: E731
    append = lambda q, **kw: serve.append(x, x, slots, pages, q=q, pos=pos, table=table, **kw)  # noqa: E731
    for call in (attend, turn, turn_k, append):
        leaf = x.clone().requires_grad_()
        y = call(leaf)
        assert torch.equal(y.detach(), call(x)) and y.requires_grad and not call(x).requires_grad
        with pytest.raises(RuntimeError, match="not implemented"):
            y.sum().backward()
        with torch.no_grad():
            assert not call(leaf).requires_grad
    for call, out in ((attend, torch.empty_like(x)), (append, None), (turn, (torch.empty_like(x)[None], None))):
        kw = dict(q_out=torch.empty_like(x)) if out is None else dict(out=out)
        with pytest.raises(ValueError):
            call(x.clone().requires_grad_(), **kw)
    w = x.clone().requires_grad_()
    with pytest.raises(ValueError):  # into what gradients are asked of
        attend(x, out=w)
    assert torch.equal(w.detach(), x)
