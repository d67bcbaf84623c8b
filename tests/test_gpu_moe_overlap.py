"""Tensors of the operators for rows that go to different weights that lie in one
another's memory (run with -m gpu): columns beside columns give what separate tensors
do, a result over what is still read is refused."""
import pytest
import torch

import paper_2003_04296_amd as q

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    q.lib()
    return torch.device("cuda:0")


def _beside(dev, seed, rows, *widths):
    """Tensors of so many columns beside each other in one, bf16."""
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    t = torch.randn((rows, sum(widths)), generator=gen, device=dev).bfloat16()
    return t.split(list(widths), dim=1)


@pytest.mark.parametrize("m", [1, 20, 3000])
def test_adapters(dev, m):
    k = n = 72
    x, y, out = _beside(dev, 1, m, k, n, n)
    a, b = _beside(dev, 2, 3 * 8, k)[0].reshape(3, 8, k), _beside(dev, 3, 3 * n, 8)[0].reshape(3, n, 8)
    offsets, order, _ = q.moe_sort(torch.arange(m, device=dev) % 4, 3)
    want, _ = q.lora_forward(y.clone(), x.clone(), a, b, offsets, order)  # one row is contiguous as it is
    x0 = x.clone()
    got, _ = q.lora_forward(y, x, a, b, offsets, order, out=out)
    assert torch.equal(got, want) and torch.equal(x, x0)
    got, _ = q.lora_forward(y, x, a, b, offsets, order)
    assert torch.equal(got, want) and torch.equal(x, x0)
    c = x.contiguous()
    for call in (lambda: q.lora_forward(c, c, a, b, offsets, order), lambda: q.lora_forward(y, c, a, b, offsets, order, out=c),
                 lambda: q.lora_forward(y, x, a, b, offsets, order, out=x)):
        with pytest.raises(q.QconvError):
            call()
    assert torch.equal(x, x0) and torch.equal(c, x0)


def _same(a, b):
    for i, (u, v) in enumerate(zip(a, b, strict=True)):
        assert torch.equal(u, v), i


@pytest.mark.parametrize("tokens", [70, 9000])
def test_rows(dev, tokens):
    slots, w = 2, 40
    ids = torch.arange(tokens * slots, device=dev, dtype=torch.int32).view(tokens, slots) * 7 % 6
    offsets, order, place = want = q.moe_sort(ids, 5)
    # an id's place in the id's stead
    over = ids.clone()
    _same(q.moe_sort(over, 5, out=(torch.empty_like(offsets), torch.empty_like(order), over)), want)
    with pytest.raises(q.QconvError):
        q.moe_sort(ids, 5, out=(offsets, ids.view(-1), place))
    x, y, gy = _beside(dev, 1, tokens, w, w, w)
    c = x.contiguous()
    rows, grows, spare = _beside(dev, 2, tokens * slots, w, w, w)
    weights = torch.rand((tokens, slots), device=dev)
    named = place[place >= 0].long()
    got = q.moe_gather(x, place, out=rows)
    assert torch.equal(got[named], q.moe_gather(c, place)[named]) and torch.equal(x, c)
    want_y = q.moe_combine(rows.contiguous(), place, weights)
    _same([q.moe_combine(rows, place, weights, out=y)], [want_y])
    want = q.moe_combine_backward(gy.contiguous(), rows.contiguous(), place, weights)
    got = q.moe_combine_backward(gy, rows, place, weights, out=(grows, None))
    assert torch.equal(got[0][named], want[0][named]) and torch.equal(got[1], want[1])
    # over rows and weights themselves
    wc = weights.clone()
    got = q.moe_combine_backward(gy, rows, place, wc, out=(rows, wc))
    assert got[0] is rows and torch.equal(rows[named], want[0][named]) and torch.equal(wc, want[1])
    one = q.moe_sort(ids[:, 0], 6)[2]
    for call in (lambda: q.moe_gather(c, one, out=c), lambda: q.moe_combine(c, one, out=c),
                 lambda: q.moe_combine_backward(c, y, one, out=(c, None))):
        with pytest.raises(q.QconvError):
            call()
    assert torch.equal(x, c)


@pytest.mark.parametrize("rows", [30, 600])
def test_products(dev, rows):
    k = f = 64
    x, h, gh, spare = _beside(dev, 3, rows, k, f, f, k)
    w = _beside(dev, 4, 3 * f, k, k)
    wg, wu = w[0].unflatten(0, (3, f)), w[1].unflatten(0, (3, f))  # columns of one tensor
    offsets = torch.tensor([0, rows // 2, rows // 2, rows], dtype=torch.int32, device=dev)
    c = [t.contiguous() for t in (x, wg, wu, gh)]
    want, pre = q.moe_gated_forward(c[0], c[1], c[2], offsets, keep_pre=True)
    _same([q.moe_gated_forward(x, wg, wu, offsets, out=h)[0]], [want])
    grads = q.moe_gated_backward(*c[:3], offsets, pre, c[3])
    _same(q.moe_gated_backward(x, wg, wu, offsets, pre, gh), grads)
    linear = q.moe_linear_backward(c[0], c[1], offsets, c[3])
    # the gradient of x over what its products have no more use for
    over = c[3].clone()
    _same(q.moe_gated_backward(*c[:3], offsets, pre, over, out=(over, None, None)), grads)
    over = c[0].clone()
    _same([q.moe_linear_backward(over, c[1], offsets, c[3], need_w=False, out=(over, None))[0]], [linear[0]])
    for call in (lambda: q.moe_gated_forward(*c[:3], offsets, out=c[0]), lambda: q.moe_linear_forward(c[0], c[1], offsets, out=c[0]),
                 lambda: q.moe_gated_backward(*c[:3], offsets, pre, c[3], out=(c[0], None, None)),
                 lambda: q.moe_linear_backward(c[0], c[1], offsets, c[3], out=(c[3], None))):
        with pytest.raises(q.QconvError):
            call()
    assert torch.equal(x, c[0]) and torch.equal(gh, c[3])


def test_adapters_gradients(dev):
    m, k = 200, 48
    x, y, gy = _beside(dev, 5, m, k, k, k)
    a, b = _beside(dev, 6, 3 * 8, k)[0].reshape(3, 8, k), _beside(dev, 7, 3 * k, 8)[0].reshape(3, k, 8)
    offsets, order, _ = q.moe_sort(torch.arange(m, device=dev) % 4, 3)
    _, mid = q.lora_forward(y, x, a, b, offsets, order, keep_mid=True, out=torch.empty((m, k), dtype=x.dtype, device=dev))
    c = [x.contiguous(), gy.contiguous()]
    want = q.lora_backward(c[0], a, b, offsets, order, mid, c[1])
    _same(q.lora_backward(x, a, b, offsets, order, mid, gy), want)
    over = c[1].clone()
    _same([q.lora_backward(x, a, b, offsets, order, mid, over, need_w=False, out=(over, None, None))[0]], [want[0]])
    for out in ((c[0], None, None), (c[1], None, None)):
        with pytest.raises(q.QconvError):
            q.lora_backward(c[0], a, b, offsets, order, mid, c[1], out=out)
    assert torch.equal(c[0], x) and torch.equal(c[1], gy)
