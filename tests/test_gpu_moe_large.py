"""Tensors of more than 2^31 values in the operators for rows that go to different
weights (run with -m gpu): results at the ends of the tensors against 64 bits, with
the bounds of the smaller tests."""
import pytest
import torch

import paper_2003_04296_amd as q
from test_gpu_lora import _product
from test_gpu_moe_products import _linear, _close

pytestmark = pytest.mark.gpu
R = 2.0 ** -8
W = 4096
N = 600_000  # rows of W values: 2.46e9


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    if torch.cuda.mem_get_info()[1] < 100 << 30:
        pytest.skip("too little memory")
    q.lib()
    yield torch.device("cuda:0")
    torch.cuda.empty_cache()


def _draw(dev, seed, *shape):
    """bf16 values in (-1, 1), made without wider copies."""
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    return torch.empty(shape, dtype=torch.bfloat16, device=dev).uniform_(-1, 1, generator=gen)


def _some(n, dev):
    return torch.cat([torch.arange(20), torch.arange(n // 2, n // 2 + 20), torch.arange(n - 20, n)]).to(dev)


def test_rows(dev):
    tokens, slots = N // 2, 2
    ids = torch.arange(tokens, device=dev).view(-1, 1) % 3 + torch.tensor([[0, 1]], device=dev)
    _, _, place = q.moe_sort(ids, 4)
    x, at = _draw(dev, 1, tokens, W), _some(tokens, dev)
    rows = q.moe_gather(x, place)
    to = place[at].long()
    assert int(to.max()) * W > 2 ** 31
    assert torch.equal(rows[to[:, 0]], x[at]) and torch.equal(rows[to[:, 1]], x[at])
    w = torch.rand((tokens, slots), device=dev)
    y = q.moe_combine(rows, place, w)
    want = x[at].double() * w[at].double().sum(1, keepdim=True)
    assert bool(((y[at].double() - want).abs() <= 1.01 * R * want.abs() + 2.0 ** -21 * x[at].double().abs()).all())
    _, gw = q.moe_combine_backward(y, rows, place, w, out=(rows.clone(), None))
    want = (y[at].double() * x[at].double()).sum(1)
    bound = (W + 1) * 2.0 ** -24 * (y[at].double() * x[at].double()).abs().sum(1)
    assert bool(((gw[at].double() - want.unsqueeze(1)).abs() <= bound.unsqueeze(1)).all())


def test_products_of_many_rows(dev):
    counts = [N // 2 + 5, 0, N // 2 - 100]
    offsets = torch.tensor([0, counts[0], counts[0], sum(counts)], dtype=torch.int32, device=dev)
    x, w, gy = _draw(dev, 1, N, W), _draw(dev, 2, 3, 40, W), _draw(dev, 3, N, 40)
    y = q.moe_linear_forward(x, w, offsets)
    gx, gw = q.moe_linear_backward(x, w, offsets, gy)
    for e, (i, j) in ((0, (0, counts[0])), (2, (counts[0], sum(counts)))):
        at = i + _some(j - i, dev)
        want = _linear(x[at], w[e], gy[at])
        _close(y[at], *want[0], "y")
        _close(gx[at], *want[1], "gx")
        # the sums over the rows, in pieces
        total = mags = 0
        for b in range(i, j, 50_000):
            g, v = gy[b:min(j, b + 50_000)].double().t().contiguous(), x[b:min(j, b + 50_000)].double()
            total, mags = total + g @ v, mags + g.abs() @ v.abs()
        _close(gw[e], total, (j - i + 8) * 2.0 ** -23 * mags + 1.01 * R * total.abs(), "gw")
    assert not gw[1].any()


@pytest.mark.parametrize("rows", [300, 900])
def test_products_of_many_weights(dev, rows):
    groups = 145
    x, w, gy = _draw(dev, 1, rows, W), _draw(dev, 2, groups, W, W), _draw(dev, 3, rows, W)
    offsets = (torch.arange(groups + 1, device=dev) * rows // groups).int()
    y = q.moe_linear_forward(x, w, offsets)
    gx, gw = q.moe_linear_backward(x, w, offsets, gy)
    for e in (0, 70, groups - 1):
        i, j = int(offsets[e]), int(offsets[e + 1])
        for got, (v, bound), what in zip((y[i:j], gx[i:j], gw[e]), _linear(x[i:j], w[e], gy[i:j]), ("y", "gx", "gw")):
            _close(got, v, bound, f"{what} of group {e}")


def test_adapters_of_many_tokens(dev):
    groups, rank = 3, 8
    ids = (torch.arange(N, device=dev) * 4 // N).int()
    ids = torch.where(ids == 3, torch.full_like(ids, -1), ids)
    offsets, order, _ = q.moe_sort(ids, groups)
    x, y, gy = _draw(dev, 1, N, W), _draw(dev, 2, N, W), _draw(dev, 3, N, W)
    a, b = _draw(dev, 4, groups, rank, W), _draw(dev, 5, groups, W, rank)
    keep = y[_some(N, dev)].clone()
    at = _some(N, dev)
    _, mid = q.lora_forward(y, x, a, b, offsets, order, keep_mid=True)
    gx, ga, gb = q.lora_backward(x, a, b, offsets, order, mid, gy)
    for n, t in enumerate(at.tolist()):
        e = int(ids[t])
        if e < 0:
            assert torch.equal(y[t], keep[n]) and not gx[t].any()
            continue
        A, B = a[e].double(), b[e].double()
        m, em = _product(x[t:t + 1].double(), A)
        d, ed = _product(m, B, em)
        want = keep[n].double() + d
        _close(y[t:t + 1], want, 1.01 * (ed + 2.0 ** -22 * d.abs() + R * want.abs()), f"out of {t}")
        p, ep = _product(gy[t:t + 1].double(), B.t().contiguous())
        v, ev = _product(p, A.t().contiguous(), ep)
        _close(gx[t:t + 1], v, 1.01 * (ev + R * v.abs()), f"gx of {t}")
    e, rows = 2, order[int(offsets[2]):int(offsets[3])].long()
    A, B = a[e].double(), b[e].double()
    sa = sb = ma = mb = 0
    for c in rows.split(25_000):
        X, G = x[c].double(), gy[c].double()
        p, ep = _product(G, B.t().contiguous())
        m, em = _product(X, A)
        sa, sb = sa + p.t().contiguous() @ X, sb + G.t().contiguous() @ m
        # per term: the factor's own error and its 16 leading bits, and the fp32 sum over all tokens
        own = lambda v, ev: ev + (2.0 ** -16 + 2.0 ** -23 * 3 * len(rows)) * v.abs()
        ma, mb = ma + own(p, ep).t().contiguous() @ X.abs(), mb + G.abs().t().contiguous() @ own(m, em)
    _close(ga[e], sa, 1.01 * (ma + R * sa.abs()), "ga")
    _close(gb[e], sb, 1.01 * (mb + R * sb.abs()), "gb")
