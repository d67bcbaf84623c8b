"""The block of experts and the adapted projection (run with -m gpu).

The block's gradients are held against the same formulas in 64 bits from the same
16-bit weights and tokens, within bounds carried along the chain: r = 2^-8 for each
rounding to bf16 (h, the experts' rows, their gradients, dg and du, the results),
through every product by the magnitudes of its other factor, and 2^-14 of the sum
of a product's magnitudes for fp32 (at most 100 terms of 2^-23) and for the
products of two errors."""
import pytest
import torch

import paper_2003_04296_amd as q
from paper_2003_04296_amd import experts

pytestmark = pytest.mark.gpu
R = 2.0 ** -8


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    q.lib()
    return torch.device("cuda:0")


class Near:
    """A value in 64 bits and how far off it may be."""

    def __init__(self, v, e=None):
        self.v, self.e = v.double(), torch.zeros_like(v, dtype=torch.float64) if e is None else e

    def __matmul__(self, o):
        a, b = self.v.abs(), o.v.abs()
        return Near(self.v @ o.v, self.e @ b + a @ o.e + self.e @ o.e + 2.0 ** -14 * (a @ b))

    def __mul__(self, o):
        a, b = self.v.abs(), o.v.abs()
        return Near(self.v * o.v, self.e * b + a * o.e + self.e * o.e + 2.0 ** -14 * a * b)

    def t(self):
        return Near(self.v.t().contiguous(), self.e.t().contiguous())

    def rounded(self):
        return Near(self.v, self.e + R * (self.v.abs() + self.e))

    def check(self, got, what):
        off = (got.double() - self.v).abs()
        assert bool((off <= self.e * 1.01 + 1e-9).all()), (what, float((off / (self.e + 1e-9)).max()))


def _sum(parts):
    return Near(sum(p.v for p in parts), sum(p.e for p in parts))


def test_gradients_against_64_bits(dev):
    m, k, f, n, slots = 60, 40, 56, 5, 2
    block = experts.ExpertBlock(k, f, n, slots, device=dev, seed=3)
    gen = torch.Generator(device=dev)
    gen.manual_seed(1)
    x = torch.randn((m, k), generator=gen, device=dev).bfloat16()
    gy = (torch.randn((m, k), generator=gen, device=dev) * 0.1).bfloat16()
    y, saved = block.forward_train(x)
    ids, w = saved[1], saved[2]
    gx, (gwg, gwu, gwd, gr) = block.gradients(gy, saved)
    X, D = Near(x), Near(gy)
    ys = [[None] * m for _ in range(slots)]
    zero = lambda *s: Near(torch.zeros(s, device=dev))
    gxs = [zero(m, k) for _ in range(slots)]
    yp = [zero(m, k) for _ in range(slots)]
    gw = zero(m, slots)
    for e in range(n):
        wg, wu, wd = (Near(v[e]) for v in block.weights)
        grads = [[], [], []]
        for s in range(slots):
            at = ids[:, s] == e
            if not at.any():
                continue
            xs, c = Near(x[at]), Near(w[at, s:s + 1])
            g, u = xs @ wg.t(), xs @ wu.t()
            p = torch.sigmoid(g.v)
            # both are kept in fp32: the activation and its slope (at most 1.1, its own slope below 0.51) err as g does
            a = Near(g.v * p, 1.13 * g.e + 2.0 ** -14 * g.v.abs())
            slope = Near(p * (1 + g.v * (1 - p)), 0.51 * g.e + 2.0 ** -14)
            h = (a * u).rounded()
            out = (h @ wd.t()).rounded()
            yp[s].v[at], yp[s].e[at] = (c * out).v, (c * out).e
            gys = (c * Near(gy[at])).rounded()
            dot = Near(gy[at]) * out
            gw.v[at, s], gw.e[at, s] = dot.v.sum(1), dot.e.sum(1)
            gh = (gys @ wd).rounded()
            dg, du = (gh * u * slope).rounded(), (gh * a).rounded()
            back = _sum([dg @ wg, du @ wu]).rounded()
            gxs[s].v[at], gxs[s].e[at] = back.v, back.e
            for i, t in enumerate((dg.t() @ xs, du.t() @ xs, gys.t() @ h)):
                grads[i].append(t)
        for got, parts, what in zip((gwg, gwu, gwd), grads, ("gate", "up", "down")):
            if parts:
                _sum(parts).rounded().check(got[e], what)
            else:
                assert not got[e].any()
    _sum(yp).rounded().check(y, "y")
    W = Near(w, 2.0 ** -22 * w.double())
    inner = W * gw
    mean = Near(inner.v.sum(1, keepdim=True), inner.e.sum(1, keepdim=True))
    gs = W * Near(gw.v - mean.v, gw.e + mean.e)
    scores = zero(m, n)
    scores.v.scatter_(1, ids, gs.v)
    scores.e.scatter_(1, ids, gs.e)
    router = Near(block.masters[3])
    (scores.t() @ X).check(gr, "router")
    _sum([_sum(gxs).rounded(), scores @ router]).rounded().check(gx, "x")


def test_step(dev):
    block = experts.ExpertBlock(48, 64, 6, 2, device=dev, seed=5)
    x = torch.randn((70, 48), device=dev).bfloat16()
    y, saved = block.forward_train(x)
    assert torch.equal(block.forward(x), y)
    gy = torch.randn_like(y)
    gx, grads = block.gradients(gy, saved)
    before = [w.clone() for w in block.masters]
    again, norm = block.step(gy, saved, 0.5, 0.25)
    want = float(torch.cat([g.double().flatten() for g in grads]).norm())
    assert torch.equal(again, gx) and abs(float(norm) - want) <= 2.0 ** -22 * want and want > 0.25
    for b, w, g in zip(before, block.masters, grads):
        ref = (b.double() - 0.5 * 0.25 / want * g.double()).clamp(-1, 1)
        # the coefficient, the product, the difference: an fp32 rounding each
        assert bool(((w.double() - ref).abs() <= 2.0 ** -22 * (b.double().abs() + 0.5 * 0.25 / want * g.double().abs())).all())
    for w, master in zip(block.weights, block.masters):
        assert torch.equal(w, master.to(w.dtype))


def test_example_runs(dev):
    block, losses = experts.train(steps=6, device=dev)
    assert len(losses) == 6 and all(v == v for v in losses)
    experts.main()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_adapted_projection(dev, dtype):
    """Requests together and one by one: the shared projection's own result plus each one's adapter."""
    gen = torch.Generator(device=dev)
    gen.manual_seed(2)
    draw = lambda *s: torch.randn(s, generator=gen, device=dev)
    n, k, adapters, rank = 200, 320, 6, 12
    layer = experts.AdaptedProjection(draw(n, k) * k ** -0.5, (draw(adapters, rank, k) * k ** -0.5).to(dtype),
                                      (draw(adapters, n, rank) * rank ** -0.5).to(dtype), torch.rand(adapters, device=dev))
    ids = torch.randint(-1, adapters, (90,), generator=gen, device=dev)
    x = draw(90, k).to(dtype)
    y = layer.forward(x, layer.plan(ids))
    base = q.q4_linear(x, *layer.packed)
    u = torch.finfo(dtype).eps / 2
    for t in range(90):
        e = int(ids[t])
        if e < 0:
            assert torch.equal(y[t], base[t])
            continue
        a, b, c = layer.a[e].double(), layer.b[e].double(), layer.scale[e].double()
        mid = a @ x[t].double()
        want = base[t].double() + c * (b @ mid)
        # mid: 320 terms in fp32, then its leading 16 bits; the result's rounding
        off = 2.0 ** -14 * c * (b.abs() @ (a.abs() @ x[t].double().abs())) + 2.0 ** -15 * c * (b.abs() @ mid.abs())
        assert bool(((y[t].double() - want).abs() <= off + 1.01 * u * want.abs() + 2.0 ** -25).all()), t
        alone = layer.forward(x[t:t + 1], layer.plan(ids[t:t + 1]))[0]
        # one token's projection sums in another order: an fp32 sum of 320 terms, two roundings
        ref = q.q4_linear(x[t:t + 1], *layer.packed)[0]
        want = ref.double() + c * (b @ mid)
        assert bool(((alone.double() - want).abs() <= off + 1.01 * u * want.abs() + 2.0 ** -25).all()), t
