"""Low-rank adapters of many requests (lora_forward, lora_backward) against their
formulas in 64 bits (run with -m gpu).

Bounds per value, with u half a step of the tensors' type (2^-11 fp16, 2^-8 bf16;
half the smallest subnormal absolutely) and e = 2^-23 for every fp32 operation:
  mid, p       sums of K products: (K + 8) e sum |x||a|
  operands     mid and p enter the second products in 16 leading bits: 2^-16 of
               them (two roundings of 2^-9 each: 2^-18, and 2^-17 for the rests'
               product that fp16 leaves out)
  out, gx      the errors of mid through the sum, the sum's own (rank + 8) e (three
               products a term: 3 rank), one more fp32 operation, u of the result
  ga, gb       the same with the sum over the adapter's tokens
"""
import pytest
import torch

import paper_2003_04296_amd as q

pytestmark = pytest.mark.gpu

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
E = 2.0 ** -23
PARTS = 2.0 ** -16


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    q.lib()
    return torch.device("cuda:0")


def _ids(dev, m, groups, how, gen):
    i = torch.arange(m, device=dev)
    if how == "mixed":
        ids = torch.randint(-1, groups, (m,), generator=gen, device=dev)
    elif how == "runs":
        ids = (i * 5 // max(m, 1)) * 7 % groups
    elif how == "one":
        ids = torch.full_like(i, groups - 1)
    else:  # none
        ids = torch.full_like(i, -1)
    return ids.int()


def _problem(dev, m, groups, rank, k, n, dtype, how, seed=0, big=1.0):
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed + m * 31 + k * 7 + n + rank)
    draw = lambda *s: torch.randn(s, generator=gen, device=dev)
    ids = _ids(dev, m, groups, how, gen)
    return dict(x=(draw(m, k) * big).to(dtype), y=draw(m, n).to(dtype), a=(draw(groups, rank, k) * k ** -0.5).to(dtype),
                b=(draw(groups, n, rank) * rank ** -0.5 / big).to(dtype), gy=(draw(m, n) * 0.5).to(dtype),
                scale=torch.rand((groups,), generator=gen, device=dev) + 0.5, ids=ids)


def _close(got, want, bound, what):
    assert got.shape == want.shape, what
    bad = ~((got.double() - want).abs() <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} values off, worst ratio " \
                          f"{float(((got.double() - want).abs() / bound).max()):.3g}"


def _product(a, b, ea=None):
    """(a b^T, its fp32 error, |ea| |b|^T if a is off by ea)."""
    v, n = a @ b.t().contiguous(), a.shape[1]
    err = (3 * n + 8) * E * (a.abs() @ b.abs().t().contiguous())
    return v, err if ea is None else err + (ea + PARTS * a.abs()) @ b.abs().t().contiguous() * 1.01


def _check(s, out, gx=None, ga=None, gb=None, scale=True):
    """All results, adapter by adapter."""
    r, tiny = U[s["x"].dtype], TINY[s["x"].dtype]
    groups = s["a"].shape[0]
    for e in [-1, *range(groups)]:
        at = torch.nonzero(s["ids"] == e).squeeze(1)
        if e < 0:
            assert torch.equal(out[at], s["y"][at])
            assert gx is None or not gx[at].any()
            continue
        if len(at) == 0:
            assert ga is None or not (ga[e].any() or gb[e].any()), e
            continue
        x, y, gy = (s[v][at].double() for v in ("x", "y", "gy"))
        a, b = s["a"][e].double(), s["b"][e].double()
        c = s["scale"][e].double() if scale else torch.ones((), dtype=torch.float64, device=x.device)
        mid, emid = _product(x, a)
        d, ed = _product(mid, b, emid)
        want = y + c * d
        _close(out[at], want, 1.01 * (c * ed + E * (c * d).abs() + E * want.abs() + r * want.abs()) + tiny, f"out of {e}")
        if gx is None and ga is None:
            continue
        p, ep = _product(gy, b.t().contiguous())
        if gx is not None:
            v, ev = _product(p, a.t().contiguous(), ep)
            _close(gx[at], c * v, 1.01 * (c * ev + (E + r) * (c * v).abs()) + tiny, f"gx of {e}")
        if ga is not None:
            v, ev = _product(p.t().contiguous(), x.t().contiguous(), ep.t())
            _close(ga[e], c * v, 1.01 * (c * ev + (E + r) * (c * v).abs()) + tiny, f"ga of {e}")
            v, ev = _product(mid.t().contiguous(), gy.t().contiguous(), emid.t())
            _close(gb[e], (c * v).t(), 1.01 * (c * ev + (E + r) * (c * v).abs()).t() + tiny, f"gb of {e}")


SIZES = [
    # m, groups, rank, k, n: one of each, odd ones, both sides of 16 and 32 tokens, of 16, 32, 64 ranks, of 128 inputs
    (1, 1, 1, 1, 1), (1, 3, 16, 4096, 4096), (2, 2, 3, 5, 7), (15, 4, 4, 127, 63), (16, 1, 8, 128, 64), (17, 5, 15, 129, 65),
    (31, 2, 17, 200, 300), (33, 40, 24, 640, 264), (64, 7, 32, 1000, 1001), (70, 3, 33, 256, 100), (100, 2, 64, 2048, 520),
    (129, 9, 65, 96, 200), (50, 2, 130, 72, 136), (40, 3, 256, 300, 257),
    # both sides of what one launch takes: 1024 inputs, 128 pieces, rank 64
    (90, 4, 16, 1025, 72), (20, 3, 33, 1032, 40), (1950, 6, 12, 64, 72), (2100, 6, 12, 64, 72), (30, 20, 20, 2500, 130),
]


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("how", ["mixed", "runs", "one", "none"])
@pytest.mark.parametrize("m,groups,rank,k,n", SIZES)
def test_forward_and_backward(dev, m, groups, rank, k, n, how, dtype):
    s = _problem(dev, m, groups, rank, k, n, TYPES[dtype], how)
    offsets, order, _ = q.moe_sort(s["ids"], groups)
    args = s["a"], s["b"], offsets, order
    out, mid = q.lora_forward(s["y"], s["x"], *args, s["scale"], keep_mid=True, out=torch.empty_like(s["y"]))
    gx, ga, gb = q.lora_backward(s["x"], *args, mid, s["gy"], s["scale"])
    _check(s, out, gx, ga, gb)
    # in place, and without mid; parts of the backward
    y = s["y"].clone()
    same, none = q.lora_forward(y, s["x"], *args, s["scale"])
    assert same is y and none is None and torch.equal(y, out)
    only_x = q.lora_backward(s["x"], *args, mid, s["gy"], s["scale"], need_w=False)
    only_w = q.lora_backward(s["x"], *args, mid, s["gy"], s["scale"], need_x=False)
    assert only_x[1] is None and only_x[2] is None and only_w[0] is None
    assert torch.equal(only_x[0], gx) and torch.equal(only_w[1], ga) and torch.equal(only_w[2], gb)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("m,groups,rank,k,n,how", [(8200, 5, 16, 264, 300, "runs"), (8200, 5, 24, 264, 300, "mixed"), (2050, 5, 40, 264, 300, "runs"), (5000, 3, 64, 200, 128, "mixed"),
                                                   (1500, 2, 20, 1100, 77, "one"), (513, 2, 8, 64, 72, "one"),
                                                   (4096, 300, 8, 128, 40, "mixed"), (6000, 4096, 4, 40, 24, "mixed")])
def test_many_tokens(dev, m, groups, rank, k, n, how, dtype):
    """The pieces of 32 tokens, and weight gradients summed in several pieces."""
    s = _problem(dev, m, groups, rank, k, n, TYPES[dtype], how)
    offsets, order, _ = q.moe_sort(s["ids"], groups)
    args = s["a"], s["b"], offsets, order
    out, mid = q.lora_forward(s["y"], s["x"], *args, None, keep_mid=True, out=torch.empty_like(s["y"]))
    _check(s, out, *q.lora_backward(s["x"], *args, mid, s["gy"]), scale=False)


@pytest.mark.parametrize("m", [20, 700])
@pytest.mark.parametrize("k,n,off,pad", [(61, 45, 1, 3), (96, 40, 0, 8), (130, 129, 4, 11)])
def test_rows_of_wider_tensors(dev, m, k, n, off, pad):
    """Row strides past the columns, odd addresses, NaN beside every row; what lies beside the results stays."""
    s = _problem(dev, m, 4, 9, k, n, torch.float16, "mixed")
    offsets, order, _ = q.moe_sort(s["ids"], 4)

    def inside(t, fill=float("nan")):
        b = torch.full((len(t) + 1, t.shape[1] + pad), fill, dtype=t.dtype, device=dev)
        b[:-1, off:off + t.shape[1]] = t
        return b, b[:-1, off:off + t.shape[1]]

    xs, gys = inside(s["x"])[1], inside(s["gy"])[1]
    store, ys = inside(s["y"], 7.0)
    args = s["a"], s["b"], offsets, order
    mid = torch.full((q.lib().qconv_lora_mid_floats(m, 9) + 64,), float("nan"), device=dev)
    out, mid = q.lora_forward(ys, xs, *args, s["scale"], mid=mid)
    assert out is ys
    _check(s, ys, *q.lora_backward(xs, *args, mid, gys, s["scale"]))
    mask = torch.ones_like(store, dtype=torch.bool)
    mask[:-1, off:off + n] = False
    assert bool((store[mask] == 7.0).all())


def test_fp16_sums_past_the_type(dev):
    """x a^T past fp16's 65504 and below its smallest value: results that fp16 holds are right."""
    for big in (1e4, 1e-3):
        s = _problem(dev, 90, 3, 12, 256, 72, torch.float16, "mixed", big=big)
        s["a"] = (s["a"].float() * (8 if big > 1 else 1e-3)).half()
        s["b"] = (s["b"].float() * (0.5 if big > 1 else 1)).half()
        offsets, order, _ = q.moe_sort(s["ids"], 3)
        out, mid = q.lora_forward(s["y"], s["x"], s["a"], s["b"], offsets, order, s["scale"], keep_mid=True,
                                  out=torch.empty_like(s["y"]))
        if big > 1:
            assert float(mid.view(-1, 12)[:int(offsets[3])].abs().max()) > 65504
        _check(s, out)


def test_nan_of_one_token_stays_with_it(dev):
    """A NaN in one token's row, or in an adapter that no token has, reaches no other token; the unused one's gradient is zero."""
    s = _problem(dev, 40, 4, 8, 64, 72, torch.bfloat16, "mixed")
    s["ids"] = torch.where(s["ids"] == 2, torch.zeros_like(s["ids"]), s["ids"])
    offsets, order, _ = q.moe_sort(s["ids"], 4)
    t = int(torch.nonzero(s["ids"] == 1)[0])
    x, a, b = s["x"].clone(), s["a"].clone(), s["b"].clone()
    x[t, 3], a[2], b[2] = float("nan"), float("nan"), float("inf")
    out, mid = q.lora_forward(s["y"], x, a, b, offsets, order, keep_mid=True, out=torch.empty_like(s["y"]))
    assert bool(torch.isnan(out[t]).all())
    clean, _ = q.lora_forward(s["y"], s["x"], s["a"], s["b"], offsets, order, out=torch.empty_like(s["y"]))
    rest = torch.arange(40, device=dev) != t
    assert torch.equal(out[rest], clean[rest])
    gx, ga, gb = q.lora_backward(x, a, b, offsets, order, mid, s["gy"])
    assert bool(torch.isfinite(gx).all()) and not ga[2].any() and not gb[2].any()
    assert bool(torch.isfinite(ga[0]).all()) and bool(torch.isnan(ga[1][:, 3]).all())


def test_indices_outside_the_tokens_are_passed_over(dev):
    """Tokens that are none, and offsets of no order: nothing outside the tensors is read or written."""
    s = _problem(dev, 30, 3, 8, 64, 72, torch.bfloat16, "mixed")
    offsets, order, _ = q.moe_sort(s["ids"], 3)
    bad = order.clone()
    bad[0], bad[5], bad[-1] = 30, -4, 0x7fffffff
    out, mid = q.lora_forward(s["y"], s["x"], s["a"], s["b"], offsets, bad, keep_mid=True, out=s["y"].clone())
    good, _ = q.lora_forward(s["y"], s["x"], s["a"], s["b"], offsets, order, out=torch.empty_like(s["y"]))
    named = torch.zeros(30, dtype=torch.bool, device=dev)
    named[bad[(bad >= 0) & (bad < 30)].long()] = True
    assert torch.equal(out[named], good[named]) and torch.equal(out[~named], s["y"][~named])
    q.lora_backward(s["x"], s["a"], s["b"], offsets, bad, mid, s["gy"])
    for o in ([0, 40, 10, 35], [-7, 1 << 30, 3, -1], [30, 20, 10, 0]):
        o = torch.tensor(o, dtype=torch.int32, device=dev)
        q.lora_forward(s["y"], s["x"], s["a"], s["b"], o, order, out=torch.empty_like(s["y"]))
        q.lora_backward(s["x"], s["a"], s["b"], o, order, torch.zeros_like(mid), s["gy"])
    torch.cuda.synchronize()


def test_gradients_against_differences(dev):
    """The gradients are those of sum(gy out): central differences of the formula in 64 bits along random directions."""
    s = _problem(dev, 24, 2, 6, 40, 48, torch.float16, "runs", seed=5)
    s["ids"] = s["ids"] % 2
    offsets, order, _ = q.moe_sort(s["ids"], 2)
    _, mid = q.lora_forward(s["y"], s["x"], s["a"], s["b"], offsets, order, s["scale"], keep_mid=True,
                            out=torch.empty_like(s["y"]))
    grads = q.lora_backward(s["x"], s["a"], s["b"], offsets, order, mid, s["gy"], s["scale"])
    base = [s[v].double() for v in ("x", "a", "b")]

    def loss(v):
        total = 0.0
        for e in range(2):
            at = s["ids"] == e
            total = total + s["scale"][e].double() * ((v[0][at] @ v[1][e].t() @ v[2][e].t()) * s["gy"][at].double()).sum()
        return total

    gen = torch.Generator(device=dev)
    gen.manual_seed(3)
    h = 1e-5
    for i in range(3):
        d = torch.randn(base[i].shape, generator=gen, device=dev, dtype=torch.float64)
        hi, lo = ([w + sign * h * d if j == i else w for j, w in enumerate(base)] for sign in (1, -1))
        slope = float(loss(hi) - loss(lo)) / (2 * h)  # linear in each
        # a gradient value carries one rounding of 2^-11 (and less of its terms), independent of d's signs
        assert abs(float((grads[i].double() * d).sum()) - slope) <= 6 * 2.0 ** -11 * float((grads[i].double() * d).norm()) + 1e-6, i


def test_no_tokens(dev):
    s = _problem(dev, 0, 3, 8, 32, 40, torch.bfloat16, "none")
    offsets, order, _ = q.moe_sort(s["ids"], 3)
    out, mid = q.lora_forward(s["y"], s["x"], s["a"], s["b"], offsets, order, keep_mid=True)
    assert out.shape == (0, 40) and mid.numel() == 0
    gx, ga, gb = q.lora_backward(s["x"], s["a"], s["b"], offsets, order, mid, s["gy"])
    assert gx.shape == (0, 32) and not ga.any() and not gb.any()
