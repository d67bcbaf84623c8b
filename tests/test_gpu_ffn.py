"""The gated feed-forward block (ffn_forward / ffn_backward) against its
formulas in 64 bits (run with -m gpu).

Bounds per value, with u = 2^-11 (fp16) or 2^-8 (bf16) a rounding to the
tensors' type (half an ulp relative to the value, half the smallest
subnormal absolutely) and e = 2^-23 for every fp32 operation, whatever order
the sums take:
  sum of K products       |d| <= (K + 8) e sum |x||w|
  h = act(g) u            |act'| <= 1.13: 1.13 dg (|u| + du) + |act(g)| du,
                          16 e (|g| + |act(g)|) |u| for the activation itself,
                          u |h| for the result
  dg, du                  rounded once: u, plus 16 e (1 + |g|) |gh||u| (the
                          slope's own rounding); the backward's reference
                          starts from the kernel's pre, which is its input
  gx, gw                  the factors' errors through the sum, the sum's own,
                          and u of the result
"""
import math

import pytest
import torch

import paper_2003_04296_amd as q

pytestmark = pytest.mark.gpu

ACTS = {"silu": q.ACT_SILU, "gelu": q.ACT_GELU, "relu": q.ACT_RELU}
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
E = 2.0 ** -23


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    q.lib()
    return torch.device("cuda:0")


def _gate(g, act):
    """act(g), act'(g) in 64 bits."""
    if act == "relu":
        return g.clamp_min(0), (g > 0).double()
    if act == "silu":
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * (1 - p))
    c = 0.5 * torch.erfc(-g / math.sqrt(2))
    return g * c, c + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)


def _normal(gen, shape, std, dtype, dev, wide=0):
    t = torch.randn((shape[0], shape[1] + wide), generator=gen, device=dev) * std
    return t.to(dtype)[:, :shape[1]]


def _problem(dev, m, k, f, dtype, wide=0, seed=0):
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed + m * 31 + k * 7 + f)
    return (_normal(gen, (m, k), 1.0, dtype, dev, wide), _normal(gen, (f, k), k ** -0.5, dtype, dev),
            _normal(gen, (f, k), k ** -0.5, dtype, dev), _normal(gen, (m, f), 0.5, dtype, dev, wide))


def _close(got, want, bound, what):
    assert got.shape == want.shape, what
    bad = ~((got.double() - want).abs() <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} values off, worst ratio " \
                          f"{float(((got.double() - want).abs() / bound).max()):.3g}"


def _check_forward(h, pre, x, wg, wu, act):
    m, k = x.shape
    f = wg.shape[0]
    X, G, Uw = x.double(), wg.double(), wu.double()
    g, u = X @ G.t(), X @ Uw.t()
    dg, du = ((k + 8) * E * (X.abs() @ w.abs().t()) for w in (G, Uw))
    a, _ = _gate(g, act)
    want = a * u
    r = U[x.dtype]
    _close(h, want, 1.13 * dg * (u.abs() + du) + (a.abs() + 1.13 * dg) * du + 16 * E * (g.abs() + a.abs()) * u.abs()
           + r * want.abs() * 1.01 + TINY[x.dtype] + 1e-37, "h")
    if pre is not None:
        fp = (f + 7) // 8 * 8
        p = pre[:m * 2 * fp].view(m, 2, fp)
        _close(p[:, 0, :f], g, dg + 1e-37, "pre gate")
        _close(p[:, 1, :f], u, du + 1e-37, "pre up")


def _check_backward(gx, gg, gu, x, wg, wu, pre, gh, act):
    m, k = x.shape
    f = wg.shape[0]
    fp = (f + 7) // 8 * 8
    p = pre[:m * 2 * fp].view(m, 2, fp)
    g, u = p[:, 0, :f].double(), p[:, 1, :f].double()
    X, G, Uw, D = x.double(), wg.double(), wu.double(), gh.double()
    a, s = _gate(g, act)
    dg, du = D * u * s, D * a
    r, tiny = U[x.dtype], TINY[x.dtype]
    eg = 1.01 * r * dg.abs() + tiny + 16 * E * (1 + g.abs()) * (D * u).abs()
    eu = 1.01 * r * du.abs() + tiny + 16 * E * (g.abs() + a.abs()) * D.abs()
    if gx is not None:
        want = dg @ G + du @ Uw
        _close(gx, want, eg @ G.abs() + eu @ Uw.abs()
               + (2 * f + 8) * E * ((dg.abs() + eg) @ G.abs() + (du.abs() + eu) @ Uw.abs())
               + 1.01 * r * want.abs() + tiny, "gx")
    for got, d, e, what in ((gg, dg, eg, "gw_gate"), (gu, du, eu, "gw_up")):
        if got is not None:
            want = d.t() @ X
            _close(got, want, e.t() @ X.abs() + (m + 8) * E * ((d.abs() + e).t() @ X.abs()) + 1.01 * r * want.abs()
                   + tiny, what)


SIZES = [
    # m, k, f: one token, one feature, odd ones, both sides of 64 and 128, several tiles
    (1, 1, 1), (1, 64, 64), (1, 4096, 520), (2, 7, 9), (3, 129, 65), (16, 64, 200), (17, 1000, 33), (63, 72, 127),
    (64, 128, 128), (65, 200, 136), (127, 63, 64), (128, 256, 192), (129, 1001, 129), (200, 136, 1023),
    (257, 264, 300), (1000, 96, 80), (300, 2048, 64), (70, 520, 2049),
]


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("act", sorted(ACTS))
@pytest.mark.parametrize("m,k,f", SIZES)
def test_forward_and_backward(dev, m, k, f, act, dtype):
    x, wg, wu, gh = _problem(dev, m, k, f, TYPES[dtype])
    h, pre = q.ffn_forward(x, wg, wu, ACTS[act], keep_pre=True)
    _check_forward(h, pre, x, wg, wu, act)
    gx, gg, gu = q.ffn_backward(x, wg, wu, pre, gh, ACTS[act])
    _check_backward(gx, gg, gu, x, wg, wu, pre, gh, act)
    # without pre the forward gives the same h; parts of the backward give the same parts
    assert torch.equal(q.ffn_forward(x, wg, wu, ACTS[act])[0], h)
    only_x = q.ffn_backward(x, wg, wu, pre, gh, ACTS[act], need_w=False)
    only_w = q.ffn_backward(x, wg, wu, pre, gh, ACTS[act], need_x=False)
    assert only_x[1] is None and only_x[2] is None and only_w[0] is None
    assert torch.equal(only_x[0], gx) and torch.equal(only_w[1], gg) and torch.equal(only_w[2], gu)


@pytest.mark.parametrize("wide", [1, 3, 8, 64])
@pytest.mark.parametrize("m,k,f", [(5, 64, 72), (130, 200, 129), (40, 99, 256)])
def test_rows_of_wider_tensors(dev, m, k, f, wide):
    """x, gh and h with row strides past their columns, weights as a slice that starts at an odd address."""
    x, wg, wu, gh = _problem(dev, m, k, f, torch.bfloat16, wide)
    both = torch.empty((2 * f, k + 2 * wide), dtype=torch.bfloat16, device=dev)
    both[:f, wide:wide + k], both[f:, wide:wide + k] = wg, wu
    wg, wu = both[:f, wide:wide + k], both[f:, wide:wide + k]
    store = torch.full((m, f + wide), 7.0, dtype=torch.bfloat16, device=dev)
    h, pre = q.ffn_forward(x, wg, wu, q.ACT_SILU, keep_pre=True, out=store[:, :f])
    _check_forward(h, pre, x, wg, wu, "silu")
    assert bool((store[:, f:] == 7.0).all())
    gx, gg, gu = q.ffn_backward(x, wg, wu, pre, gh, q.ACT_SILU)
    _check_backward(gx, gg, gu, x, wg, wu, pre, gh, "silu")


@pytest.mark.parametrize("k", [96, 61])
@pytest.mark.parametrize("off_x,off_g,off_u,pad", [(4, 4, 4, 8), (4, 0, 0, 8), (0, 0, 4, 8), (0, 0, 4, 3), (1, 2, 3, 5),
                                                   (0, 0, 0, 3), (0, 8, 4, 11)])
def test_operands_aligned_differently(dev, k, off_x, off_g, off_u, pad):
    """Each operand at an address of its own, with row strides that are and are not multiples of 16 bytes, NaN beside
    every row: more tokens than the kernels for few take."""
    m, f = 150 if off_x else 390, 137
    x, wg, wu, gh = _problem(dev, m, k, f, torch.float16)
    ld = (k + 8 + 7) // 8 * 8 + pad

    def put(t, off, stride):
        b = torch.full(((t.shape[0] + 1) * stride,), float("nan"), dtype=t.dtype, device=dev)
        v = b[off:].as_strided(t.shape, (stride, 1), b.storage_offset() + off)
        v.copy_(t)
        return v

    xs, gs, us = put(x, off_x, ld), put(wg, off_g, ld), put(wu, off_u, ld)
    h, pre = q.ffn_forward(xs, gs, us, q.ACT_SILU, keep_pre=True)
    _check_forward(h, pre, x, wg, wu, "silu")
    gx, gg, gu = q.ffn_backward(xs, gs, us, pre, gh, q.ACT_SILU)
    _check_backward(gx, gg, gu, x, wg, wu, pre, gh, "silu")
    assert torch.equal(q.ffn_backward(xs, gs, us, pre, gh, q.ACT_SILU, need_w=False)[0], gx)
    assert torch.equal(q.ffn_backward(xs, gs, us, pre, gh, q.ACT_SILU, need_x=False)[1], gg)


def test_values_past_the_ends_are_not_read(dev):
    """NaN in a row's columns past k, in the rows after the last and in the pre buffer's padding reaches no result."""
    m, k, f = 37, 61, 45
    x, wg, wu, gh = _problem(dev, m, k, f, torch.float16)

    def inside(t):
        b = torch.full((t.shape[0] + 3, t.shape[1] + 5), float("nan"), dtype=t.dtype, device=dev)
        b[:t.shape[0], :t.shape[1]] = t
        return b[:t.shape[0], :t.shape[1]]

    xs, gs, us, ds = inside(x), inside(wg), inside(wu), inside(gh)
    pre = torch.full((q.lib().qconv_ffn_pre_floats(m, f) + 64,), float("nan"), device=dev)
    h, pre = q.ffn_forward(xs, gs, us, q.ACT_GELU, pre=pre)
    _check_forward(h, pre, x, wg, wu, "gelu")
    out = q.ffn_backward(xs, gs, us, pre, ds, q.ACT_GELU)
    _check_backward(*out, x, wg, wu, pre, gh, "gelu")


@pytest.mark.parametrize("act", sorted(ACTS))
def test_gradient_against_differences(dev, act):
    """The gradients are those of sum(h * c): central differences of the formula in 64 bits along a random direction."""
    m, k, f = 24, 40, 48
    x, wg, wu, gh = _problem(dev, m, k, f, torch.float16, seed=5)
    _, pre = q.ffn_forward(x, wg, wu, ACTS[act], keep_pre=True)
    grads = q.ffn_backward(x, wg, wu, pre, gh, ACTS[act])
    base = [t.double() for t in (x, wg, wu)]

    def loss(p):
        g, u = p[0] @ p[1].t(), p[0] @ p[2].t()
        return (_gate(g, act)[0] * u * gh.double()).sum()

    gen = torch.Generator(device=dev)
    gen.manual_seed(3)
    step = 1e-6
    for i in range(3):
        v = torch.randn(base[i].shape, generator=gen, device=dev, dtype=torch.float64)
        hi, lo = ([b + s * step * v if j == i else b for j, b in enumerate(base)] for s in (1, -1))
        slope = float((loss(hi) - loss(lo)) / (2 * step))
        got = float((grads[i].double() * v).sum())
        # each gradient value carries about two roundings of 2^-11, independent of v's signs
        scale = float((grads[i].double() * v).norm())
        assert abs(got - slope) <= 6 * 2.0 ** -11 * scale + 1e-5 * abs(slope) + 1e-6, (i, got, slope, scale)


def test_no_tokens(dev):
    x, wg, wu, gh = _problem(dev, 0, 33, 20, torch.bfloat16)
    h, pre = q.ffn_forward(x, wg, wu, keep_pre=True)
    assert h.shape == (0, 20) and pre.numel() == 0
    gx, gg, gu = q.ffn_backward(x, wg, wu, pre, gh)
    assert gx.shape == (0, 33)
    assert not gg.any() and not gu.any() and gg.shape == gu.shape == (20, 33)


@pytest.mark.parametrize("act", sorted(ACTS))
def test_infinities_and_nan_follow_the_formula(dev, act):
    """A NaN token gives NaN in its row alone; large inputs saturate as the formula does."""
    x, wg, wu, gh = _problem(dev, 40, 64, 72, torch.bfloat16)
    x[7, 3] = float("nan")
    x[9] *= 1e30
    h, pre = q.ffn_forward(x, wg, wu, ACTS[act], keep_pre=True)
    rows = torch.isnan(h).any(1)
    assert bool(torch.isnan(h[7]).all()) and int(rows.sum()) == 1
    g, u = x[9].double() @ wg.double().t(), x[9].double() @ wu.double().t()
    want = (_gate(g, act)[0] * u).float().to(torch.bfloat16).double()
    got = h[9].double()
    assert torch.equal(torch.isinf(got), torch.isinf(want))
    ok = torch.isfinite(want)
    assert bool(((got - want)[ok].abs() <= 2.0 ** -7 * want[ok].abs() + 1e-30).all())
    gx, gg, gu = q.ffn_backward(x, wg, wu, pre, gh, ACTS[act])
    assert bool(torch.isnan(gx[7]).all() if act != "relu" else torch.isnan(gx[7]).any())
    assert bool(torch.isfinite(gx[:7]).all())


@pytest.mark.parametrize("m,k,f", [(1, 64, 8), (77, 130, 91), (130, 128, 264)])
def test_guard_bands(dev, m, k, f):
    """Every buffer written is the middle of one whose ends stay as they were."""
    x, wg, wu, gh = _problem(dev, m, k, f, torch.float16)
    guard, sent = 4096, 0x7E5A

    def guarded(nbytes):
        return torch.full((2 * guard + (nbytes + 1) // 2,), sent, dtype=torch.int16, device=dev)

    def middle(b, nbytes, dtype, shape):
        return b[guard:guard + (nbytes + 1) // 2].view(dtype)[:math.prod(shape)].view(shape)

    n_pre = q.lib().qconv_ffn_pre_floats(m, f)
    fp = (f + 7) // 8 * 8
    d = q.qconv_ffn_desc(m, k, f, q.DT_F16, q.ACT_SILU, k, k, f)
    import ctypes
    n_ws = q.lib().qconv_ffn_backward_bytes(ctypes.byref(d))
    bufs = {"h": (m * f * 2, torch.float16, (m, f)), "pre": (n_pre * 4, torch.float32, (m * 2 * fp,)),
            "gx": (m * k * 2, torch.float16, (m, k)), "gg": (f * k * 2, torch.float16, (f, k)),
            "gu": (f * k * 2, torch.float16, (f, k)), "ws": (n_ws, torch.uint8, (n_ws,))}
    raw = {n: guarded(b[0]) for n, b in bufs.items()}
    t = {n: middle(raw[n], *bufs[n]) for n in bufs}
    h, _ = q.ffn_forward(x, wg, wu, pre=t["pre"], out=t["h"])
    q.ffn_backward(x, wg, wu, t["pre"], gh, out=(t["gx"], t["gg"], t["gu"]), workspace=t["ws"])
    torch.cuda.synchronize()
    for n, b in raw.items():
        assert bool((b[:guard] == sent).all()) and bool((b[guard + (bufs[n][0] + 1) // 2:] == sent).all()), n
    _check_forward(t["h"], t["pre"], x, wg, wu, "silu")
    _check_backward(t["gx"], t["gg"], t["gu"], x, wg, wu, t["pre"], gh, "silu")


def test_other_stream_and_graph(dev):
    """Calls on a side stream, and captured once and replayed with other inputs in the same buffers, give the eager
    results bit for bit."""
    x, wg, wu, gh = _problem(dev, 70, 256, 200, torch.bfloat16)
    want = []
    inputs = [_problem(dev, 70, 256, 200, torch.bfloat16, seed=s)[0] for s in range(3)]
    for v in inputs:
        h, pre = q.ffn_forward(v, wg, wu, keep_pre=True)
        want.append((h, *q.ffn_backward(v, wg, wu, pre, gh)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    h, pre = q.ffn_forward(inputs[0], wg, wu, keep_pre=True, stream=side)
    got = (h, *q.ffn_backward(inputs[0], wg, wu, pre, gh, stream=side))
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want[0]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        h, pre = q.ffn_forward(x, wg, wu, keep_pre=True)
        got = (h, *q.ffn_backward(x, wg, wu, pre, gh))
    for v, w in zip(inputs, want):
        x.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, w))
        torch.mm(v.float(), wg.float().t())  # eager work between replays
        torch.cuda.synchronize()


def test_refusals(dev):
    x, wg, wu, gh = _problem(dev, 4, 16, 24, torch.float16)
    h, pre = q.ffn_forward(x, wg, wu, keep_pre=True)
    for bad in (lambda: q.ffn_forward(x, wg, wu[:, :8]), lambda: q.ffn_forward(x, wg, wu.bfloat16()),
                lambda: q.ffn_forward(x.t(), wg, wu), lambda: q.ffn_forward(x, wg, wu, out=h.float()),
                lambda: q.ffn_forward(x, wg, wu, pre=pre[:-1]), lambda: q.ffn_forward(x.cpu(), wg, wu),
                lambda: q.ffn_forward(x, wg, torch.empty((24, 20), dtype=x.dtype, device=dev)[:, :16]),
                lambda: q.ffn_backward(x, wg, wu, pre, gh[:2]), lambda: q.ffn_backward(x, wg, wu, pre.half(), gh),
                lambda: q.ffn_backward(x, wg, wu, pre, gh, out=(gh, None, None))):
        with pytest.raises(ValueError):
            bad()
    for bad, status in ((lambda: q.ffn_forward(x, wg, wu, 3), q.QCONV_EINVAL),
                        (lambda: q.ffn_forward(x.float(), wg.float(), wu.float()), q.QCONV_EUNSUPPORTED),
                        (lambda: q.ffn_backward(x, wg, wu, pre, gh, workspace=torch.empty(
                            8, dtype=torch.uint8, device=dev)), q.QCONV_EWORKSPACE)):
        with pytest.raises(q.QconvError) as e:
            bad()
        assert e.value.status == status
