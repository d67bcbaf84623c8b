"""4-bit weights with group scales (q4_pack, q4_linear, q4_gated) against the
format's definition in 64 bits (run with -m gpu).

Bounds: a sum of K products and its group scales, in any order, is within
(K + 64) 2^-23 sum |x||w| of the exact one (weights are used exactly); a
result is rounded once, 2^-11 (fp16) or 2^-8 (bf16) of it or half the smallest
subnormal; the gated form as in the 16-bit block: |act'| <= 1.13 and 16 fp32
roundings for the activation."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2003_04296_amd as q

pytestmark = pytest.mark.gpu

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
E = 2.0 ** -23
MAGS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    q.lib()
    return torch.device("cuda:0")


def _decode(codes, scales, k):
    """[n][k] float64 of packed weights, from the documented layout."""
    c = codes.cpu().numpy()
    n = c.shape[0]
    nib = np.empty((n, c.shape[1] * 2), np.uint8)
    nib[:, 0::2], nib[:, 1::2] = c & 15, c >> 4
    v = np.where(nib & 8, -1.0, 1.0) * MAGS[nib & 7]
    s = scales.cpu().double().numpy()
    return (v * np.repeat(s, v.shape[1] // s.shape[1], axis=1))[:, :k], nib


def _round6(v):
    """To 6 significant bits, nearest, ties to even (v >= 0, normal)."""
    m, e = np.frexp(v)
    return np.ldexp(np.round(m * 64.0), e - 6)


def _pack_reference(w, group, top):
    """(scales, level indices) of float64 weights by the definition; |w| / scale in fp32 as documented."""
    n, k = w.shape
    kp = -(-k // group) * group
    p = np.zeros((n, kp))
    p[:, :k] = w
    g = p.reshape(n, kp // group, group)
    s = _round6((np.abs(g).max(-1).astype(np.float32) / np.float32(top)).astype(np.float64))
    with np.errstate(divide="ignore", invalid="ignore"):
        r = (np.abs(g).astype(np.float32) / s[..., None].astype(np.float32))
    r = np.where(s[..., None] > 0, r, 0.0)
    idx = sum((r > t).astype(np.uint8) for t in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0))
    return s, (idx | np.where((g < 0) & (idx > 0), 8, 0)).astype(np.uint8).reshape(n, kp)


def _weights(dev, n, k, dtype=torch.float32, seed=0):
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed + n * 17 + k)
    return (torch.randn((n, k), generator=gen, device=dev) * k ** -0.5).to(dtype)


def _x(dev, m, k, dtype, wide=0, seed=1):
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed + m * 13 + k)
    return torch.randn((m, k + wide), generator=gen, device=dev).to(dtype)[:, :k]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("top", [4, 6])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("n,k", [(1, 1), (3, 31), (16, 128), (33, 257), (130, 1000)])
def test_pack(dev, n, k, group, top, dtype):
    w = _weights(dev, n, k, TYPES[dtype])
    codes, scales = q.q4_pack(w, group, top)
    s, nib = _pack_reference(w.double().cpu().numpy(), group, top)
    np.testing.assert_array_equal(scales.double().cpu().numpy(), s)
    v, got = _decode(codes, scales, k)
    np.testing.assert_array_equal(got, nib)
    # every value within half the widest step around it (2 between 4 and 6) of its scale
    err = np.abs(v - w.double().cpu().numpy())
    assert (err <= np.repeat(s, group, 1)[:, :k] * 1.02).all()
    # the scale times any magnitude is a bf16 value
    prod = scales.float()[..., None] * torch.tensor(MAGS, device=dev, dtype=torch.float32)
    assert torch.equal(prod, prod.to(torch.bfloat16).float())


@pytest.mark.parametrize("bits", [1, 2, 3])
def test_pack_holds_low_bit_levels_exactly(dev, bits):
    """The weight levels of 1..3 bits (the AQE forward at alpha = 1) survive packing with top = 4."""
    w = _weights(dev, 40, 300, seed=bits).mul_(10)
    lv = q.aqe_forward(w, bits, 1.0)
    codes, scales = q.q4_pack(lv, 64, top=4)
    v, _ = _decode(codes, scales, 300)
    full = np.abs(lv.cpu().numpy()).reshape(40, -1)
    for g in range(0, 300, 64):
        rows = full[:, g:g + 64].max(1) == 1.0
        assert rows.any()
        np.testing.assert_array_equal(v[rows, g:g + 64], lv.cpu().numpy()[rows, g:g + 64])


def test_pack_specials(dev):
    """A group of zeros packs to zeros, one with an inf or NaN to a NaN scale; ties go to the smaller magnitude."""
    w = torch.zeros((4, 96), device=dev)
    w[1, 40], w[2, 5] = float("inf"), float("nan")
    w[3, :8] = torch.tensor([6.0, 0.25, 0.75, 1.25, -1.75, 2.5, 3.5, 5.0])
    codes, scales = q.q4_pack(w, 32)
    s = scales.float().cpu()
    want = torch.zeros((4, 3))
    want[1, 1] = want[2, 0] = float("nan")
    want[3, 0] = 1.0
    assert torch.equal(torch.isnan(s), torch.isnan(want)) and torch.equal(torch.nan_to_num(s), torch.nan_to_num(want))
    _, nib = _decode(codes, scales, 96)
    assert not nib[:3].any()
    assert list(nib[3, :8]) == [7, 0, 1, 2, 8 + 3, 4, 5, 6]
    y = q.q4_linear(torch.ones((2, 96), device=dev, dtype=torch.bfloat16), codes, scales)
    assert torch.isnan(y).cpu().tolist() == [[False, True, True, False]] * 2


def _bound_linear(x, w, y):
    return (x.shape[1] + 64) * E * (x.abs() @ w.abs().t()) + 1e-37


def _gate(g, act):
    if act == "relu":
        return g.clamp_min(0)
    if act == "silu":
        return g * torch.sigmoid(g)
    return g * 0.5 * torch.erfc(-g / math.sqrt(2))


def _close(got, want, bound, what):
    bad = ~((got.double() - want).abs() <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} values off, worst ratio " \
                          f"{float(((got.double() - want).abs() / bound).max()):.3g}"


def _check_linear(y, x, packed, bias, what=""):
    w = torch.from_numpy(_decode(*packed, x.shape[1])[0]).to(x.device)
    X = x.double()
    want = X @ w.t()
    b = _bound_linear(X, w, want)
    if bias is not None:
        want = want + bias.double()
        b = b + E * bias.double().abs()
    _close(y, want, b + 1.01 * U[x.dtype] * want.abs() + TINY[x.dtype], what)


def _check_gated(h, x, gate, up, act):
    G, W = (torch.from_numpy(_decode(*p, x.shape[1])[0]).to(x.device) for p in (gate, up))
    X = x.double()
    g, u = X @ G.t(), X @ W.t()
    dg, du = _bound_linear(X, G, g), _bound_linear(X, W, u)
    a = _gate(g, act)
    want = a * u
    _close(h, want, 1.13 * dg * (u.abs() + du) + (a.abs() + 1.13 * dg) * du + 16 * E * (g.abs() + a.abs()) * u.abs()
           + 1.01 * U[x.dtype] * want.abs() + TINY[x.dtype], f"gated {act}")


# one token to many, both sides of 16, 32, 64 and 128 tokens; odd inputs and outputs; one group and many
SHAPES = [(1, 1, 1), (1, 5, 31), (1, 33, 4096), (1, 4096, 520), (2, 16, 128), (3, 100, 129), (4, 48, 1000), (5, 7, 4000),
          (8, 1024, 256), (15, 64, 65), (16, 17, 640), (17, 40, 384), (31, 130, 200), (32, 64, 1024), (33, 50, 96),
          (48, 256, 8192), (64, 10, 2048), (65, 65, 65), (100, 129, 300), (128, 128, 128), (129, 200, 513), (300, 520, 264),
          (515, 96, 1000)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_linear(dev, m, n, k, group, dtype):
    packed = q.q4_pack(_weights(dev, n, k), group)
    x = _x(dev, m, k, TYPES[dtype])
    bias = torch.linspace(-1, 1, n, device=dev) if (m + n) % 2 else None
    _check_linear(q.q4_linear(x, *packed, bias=bias), x, packed, bias)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_gated(dev, m, n, k, group, dtype):
    gate, up = q.q4_pack(_weights(dev, n, k), group), q.q4_pack(_weights(dev, n, k, seed=9), group)
    x = _x(dev, m, k, TYPES[dtype])
    for act, code in (("silu", q.ACT_SILU), ("gelu", q.ACT_GELU), ("relu", q.ACT_RELU)):
        _check_gated(q.q4_gated(x, *gate, *up, code), x, gate, up, act)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m,n,k", [(1, 20, 9001), (2, 16, 8192), (3, 35, 12400), (4, 31, 5183), (4, 1, 640)])
def test_few_tokens_long_rows(dev, m, n, k, group, dtype):
    """Rows longer than one pass of a block's waves, with ends inside a block and a group."""
    packed, up = q.q4_pack(_weights(dev, n, k), group), q.q4_pack(_weights(dev, n, k, seed=9), group)
    x = _x(dev, m, k, TYPES[dtype], wide=3)
    bias = torch.linspace(-1, 1, n, device=dev)
    _check_linear(q.q4_linear(x, *packed, bias=bias), x, packed, bias)
    _check_gated(q.q4_gated(x, *packed, *up, q.ACT_GELU), x, packed, up, "gelu")


@pytest.mark.parametrize("scale", [2.0 ** -30, 2.0 ** 12])
@pytest.mark.parametrize("m", [1, 20, 200])
def test_scales_of_any_size(dev, m, scale):
    """Weights far below and above fp16's range with fp16 tokens: no weight is rounded or overflows on the way."""
    w = _weights(dev, 80, 512)
    w[:, 256:] *= 2.0 ** -20  # groups of one row far apart
    packed = q.q4_pack(w * scale, 64)
    x = _x(dev, m, 512, torch.float16)
    if scale < 1:
        x = x * 1000
    _check_linear(q.q4_linear(x, *packed), x, packed, None)


@pytest.mark.parametrize("wide", [1, 8, 13])
@pytest.mark.parametrize("m,n,k", [(1, 40, 200), (7, 33, 131), (40, 70, 256), (150, 66, 300)])
def test_rows_of_wider_tensors(dev, m, n, k, wide):
    packed = q.q4_pack(_weights(dev, n, k + wide)[:, wide:], 32)
    base = torch.full((m + 2, k + wide + 3), float("nan"), dtype=torch.float16, device=dev)
    x = base[1:m + 1, wide:wide + k]
    x.copy_(_x(dev, m, k, torch.float16))
    out = torch.full((m, n + wide), 7.0, dtype=torch.float16, device=dev)
    y = q.q4_linear(x, *packed, out=out[:, :n])
    assert y.data_ptr() == out.data_ptr() and bool((out[:, n:] == 7.0).all())
    _check_linear(y, x, packed, None)
    h = q.q4_gated(x, *packed, *packed, q.ACT_SILU, out=out[:, wide:])
    _check_gated(h, x, packed, packed, "silu")


@pytest.mark.parametrize("k,off,pad", [(320, 4, 8), (320, 0, 3), (317, 0, 8), (317, 3, 5), (320, 1, 7)])
def test_many_tokens_at_any_address(dev, k, off, pad):
    """x with rows at and off 16-byte addresses, NaN beside every row."""
    m, n = 130, 70
    packed = q.q4_pack(_weights(dev, n, k), 64)
    x = _x(dev, m, k, torch.bfloat16)
    stride = (k + 7) // 8 * 8 + pad
    b = torch.full(((m + 1) * stride,), float("nan"), dtype=x.dtype, device=dev)
    v = b.as_strided((m, k), (stride, 1), off)
    v.copy_(x)
    _check_linear(q.q4_linear(v, *packed), x, packed, None)
    _check_gated(q.q4_gated(v, *packed, *packed, q.ACT_RELU), x, packed, packed, "relu")


@pytest.mark.parametrize("m", [1, 3, 40, 200])
def test_nan_and_inf_stay_in_their_row(dev, m):
    packed = q.q4_pack(_weights(dev, 70, 320), 64)
    x = _x(dev, m, 320, torch.bfloat16)
    want = q.q4_linear(x, *packed)
    x[0, 77] = float("nan")
    y = q.q4_linear(x, *packed)
    assert bool(torch.isnan(y[0]).all()) and torch.equal(y[1:], want[1:])
    x[0, 77] = float("inf")
    y = q.q4_linear(x, *packed)[0].double().cpu().numpy()
    col = _decode(*packed, 320)[0][:, 77]  # inf * 0 is NaN, else an infinity of the weight's sign
    np.testing.assert_array_equal(np.isnan(y), col == 0)
    np.testing.assert_array_equal(y[col != 0], np.sign(col[col != 0]) * np.inf)


def test_no_tokens(dev):
    packed = q.q4_pack(_weights(dev, 70, 320), 64)
    x = torch.empty((0, 320), dtype=torch.float16, device=dev)
    assert q.q4_linear(x, *packed).shape == (0, 70)
    assert q.q4_gated(x, *packed, *packed).shape == (0, 70)


@pytest.mark.parametrize("m,n,k", [(1, 50, 100), (9, 33, 130), (70, 40, 96), (200, 129, 300)])
def test_guard_bands(dev, m, n, k):
    guard, sent = 8192, 0x5A

    def guarded(nbytes):
        return torch.full((2 * guard + nbytes,), sent, dtype=torch.uint8, device=dev)

    kp = -(-k // 64) * 64
    cb, sb = n * kp // 2, n * kp // 64 * 2
    c, s, y = guarded(cb), guarded(sb), guarded(m * n * 2)
    codes = c[guard:guard + cb].view(n, kp // 2)
    scales = s[guard:guard + sb].view(torch.bfloat16).view(n, kp // 64)
    q.q4_pack(_weights(dev, n, k), 64, out=(codes, scales))
    out = y[guard:guard + m * n * 2].view(torch.float16).view(m, n)
    x = _x(dev, m, k, torch.float16)
    q.q4_linear(x, codes, scales, out=out)
    _check_linear(out, x, (codes, scales), None)
    q.q4_gated(x, codes, scales, codes, scales, out=out)
    torch.cuda.synchronize()
    for b, nbytes, what in ((c, cb, "codes"), (s, sb, "scales"), (y, m * n * 2, "out")):
        assert bool((b[:guard] == sent).all()) and bool((b[guard + nbytes:] == sent).all()), what


@pytest.mark.parametrize("m", [1, 40, 200])
def test_other_stream_and_graph(dev, m):
    packed = q.q4_pack(_weights(dev, 256, 512), 128)
    inputs = [_x(dev, m, 512, torch.bfloat16, seed=s) for s in range(3)]
    want = [q.q4_linear(v, *packed) for v in inputs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = q.q4_linear(inputs[0], *packed, stream=side)
    side.synchronize()
    assert torch.equal(y, want[0])
    x = inputs[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y = q.q4_linear(x, *packed)
    for v, w in zip(inputs, want):
        x.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, w)
        q.q4_linear(inputs[1], *packed)
        torch.cuda.synchronize()


def test_refusals(dev):
    codes, scales = q.q4_pack(_weights(dev, 40, 100), 32)
    x = _x(dev, 3, 100, torch.float16)
    for bad in (lambda: q.q4_linear(x[:, :60], codes, scales), lambda: q.q4_linear(x, codes[:10], scales),
                lambda: q.q4_linear(x, codes, scales.float()), lambda: q.q4_linear(x, codes.t(), scales),
                lambda: q.q4_linear(x, codes, scales[:, :1]), lambda: q.q4_linear(x.cpu(), codes, scales),
                lambda: q.q4_linear(x, codes, scales, bias=torch.zeros(39, device=dev)),
                lambda: q.q4_linear(x, codes, scales, out=torch.empty((3, 40), device=dev)),
                lambda: q.q4_gated(x, codes, scales, *q.q4_pack(_weights(dev, 40, 100), 64)),
                lambda: q.q4_gated(x, codes, scales, codes[:1], scales[:1])):
        with pytest.raises(ValueError):
            bad()
    for bad, status in ((lambda: q.q4_pack(_weights(dev, 40, 100), 48), q.QCONV_EINVAL),
                        (lambda: q.q4_pack(_weights(dev, 40, 100), 32, top=5), q.QCONV_EINVAL),
                        (lambda: q.q4_pack(_weights(dev, 40, 100).double(), 32), q.QCONV_EINVAL),
                        (lambda: q.q4_linear(x.float(), codes, scales), q.QCONV_EUNSUPPORTED),
                        (lambda: q.q4_gated(x, codes, scales, codes, scales, 7), q.QCONV_EINVAL)):
        with pytest.raises(q.QconvError) as e:
            bad()
        assert e.value.status == status
    shift = torch.empty(codes.numel() + 16, dtype=torch.uint8, device=dev)[4:4 + codes.numel()].view(codes.shape)
    with pytest.raises(q.QconvError) as e:  # codes are 16-byte aligned
        q.q4_linear(x, shift, scales)
    assert e.value.status == q.QCONV_EINVAL
    d = q.qconv_q4_desc(3, 40, 100, 32, q.DT_F16, 99, 40)
    rc = q.lib().qconv_q4_linear(ctypes.byref(d), q._ptr(x), q._ptr(codes), q._ptr(scales), None, q._ptr(x), None, 0, None)
    assert rc == q.QCONV_EINVAL
