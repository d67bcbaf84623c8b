"""Every form of the fully connected kernels that real sizes come to, at sizes
that end inside its tiles, parts and passes (run with -m gpu): tiles of 256,
products split over blocks and joined, gx's split large tiles, blocks of 16, 32
and 64 tokens, several passes over the inputs.  Each case names the kernels it
has to launch, so that a changed choice does not leave a form untested.  The
bounds are those of the operators' own tests."""
import re

import pytest
import torch

import paper_2003_04296_amd as q
import test_gpu_ffn as ffn
import test_gpu_q4 as q4

pytestmark = pytest.mark.gpu

JOIN = r"dense_join_kernel<"
COPY = r"dense_realign_kernel"


def _gated(tile):
    return rf"dense_gemm_kernel<.*, 0, {tile}, {tile}>"


def _gx(tile, direct="true"):
    return rf"dense_gemm_kernel<[^<]*Stage16<32, {tile}, \d+, 0, false, {direct}, .*, 1, {tile}, {tile}>"


def _gw(tile, direct="true"):
    return rf"dense_gemm_kernel<[^<]*Stage16<32, {tile}, \d+, 0, true, {direct}, .*, 1, {tile}, {tile}>"


def _rows(tiles, waves):
    return rf"dense_rows_kernel<.*, {tiles}, {waves}>"


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    q.lib()
    return torch.device("cuda:0")


def _launched(fn):
    """What fn returns, and the names of the library's kernels that it launched."""
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CUDA]) as prof:
        r = fn()
        torch.cuda.synchronize()
    return r, [e.key for e in prof.key_averages() if "qc::" in e.key]


def _expect(names, patterns):
    for p in patterns:
        assert any(re.search(p, n) for n in names), (p, names)


# m, k, f; kernels of the forward; kernels of the backward
FFN = [
    (1030, 264, 8200, [_gated(256)], [_gx(128), JOIN, _gw(128)]),
    (1030, 263, 8200, [COPY, _gated(256)], [COPY, _gx(128), JOIN, _gw(128)]),
    (1030, 2600, 4104, [_gated(128)], [_gx(256), JOIN, _gw(256)]),   # gx: 55 large tiles in 4 parts
    (4100, 4104, 72, [_gated(128), JOIN], [_gx(256), _gw(128), JOIN]),
    (2100, 136, 70, [_gated(128)], [_gx(128), _gw(128), JOIN]),      # the weight gradients in 4 parts
    (300, 2056, 200, [_gated(128), JOIN], [_gx(128), _gw(128)]),
]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("case", range(len(FFN)))
def test_ffn(dev, case, dtype):
    m, k, f, forward, backward = FFN[case]
    act = ("silu", "gelu", "relu")[(case + (dtype == "f16")) % 3]
    x, wg, wu, gh = ffn._problem(dev, m, k, f, ffn.TYPES[dtype])
    (h, pre), names = _launched(lambda: q.ffn_forward(x, wg, wu, ffn.ACTS[act], keep_pre=True))
    _expect(names, forward)
    ffn._check_forward(h, pre, x, wg, wu, act)
    grads, names = _launched(lambda: q.ffn_backward(x, wg, wu, pre, gh, ffn.ACTS[act]))
    _expect(names, backward)
    ffn._check_backward(*grads, x, wg, wu, pre, gh, act)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_ffn_split_off_16_bytes(dev, dtype):
    """Rows whose base address alone is off 16 bytes pass through registers, split products among them."""
    m, k, f = 1100, 136, 1100
    x, wg, wu, gh = ffn._problem(dev, m, k, f, ffn.TYPES[dtype])

    def off(t):
        b = torch.full((t.numel() + 16,), float("nan"), dtype=t.dtype, device=dev)
        return b[3:3 + t.numel()].view(t.shape).copy_(t)

    x, wg, wu = off(x), off(wg), off(wu)
    h, pre = q.ffn_forward(x, wg, wu, q.ACT_SILU, keep_pre=True)
    ffn._check_forward(h, pre, x, wg, wu, "silu")
    grads, names = _launched(lambda: q.ffn_backward(x, wg, wu, pre, gh, q.ACT_SILU))
    _expect(names, [_gx(128, "false"), _gw(128, "false"), JOIN])
    ffn._check_backward(*grads, x, wg, wu, pre, gh, "silu")


# tokens, outputs, inputs; the kernel for 16-bit weights and for 4-bit ones
ROWS = [
    (64, 8200, 1100, _rows(4, 4)),
    (33, 8200, 700, _rows(2, 4)),
    (13, 4200, 2100, _rows(1, 8)),
    (13, 1000, 4200, _rows(1, 16)),
]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("m,n,k,kernel", ROWS)
def test_few_tokens(dev, m, n, k, kernel, dtype):
    x, wg, wu, _ = ffn._problem(dev, m, k, n, ffn.TYPES[dtype])
    (h, pre), names = _launched(lambda: q.ffn_forward(x, wg, wu, q.ACT_SILU, keep_pre=True))
    _expect(names, [kernel])
    ffn._check_forward(h, pre, x, wg, wu, "silu")
    for group in (32, 64, 128):
        gate, up = q.q4_pack(wg, group), q.q4_pack(wu, group)
        bias = torch.linspace(-1, 1, n, device=dev)
        y, names = _launched(lambda: q.q4_linear(x, *gate, bias=bias))
        _expect(names, [kernel])
        q4._check_linear(y, x, gate, bias)
        h, names = _launched(lambda: q.q4_gated(x, *gate, *up, q.ACT_RELU))
        _expect(names, [kernel])
        q4._check_gated(h, x, gate, up, "relu")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_q4_split(dev, group, dtype):
    """15 tiles of 128 for 2056 inputs: four parts, joined with the bias or through the activation."""
    m, n, k = 300, 520, 2056
    gate, up = q.q4_pack(q4._weights(dev, n, k), group), q.q4_pack(q4._weights(dev, n, k, seed=9), group)
    x = q4._x(dev, m, k, q4.TYPES[dtype])
    bias = torch.linspace(-1, 1, n, device=dev)
    y, names = _launched(lambda: q.q4_linear(x, *gate, bias=bias))
    _expect(names, [r"StageQ4<.*, 1, 128, 128>", JOIN])
    q4._check_linear(y, x, gate, bias)
    h, names = _launched(lambda: q.q4_gated(x, *gate, *up, q.ACT_GELU))
    _expect(names, [r"StageQ4<.*, 0, 128, 128>", JOIN])
    q4._check_gated(h, x, gate, up, "gelu")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_q4_large_tiles(dev, group, dtype):
    n, k = 8200, 264
    gate, up = q.q4_pack(q4._weights(dev, n, k), group), q.q4_pack(q4._weights(dev, n, k, seed=9), group)
    x = q4._x(dev, 2060, k, q4.TYPES[dtype])
    bias = torch.linspace(-1, 1, n, device=dev)
    y, names = _launched(lambda: q.q4_linear(x, *gate, bias=bias))
    _expect(names, [r"StageQ4<.*, 1, 256, 256>"])
    q4._check_linear(y, x, gate, bias)
    x = x[:1030]
    h, names = _launched(lambda: q.q4_gated(x, *gate, *up, q.ACT_SILU))
    _expect(names, [r"StageQ4<.*, 0, 256, 256>"])
    q4._check_gated(h, x, gate, up, "silu")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_offsets_past_32_bits(dev, dtype):
    """2.5e9 values of x: the last rows are read and written where they are, and the weight gradients sum over all."""
    m, k, f = 600001, 4104, 40
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of device memory")
    gen = torch.Generator(device=dev)
    gen.manual_seed(4)
    t = ffn.TYPES[dtype]
    x = torch.empty((m, k), dtype=t, device=dev)
    x.view(-1)[:1 << 20].normal_(generator=gen)
    flat, n = x.view(-1), 1 << 20
    while n < flat.numel():  # rows that repeat at no multiple of the tile
        flat[n:2 * n].copy_(flat[:min(n, flat.numel() - n)])
        n *= 2
    wg, wu = (ffn._normal(gen, (f, k), k ** -0.5, t, dev) for _ in range(2))
    gh = ffn._normal(gen, (m, f), 0.5, t, dev)
    h, pre = q.ffn_forward(x, wg, wu, q.ACT_SILU, keep_pre=True)
    gx, gg, gu = q.ffn_backward(x, wg, wu, pre, gh, q.ACT_SILU)
    p = pre.view(m, 2, f)
    for a in (0, 522000, m - 300):  # the values of row 523282 pass 2^31
        s = slice(a, a + 2000 if a else 300)
        part = p[s].contiguous().view(-1)
        ffn._check_forward(h[s], part, x[s], wg, wu, "silu")
        ffn._check_backward(gx[s], None, None, x[s], wg, wu, part, gh[s], "silu")
    want, bound = [0, 0], [0, 0]
    for a in range(0, m, 50000):
        s = slice(a, a + 50000)
        X, D, g, u = x[s].double(), gh[s].double(), p[s, 0].double(), p[s, 1].double()
        act, slope = ffn._gate(g, "silu")
        dg, du = D * u * slope, D * act
        r, tiny, E = ffn.U[t], ffn.TINY[t], ffn.E
        eg = 1.01 * r * dg.abs() + tiny + 16 * E * (1 + g.abs()) * (D * u).abs()
        eu = 1.01 * r * du.abs() + tiny + 16 * E * (g.abs() + act.abs()) * D.abs()
        for i, (d, e) in enumerate(((dg, eg), (du, eu))):
            want[i] = want[i] + d.t() @ X
            # the sum's own rounding: parts of the sum run one after another in fp32
            bound[i] = bound[i] + e.t() @ X.abs() + (m + 8) * E * ((d.abs() + e).t() @ X.abs())
    for got, w, b in zip((gg, gu), want, bound):
        ffn._close(got, w, b + 1.01 * ffn.U[t] * w.abs() + ffn.TINY[t], "weight gradient")
