"""4-bit weights whose scales q4_pack would not make: any bf16 value is a scale,
and the weights are used exactly with any number of tokens (run with -m gpu).

The tokens have few values that are not zero, placed so that a result is a
small difference of products, or comes from a row's smallest groups alone: a
weight rounded to 8 or 11 bits on the way shows.  Bounds as in the operators'
own tests, (K + 64) 2^-23 sum |x||w| and one rounding of the result."""
import pytest
import torch

import paper_2003_04296_amd as q
import test_gpu_q4 as q4

pytestmark = pytest.mark.gpu

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
# tokens, outputs, inputs: both sides of 64 tokens; ragged tiles of 128; split
# over blocks; 256 x 256 tiles plain and gated
SIZES = [(1, 70, 512), (5, 70, 512), (64, 70, 512), (65, 70, 512), (130, 200, 317), (300, 520, 2056), (2060, 8200, 264),
         (1030, 8200, 264)]


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    q.lib()
    return torch.device("cuda:0")


def _gen(dev, seed):
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    return gen


def _packed(dev, n, k, group, scale, seed):
    """Random codes (zero past k) and the scales scale(gen, shape)."""
    kp, gen = -(-k // group) * group, _gen(dev, seed + n + k)
    c = torch.randint(0, 16, (n, kp), generator=gen, device=dev, dtype=torch.uint8)
    c[:, k:] = 0
    s = scale(gen, (n, kp // group)).to(torch.bfloat16)
    return (c[:, 0::2] | c[:, 1::2] << 4).contiguous(), s


def _pairs(dev, m, k, dtype, group, seed, size=1.0):
    """Tokens with one value in a group and its negative in another."""
    gen = _gen(dev, seed + m * 3 + k)
    x = torch.zeros((m, k), device=dev)
    at = torch.randint(0, k, (m, 2), generator=gen, device=dev)
    at[:, 1] = torch.where(at[:, 0] // group == at[:, 1] // group, (at[:, 0] + group) % k, at[:, 1])
    v = size * (1.0 + torch.randint(0, 8, (m, 1), generator=gen, device=dev) / 8)
    return x.scatter_(1, at, torch.cat((v, -v), 1)).to(dtype)


def _eight_bits(gen, shape):
    """Scales of 8 significant bits around 1, close to each other."""
    return 1.5 + torch.randint(0, 64, shape, generator=gen, device=gen.device) / 128.0


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_eight_bit_scales(dev, m, n, k, group, dtype):
    gate, up = (_packed(dev, n, k, group, _eight_bits, s) for s in (1, 2))
    x = _pairs(dev, m, k, TYPES[dtype], group, 3)
    bias = torch.linspace(-1, 1, n, device=dev) if group == 64 else None
    q4._check_linear(q.q4_linear(x, *gate, bias=bias), x, gate, bias)
    q4._check_gated(q.q4_gated(x, *gate, *up, q.ACT_RELU), x, gate, up, "relu")


@pytest.mark.parametrize("m,n,k", SIZES)
def test_one_scale_among_many(dev, m, n, k):
    """A single scale of 8 bits, in a weight packed otherwise, in the last row and group or in the middle."""
    x = _pairs(dev, m, k, torch.bfloat16, 32, 5)
    x[:, k - 1], x[:, k // 2] = 1.0, -1.0
    for row, at in ((n - 1, k - 1), (n // 2, k // 2)):
        codes, scales = q.q4_pack(q4._weights(dev, n, k), 32)
        g = at // 32
        scales[row, g] = 255 / 128
        codes[row, g * 16:(at + 2) // 2] = 0x33  # magnitudes 1.5: 2.98828125 has 9 bits
        if k % 2 and at == k - 1:
            codes[row, at // 2] = 0x03
        q4._check_linear(q.q4_linear(x, codes, scales), x, (codes, scales), None)
        q4._check_gated(q.q4_gated(x, codes, scales, codes, scales, q.ACT_RELU), x, (codes, scales), (codes, scales), "relu")


@pytest.mark.parametrize("apart", [12, 19, 24, 27, 29, 31, 60])
@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_small_groups_of_a_row(dev, m, n, k, group, apart):
    """fp16 tokens that are zero but in groups far below their row's largest scale."""
    def scale(gen, shape):
        s = _eight_bits(gen, shape)
        s[:, 1:] *= 2.0 ** -apart
        return s * 2.0 ** (apart - 8)

    packed, up = (_packed(dev, n, k, group, scale, s) for s in (4, 5))
    x = _pairs(dev, m, k, torch.float16, group, 6, 16.0)
    x[:, :group] = 0
    q4._check_linear(q.q4_linear(x, *packed), x, packed, None)
    q4._check_gated(q.q4_gated(x, *packed, *up, q.ACT_RELU), x, packed, up, "relu")


@pytest.mark.parametrize("scale,size", [(2.0 ** -131, 2.0 ** 100), (2.0 ** -126, 2.0 ** 100), (2.0 ** 126, 2.0 ** -100)])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_scales_at_the_ends_of_the_type(dev, m, n, k, scale, size):
    """Subnormal scales, and ones whose largest weight, 6 times as much, passes the type's range."""
    packed = _packed(dev, n, k, 64, lambda gen, shape: torch.full(shape, scale, device=dev), 7)
    x = _pairs(dev, m, k, torch.bfloat16, 64, 8, size)
    q4._check_linear(q.q4_linear(x, *packed), x, packed, None)


@pytest.mark.parametrize("m", [64, 200])
@pytest.mark.parametrize("off", [1, 4])
def test_x_off_16_bytes(dev, m, off):
    n, k = 150, 200
    packed = _packed(dev, n, k, 32, _eight_bits, 9)
    x = _pairs(dev, m, k, torch.bfloat16, 32, 10)
    base = torch.full((m * k + 16,), float("nan"), dtype=x.dtype, device=dev)
    v = base[off:off + m * k].view(m, k).copy_(x)
    q4._check_linear(q.q4_linear(v, *packed), x, packed, None)


@pytest.mark.parametrize("m", [40, 200])
def test_nan_scale_stays_in_its_output(dev, m):
    codes, scales = _packed(dev, 150, 256, 64, _eight_bits, 11)
    x = _pairs(dev, m, 256, torch.bfloat16, 64, 12)
    want = q.q4_linear(x, codes, scales)
    scales[77, 2] = float("nan")
    y = q.q4_linear(x, codes, scales)
    assert bool(torch.isnan(y[:, 77]).all())
    keep = [i for i in range(150) if i != 77]
    assert torch.equal(y[:, keep], want[:, keep])


@pytest.mark.parametrize("m", [40, 200])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_infinity_stays_one(dev, m, dtype):
    """An infinite token value gives infinities of the weights' signs (NaN where the weight is zero), in its row alone."""
    codes, scales = _packed(dev, 150, 256, 64, _eight_bits, 13)
    x = _pairs(dev, m, 256, TYPES[dtype], 64, 14)
    x[3] = 0
    want = q.q4_linear(x, codes, scales)
    x[3, 77] = float("inf")
    y = q.q4_linear(x, codes, scales)
    w = torch.from_numpy(q4._decode(codes, scales, 256)[0]).to(dev)[:, 77]
    assert torch.equal(torch.isnan(y[3]), w == 0)
    assert torch.equal(y[3][w != 0].double(), w[w != 0].sign() * float("inf"))
    keep = [i for i in range(m) if i != 3]
    q4._close(y[keep], want[keep].double(), 1e-3 + want[keep].double().abs() * 2.0 ** -8, "rows beside it")
