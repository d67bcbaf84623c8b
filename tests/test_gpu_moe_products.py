"""The experts' products (moe_gated_*, moe_linear_*) against their formulas in
64 bits, group by group (run with -m gpu).  Bounds as for one weight: see the
gated block's tests, whose checks take each group here; for the linear form a sum
of K products in fp32 is off by (K + 8) 2^-23 of the sum of their magnitudes and
the result by half a step of its type more.
"""
import pytest
import torch

import paper_2003_04296_amd as q
from test_gpu_ffn import ACTS, E, TINY, TYPES, U, _check_backward, _check_forward, _close, _normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    q.lib()
    return torch.device("cuda:0")


def _problem(dev, counts, spare, k, f, dtype, seed=0):
    """x, two weights, gh and offsets of groups with so many rows, `spare` rows of none behind them."""
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed + 31 * len(counts) + k * 7 + f)
    rows, groups = sum(counts) + spare, len(counts)
    weight = lambda: _normal(gen, (groups * f, k), k ** -0.5, dtype, dev).view(groups, f, k)
    offsets = torch.tensor([0, *torch.tensor(counts).cumsum(0).tolist()], dtype=torch.int32, device=dev)
    return (_normal(gen, (rows, k), 1.0, dtype, dev), weight(), weight(), _normal(gen, (rows, f), 0.5, dtype, dev), offsets)


def _groups(counts):
    at = 0
    for e, n in enumerate(counts):
        yield e, at, at + n
        at += n


def _run_gated(x, wg, wu, gh, offsets, act):
    """All outputs, where no rows are written into sevens."""
    rows, (groups, f, k) = x.shape[0], wg.shape
    h = torch.full((rows, f), 7.0, dtype=x.dtype, device=x.device)
    h, pre = q.moe_gated_forward(x, wg, wu, offsets, act, keep_pre=True, out=h)
    gx = torch.full((rows, k), 7.0, dtype=x.dtype, device=x.device)
    return h, pre, q.moe_gated_backward(x, wg, wu, offsets, pre, gh, act, out=(gx, None, None))


def _check_gated(counts, spare, x, wg, wu, gh, h, pre, grads, act):
    f = wg.shape[1]
    fp = (f + 7) // 8 * 8
    gx, gg, gu = grads
    for e, i, j in _groups(counts):
        if i == j:
            assert not gg[e].any() and not gu[e].any(), e
            continue
        p = pre[i * 2 * fp:j * 2 * fp]
        _check_forward(h[i:j], p, x[i:j], wg[e], wu[e], act)
        _check_backward(gx[i:j], gg[e], gu[e], x[i:j], wg[e], wu[e], p, gh[i:j], act)
    end = sum(counts)
    assert bool((h[end:] == 7.0).all()) and bool((gx[end:] == 7.0).all())


def _linear(x, w, gy):
    """(y and its bound, gx and its bound, gw and its bound) of one group in 64 bits."""
    X, W, G, r, tiny = x.double(), w.double(), gy.double(), U[x.dtype], TINY[x.dtype]
    out = []
    for a, b, n in ((X, W.t(), X.shape[1]), (G, W, W.shape[0]), (G.t(), X, X.shape[0])):
        v = a.contiguous() @ b.contiguous()
        out.append((v, (n + 8) * E * (a.abs().contiguous() @ b.abs().contiguous()) + 1.01 * r * v.abs() + tiny + 1e-37))
    return out


COUNTS = [
    # groups' rows, rows of none behind them, inputs, outputs: one row, none, both sides of the tiles' 128 and 256 rows
    ([1], 0, 1, 1), ([3, 0, 5], 2, 7, 9), ([0, 0], 4, 64, 40), ([1, 1, 1, 1], 0, 256, 200), ([130, 1, 0, 129], 3, 65, 129),
    ([128, 127, 200], 0, 128, 256), ([16, 40, 0, 33, 7], 1, 1001, 77), ([300, 255, 2], 5, 96, 300),
    ([0, 17, 0, 0, 64, 65, 1, 0], 0, 136, 264),
]


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("act", sorted(ACTS))
@pytest.mark.parametrize("counts,spare,k,f", COUNTS)
def test_gated(dev, counts, spare, k, f, act, dtype):
    x, wg, wu, gh, offsets = _problem(dev, counts, spare, k, f, TYPES[dtype])
    h, pre, grads = _run_gated(x, wg, wu, gh, offsets, ACTS[act])
    _check_gated(counts, spare, x, wg, wu, gh, h, pre, grads, act)
    end = sum(counts)
    assert torch.equal(q.moe_gated_forward(x, wg, wu, offsets, ACTS[act])[0][:end], h[:end])
    only_x = q.moe_gated_backward(x, wg, wu, offsets, pre, gh, ACTS[act], need_w=False)
    only_w = q.moe_gated_backward(x, wg, wu, offsets, pre, gh, ACTS[act], need_x=False)
    assert only_x[1] is None and only_x[2] is None and only_w[0] is None
    assert torch.equal(only_x[0][:end], grads[0][:end]) and all(torch.equal(a, b) for a, b in zip(only_w[1:], grads[1:]))


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("counts,spare,k,f", COUNTS)
def test_linear(dev, counts, spare, k, f, dtype):
    x, w, _, gy, offsets = _problem(dev, counts, spare, k, f, TYPES[dtype])
    rows, end = len(x), sum(counts)
    y = q.moe_linear_forward(x, w, offsets, out=torch.full((rows, f), 7.0, dtype=x.dtype, device=dev))
    gx, gw = q.moe_linear_backward(x, w, offsets, gy, out=(torch.full((rows, k), 7.0, dtype=x.dtype, device=dev), None))
    for e, i, j in _groups(counts):
        if i == j:
            assert not gw[e].any()
            continue
        want = _linear(x[i:j], w[e], gy[i:j])
        for got, (v, bound), what in zip((y[i:j], gx[i:j], gw[e]), want, ("y", "gx", "gw")):
            _close(got, v, bound, f"{what} of group {e}")
    assert bool((y[end:] == 7.0).all()) and bool((gx[end:] == 7.0).all())
    assert torch.equal(q.moe_linear_backward(x, w, offsets, gy, need_w=False)[0][:end], gx[:end])
    assert torch.equal(q.moe_linear_backward(x, w, offsets, gy, need_x=False)[1], gw)


@pytest.mark.parametrize("counts,k,f", [([700, 1100], 512, 16400), ([2100, 0, 1999], 264, 8200)])
def test_larger_tiles(dev, counts, k, f):
    """Rows and outputs enough for the tiles of 256 x 256."""
    x, wg, wu, gh, offsets = _problem(dev, counts, 3, k, f, torch.bfloat16)
    h, pre, grads = _run_gated(x, wg, wu, gh, offsets, q.ACT_SILU)
    _check_gated(counts, 3, x, wg, wu, gh, h, pre, grads, "silu")


@pytest.mark.parametrize("groups", [63, 64, 65, 300, 4096])
def test_many_groups(dev, groups):
    """More groups than a wave has lanes, most of them empty."""
    counts = [0] * groups
    for i, n in enumerate((5, 130, 1, 64, 2)):
        counts[i * (groups - 1) // 4] = n
    x, w, _, gy, offsets = _problem(dev, counts, 4, 64, 24, torch.float16)
    y = q.moe_linear_forward(x, w, offsets)
    gx, gw = q.moe_linear_backward(x, w, offsets, gy)
    for e, i, j in _groups(counts):
        if i < j:
            for got, (v, bound), what in zip((y[i:j], gx[i:j], gw[e]), _linear(x[i:j], w[e], gy[i:j]), ("y", "gx", "gw")):
                _close(got, v, bound, f"{what} of group {e}")
    assert not gw[torch.tensor(counts, device=dev) == 0].any()


@pytest.mark.parametrize("k,f", [(61, 45), (96, 40), (200, 129)])
@pytest.mark.parametrize("counts", [[40, 7, 150], [800, 400]])
@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_rows_of_wider_tensors(dev, counts, k, f, dtype):
    """Row strides past the columns, odd addresses, and NaN beside every row of every operand."""
    x, wg, wu, gh, offsets = _problem(dev, counts, 2, k, f, TYPES[dtype])

    def inside(t, off, pad):
        rows = t.reshape(-1, t.shape[-1])
        b = torch.full((rows.shape[0] + 1, t.shape[-1] + pad), float("nan"), dtype=t.dtype, device=dev)
        v = b[:-1, off:off + t.shape[-1]]
        v.copy_(rows)
        return v if t.dim() == 2 else b.as_strided(t.shape, (t.shape[1] * b.stride(0), b.stride(0), 1), off)

    for off, pad in ((1, 3), (0, 8), (4, 11), (4, 8), (3, 16)):
        xs, gs, us, ds = inside(x, off, pad), inside(wg, off, pad), inside(wu, off, pad), inside(gh, off, pad)
        h, pre, grads = _run_gated(xs, gs, us, ds, offsets, q.ACT_GELU)
        _check_gated(counts, 2, x, wg, wu, gh, h, pre, grads, "gelu")
        y = q.moe_linear_forward(xs, gs, offsets)
        lx, lw = q.moe_linear_backward(xs, gs, offsets, ds)
        for e, i, j in _groups(counts):
            for got, (v, bound), what in zip((y[i:j], lx[i:j], lw[e]), _linear(x[i:j], wg[e], gh[i:j]), ("y", "gx", "gw")):
                _close(got, v, bound, f"{what} of group {e}")


def test_offsets_of_no_order_stay_inside(dev):
    """Offsets that fall, are negative or lie past the rows: nothing outside the tensors is read or written."""
    x, wg, wu, gh, _ = _problem(dev, [40, 40], 0, 64, 48, torch.bfloat16)
    for bad in ([0, 200, 80], [-5, 40, 1 << 30], [80, 40, 0], [-(1 << 31), (1 << 31) - 1, 3]):
        offsets = torch.tensor(bad, dtype=torch.int32, device=dev)
        h, pre = q.moe_gated_forward(x, wg, wu, offsets, keep_pre=True)
        pre.nan_to_num_()
        out = q.moe_gated_backward(x, wg, wu, offsets, pre, gh)
        y = q.moe_linear_forward(x, wg, offsets)
        q.moe_linear_backward(x, wg, offsets, gh)
        torch.cuda.synchronize()
        assert h.shape == y.shape and len(out) == 3


def test_no_rows(dev):
    x, wg, wu, gh, offsets = _problem(dev, [0, 0, 0], 0, 33, 20, torch.bfloat16)
    h, pre = q.moe_gated_forward(x, wg, wu, offsets, keep_pre=True)
    assert h.shape == (0, 20) and pre.numel() == 0
    gx, gg, gu = q.moe_gated_backward(x, wg, wu, offsets, pre, gh)
    assert gx.shape == (0, 33) and not gg.any() and not gu.any() and gg.shape == gu.shape == (3, 20, 33)
    assert q.moe_linear_forward(x, wg, offsets).shape == (0, 20)
    gx, gw = q.moe_linear_backward(x, wg, offsets, gh)
    assert gx.shape == (0, 33) and not gw.any()


@pytest.mark.parametrize("counts,k,f", [
    ([1500, 1300, 40], 2048, 6000),  # forward and gx: the last large tiles split over idle units
    ([3400, 0, 2700], 2048, 4096),   # weight gradients: large tiles, the longer expert in pieces
    ([2400, 300], 520, 1000),        # the same in small tiles
    ([2, 130, 60], 4100, 120),       # few tiles of long sums
])
@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_split_sums(dev, counts, k, f, dtype):
    x, wg, wu, gh, offsets = _problem(dev, counts, 2, k, f, TYPES[dtype])
    h, pre, grads = _run_gated(x, wg, wu, gh, offsets, q.ACT_SILU)
    _check_gated(counts, 2, x, wg, wu, gh, h, pre, grads, "silu")
    y = q.moe_linear_forward(x, wg, offsets, out=torch.full_like(gh, 7.0))
    gx, gw = q.moe_linear_backward(x, wg, offsets, gh, out=(torch.full_like(x, 7.0), None))
    for e, i, j in _groups(counts):
        if i == j:
            assert not gw[e].any()
            continue
        for got, (v, bound), what in zip((y[i:j], gx[i:j], gw[e]), _linear(x[i:j], wg[e], gh[i:j]), ("y", "gx", "gw")):
            _close(got, v, bound, f"{what} of group {e}")
    end = sum(counts)
    assert bool((y[end:] == 7.0).all()) and bool((gx[end:] == 7.0).all())


def test_rows_before_the_first_group(dev):
    """Offsets that do not start at 0: the rows before the first group are no group's, split sums or not."""
    for counts, k, f in (([20, 200], 96, 72), ([2, 130, 60], 4100, 120), ([5, 3], 2048, 64)):
        x, wg, wu, gh, offsets = _problem(dev, counts, 9, k, f, torch.float16)
        offsets = offsets + 6
        h, pre, grads = _run_gated(x, wg, wu, gh, offsets, q.ACT_RELU)
        y = q.moe_linear_forward(x, wg, offsets, out=torch.full_like(gh, 7.0))
        end = 6 + sum(counts)
        for t in (h, y, grads[0]):
            assert bool((t[:6] == 7.0).all()) and bool((t[end:] == 7.0).all())
        fp = (f + 7) // 8 * 8
        _check_gated(counts, 3, x[6:], wg, wu, gh[6:], h[6:], pre[6 * 2 * fp:], (grads[0][6:], *grads[1:]), "relu")
