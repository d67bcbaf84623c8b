"""The experts' products in the form for few rows where an expert has several pieces
of 16 of them, beside empty experts, more of them than a wave has lanes, and several
passes over the inputs (run with -m gpu).  Bounds as in the products' own tests."""
import pytest
import torch

import paper_2003_04296_amd as q
from test_gpu_dense_forms import _expect, _launched
from test_gpu_ffn import ACTS, TYPES
from test_gpu_moe_products import _check_gated, _close, _groups, _linear, _problem, _run_gated

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    q.lib()
    return torch.device("cuda:0")


def _skewed(groups, **rows):
    counts = [0] * groups
    for g, n in rows.items():
        counts[int(g[1:])] = n
    return counts


COUNTS = [
    # groups' rows, rows of none behind them, inputs, outputs
    ([0, 33, 0, 17, 1], 2, 1100, 40), ([64], 0, 2048, 72), ([17, 15], 0, 96, 33), ([0, 0, 16, 32, 0], 5, 1025, 17),
    (_skewed(70, g0=3, g5=100, g6=16, g63=31, g64=1, g66=49), 7, 1032, 24),
    (_skewed(200, g1=5, g64=300, g130=33, g199=18), 0, 1200, 136),
]


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("act", sorted(ACTS))
@pytest.mark.parametrize("counts,spare,k,f", COUNTS)
def test_gated(dev, counts, spare, k, f, act, dtype):
    x, wg, wu, gh, offsets = _problem(dev, counts, spare, k, f, TYPES[dtype])
    (h, pre, grads), names = _launched(lambda: _run_gated(x, wg, wu, gh, offsets, ACTS[act]))
    _expect(names, [r"moe_rows_kernel<.*, 2, 8>"])
    _check_gated(counts, spare, x, wg, wu, gh, h, pre, grads, act)
    end = sum(counts)
    assert torch.equal(q.moe_gated_forward(x, wg, wu, offsets, ACTS[act])[0][:end], h[:end])


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("counts,spare,k,f", COUNTS)
def test_linear(dev, counts, spare, k, f, dtype):
    x, w, _, gy, offsets = _problem(dev, counts, spare, k, f, TYPES[dtype])
    y, names = _launched(lambda: q.moe_linear_forward(x, w, offsets, out=torch.full_like(gy, 7.0)))
    _expect(names, [r"moe_rows_kernel<.*, 1, 8>"])
    for e, i, j in _groups(counts):
        if i < j:
            _close(y[i:j], *_linear(x[i:j], w[e], gy[i:j])[0], f"y of group {e}")
    assert bool((y[sum(counts):] == 7.0).all())


@pytest.mark.parametrize("counts,k,f", [([40, 0, 22], 1024, 40), ([100, 3, *[0] * 40], 1033, 24)])
def test_rows_of_wider_tensors(dev, counts, k, f):
    """Odd addresses, NaN beside every row and behind the last."""
    x, wg, wu, gh, offsets = _problem(dev, counts, 0, k, f, torch.bfloat16)

    def inside(t, off, pad):
        rows = t.reshape(-1, t.shape[-1])
        b = torch.full((len(rows) + 1, t.shape[-1] + pad), float("nan"), dtype=t.dtype, device=dev)
        v = b[:-1, off:off + t.shape[-1]]
        v.copy_(rows)
        return v if t.dim() == 2 else b.as_strided(t.shape, (t.shape[1] * b.stride(0), b.stride(0), 1), off)

    for off, pad in ((1, 3), (4, 8)):
        h, pre, grads = _run_gated(inside(x, off, pad), inside(wg, off, pad), inside(wu, off, pad), inside(gh, off, pad), offsets,
                                   q.ACT_GELU)
        _check_gated(counts, 0, x, wg, wu, gh, h, pre, grads, "gelu")
