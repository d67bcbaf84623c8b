"""Rows of no group, before the first and behind the last, in the experts' products
(run with -m gpu): whatever they hold, NaN here, reaches no result, also where operands
off 16-byte rows are copied, and nothing is written there."""
import pytest
import torch

import paper_2003_04296_amd as q
from test_gpu_dense_forms import _expect, _launched
from test_gpu_moe_products import _check_gated, _close, _groups, _linear, _problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    q.lib()
    return torch.device("cuda:0")


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("counts,k,f,copied", [
    ([5, 0, 20], 136, 72, False), ([5, 20], 133, 71, True), ([40, 7, 150], 96, 40, False), ([500, 420], 333, 250, True),
    ([2, 130, 60], 4100, 120, True), ([2400, 300], 520, 1000, False)])
def test_they_hold_nan(dev, counts, k, f, copied, dtype):
    before, end = 6, 6 + sum(counts)
    x, wg, wu, gh, offsets = _problem(dev, counts, before + 3, k, f, dtype)
    offsets = offsets + before
    for t in (x, gh):
        t[:before], t[end:] = float("nan"), float("nan")
    rows, fp = len(x), (f + 7) // 8 * 8
    sevens = lambda c: torch.full((rows, c), 7.0, dtype=dtype, device=dev)
    pre = torch.full((rows * 2 * fp,), float("nan"), device=dev)
    h, _ = q.moe_gated_forward(x, wg, wu, offsets, q.ACT_SILU, pre=pre, out=sevens(f))
    kept = pre.view(rows, -1)
    assert bool(torch.isnan(kept[:before]).all()) and bool(torch.isnan(kept[end:]).all())
    grads, names = _launched(lambda: q.moe_gated_backward(x, wg, wu, offsets, pre, gh, q.ACT_SILU, out=(sevens(k), None, None)))
    if copied:
        _expect(names, [r"dense_realign_kernel"])
    y = q.moe_linear_forward(x, wg, offsets, out=sevens(f))
    gx, gw = q.moe_linear_backward(x, wg, offsets, gh, out=(sevens(k), None))
    for t in (h, y, grads[0], gx):
        assert bool((t[:before] == 7.0).all()) and bool((t[end:] == 7.0).all())
    _check_gated(counts, 3, x[before:], wg, wu, gh[before:], h[before:], pre[before * 2 * fp:], (grads[0][before:], *grads[1:]), "silu")
    for e, i, j in _groups(counts):
        if i < j:
            i, j = i + before, j + before
            for got, (v, bound), what in zip((y[i:j], gx[i:j], gw[e]), _linear(x[i:j], wg[e], gh[i:j]), ("y", "gx", "gw")):
                _close(got, v, bound, f"{what} of group {e}")
        else:
            assert not gw[e].any()
