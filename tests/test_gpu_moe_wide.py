"""Few rows of very many outputs in the experts' products (run with -m gpu): past the
number of blocks that the form for few rows may have, tiles take them.  Bounds as in
the products' own tests: K products in fp32 and half a step of the result's type."""
import pytest
import torch

import paper_2003_04296_amd as q
from test_gpu_ffn import _check_forward
from test_gpu_moe_products import _close, _groups, _linear, _problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    q.lib()
    yield torch.device("cuda:0")
    torch.cuda.empty_cache()


# 34 pieces of 16 rows by 16 outputs: 2^22 blocks lie between the two
@pytest.mark.parametrize("f", [1973600, 1973800])
def test_outputs_past_the_blocks_of_few_rows(dev, f):
    counts = [1, 0, 17, *[0] * 20, 3, *[0] * 7, 9]
    x, wg, wu, gh, offsets = _problem(dev, counts, 2, 8, f, torch.bfloat16)
    assert x.shape[0] == 32 and wg.shape[0] == 32
    y = q.moe_linear_forward(x, wg, offsets, out=torch.full_like(gh, 7.0))
    h, pre = q.moe_gated_forward(x, wg, wu, offsets, keep_pre=True, out=torch.full_like(gh, 7.0))
    fp = (f + 7) // 8 * 8
    for e, i, j in _groups(counts):
        if i < j:
            _close(y[i:j], *_linear(x[i:j], wg[e], gh[i:j])[0], f"y of group {e}")
            _check_forward(h[i:j], pre[i * 2 * fp:j * 2 * fp], x[i:j], wg[e], wu[e], "silu")
    end = sum(counts)
    assert bool((y[end:] == 7.0).all()) and bool((h[end:] == 7.0).all())
