"""Gradients of the gated block at the ends of their types' ranges (run with -m
gpu); the bounds are those of the operators' own tests, whose absolute part is
half the smallest subnormal for each rounding."""
import pytest
import torch

import paper_2003_04296_amd as q
import test_gpu_ffn as ffn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    q.lib()
    return torch.device("cuda:0")


@pytest.mark.parametrize("size", [2.0 ** -22, 2.0 ** -16, 2.0 ** -10, 2.0 ** 7])
@pytest.mark.parametrize("m,k,f", [(3, 64, 40), (130, 128, 264), (200, 99, 72)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_small_and_large_gradients(dev, m, k, f, size, dtype):
    """With fp16, factors and results among the subnormals, and results near 65504."""
    x, wg, wu, gh = ffn._problem(dev, m, k, f, ffn.TYPES[dtype])
    gh = (gh.float() * size).to(gh.dtype)
    _, pre = q.ffn_forward(x, wg, wu, q.ACT_SILU, keep_pre=True)
    grads = q.ffn_backward(x, wg, wu, pre, gh, q.ACT_SILU)
    assert all(bool(torch.isfinite(g).all()) for g in grads)
    ffn._check_backward(*grads, x, wg, wu, pre, gh, "silu")


@pytest.mark.parametrize("m", [3, 130])
def test_a_factor_past_the_range_stays_in_its_row(dev, m):
    """As documented: gh u act'(g) past 65504 is infinite in fp16, in its token's gx and its feature's weight gradients."""
    x, wg, wu, gh = ffn._problem(dev, m, 64, 72, torch.float16)
    _, pre = q.ffn_forward(x, wg, wu, q.ACT_RELU, keep_pre=True)
    want = q.ffn_backward(x, wg, wu, pre, gh, q.ACT_RELU)
    p = pre.view(m, 2, 72)
    c = int((p[1, 0].clamp_min(0) * p[1, 1].abs()).argmax())
    gh[1, c] = 65504.0
    p[1, 1, c] = 4.0
    gx, gg, gu = q.ffn_backward(x, wg, wu, pre, gh, q.ACT_RELU)
    rows, features = [i for i in range(m) if i != 1], [i for i in range(72) if i != c]
    assert not bool(torch.isfinite(gx[1]).any()) and torch.equal(gx[rows], want[0][rows])
    assert not bool(torch.isfinite(gg[c]).any())
    assert torch.equal(gg[features], want[1][features]) and torch.equal(gu[features], want[2][features])
