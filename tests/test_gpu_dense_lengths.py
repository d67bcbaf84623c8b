"""Rows of nearly 2^31 inputs, where the last pass of a block reaches past what
an int counts (run with -m gpu).  The inputs are zero but for a few, so every
result is the sum of a few products of small whole numbers and exact."""
import pytest
import torch

import paper_2003_04296_amd as q

pytestmark = pytest.mark.gpu

K = 0x7fffff00 - 0x600  # in the last pass of 2048 inputs the last wave's block ends at 2^31
AT = (0, 129, 4097, 1 << 20, (1 << 30) + 3, K - 2049, K - 130, K - 1)


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of device memory")
    q.lib()
    return torch.device("cuda:0")


def _tokens(dev, m):
    """[m][K]: token t is t + 1 + i at the i-th of the places AT."""
    x = torch.zeros((m, K), dtype=torch.bfloat16, device=dev)
    for i, k in enumerate(AT):
        x[:, k] = torch.arange(1 + i, m + 1 + i, device=dev)
    return x


def _want(m):
    return torch.tensor([float(sum(t + 1 + i for i in range(len(AT)))) for t in range(m)])


@pytest.mark.parametrize("m", [1, 5])
def test_q4_linear(dev, m):
    """Codes and scales end with the last row, whose last pass is not whole."""
    x = _tokens(dev, m)
    codes = torch.full((1, K // 2), 0x22, dtype=torch.uint8, device=dev)  # every weight 1
    scales = torch.ones((1, K // 128), dtype=torch.bfloat16, device=dev)
    y = q.q4_linear(x, codes, scales)
    assert torch.equal(y[:, 0].float().cpu(), _want(m).to(torch.bfloat16).float())


@pytest.mark.parametrize("m", [1, 5])
def test_ffn_forward(dev, m):
    x = _tokens(dev, m)
    w = torch.ones((1, K), dtype=torch.bfloat16, device=dev)
    h, pre = q.ffn_forward(x, w, w, q.ACT_RELU, keep_pre=True)
    assert torch.equal(pre.view(m, 2, 8)[:, :, 0].cpu(), _want(m)[:, None].expand(m, 2))
    assert torch.equal(h[:, 0].float().cpu(), _want(m).square().to(torch.bfloat16).float())
