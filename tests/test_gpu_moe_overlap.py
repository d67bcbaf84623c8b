"""Tensors of the operators for rows that go to different weights that lie in one
another's memory (run with -m gpu): columns beside columns give what separate tensors
do, a result over what is still read is refused."""
import pytest
import torch

import paper_2003_04296_amd as q

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    q.lib()
    return torch.device("cuda:0")


def _beside(dev, seed, rows, *widths):
    """Tensors of so many columns beside each other in one, bf16."""
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    t = torch.randn((rows, sum(widths)), generator=gen, device=dev).bfloat16()
    return t.split(list(widths), dim=1)


@pytest.mark.parametrize("m", [1, 20, 3000])
def test_adapters(dev, m):
    k = n = 72
    x, y, out = _beside(dev, 1, m, k, n, n)
    a, b = _beside(dev, 2, 3 * 8, k)[0].reshape(3, 8, k), _beside(dev, 3, 3 * n, 8)[0].reshape(3, n, 8)
    offsets, order, _ = q.moe_sort(torch.arange(m, device=dev) % 4, 3)
    want, _ = q.lora_forward(y.contiguous(), x.contiguous(), a, b, offsets, order)
    x0 = x.clone()
    got, _ = q.lora_forward(y, x, a, b, offsets, order, out=out)
    assert torch.equal(got, want) and torch.equal(x, x0)
    got, _ = q.lora_forward(y, x, a, b, offsets, order)
    assert torch.equal(got, want) and torch.equal(x, x0)
    c = x.contiguous()
    for call in (lambda: q.lora_forward(c, c, a, b, offsets, order), lambda: q.lora_forward(y, c, a, b, offsets, order, out=c),
                 lambda: q.lora_forward(y, x, a, b, offsets, order, out=x)):
        with pytest.raises(q.QconvError):
            call()
    assert torch.equal(x, x0) and torch.equal(c, x0)
