"""Calls of the gated block in other orders than the training loop's (run with
-m gpu)."""
import pytest
import torch

import paper_2003_04296_amd as q
from paper_2003_04296_amd import gated

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    q.lib()
    return torch.device("cuda:0")


@pytest.mark.parametrize("kept", [False, True])
def test_forwards_between_a_forward_and_its_step(dev, kept):
    """A step on x is the same whatever went forward since x did, with the kept pre and without it."""
    m, k, f = 48, 40, 72
    gen = torch.Generator(device=dev)
    gen.manual_seed(2)
    x, other = (torch.randn((m, k), generator=gen, device=dev).to(torch.bfloat16) for _ in range(2))
    gh = (torch.randn((m, f), generator=gen, device=dev) * 0.1).to(torch.bfloat16)
    results = []
    for between in ([], [other], [other[:7], other, x]):
        block = gated.GatedBlock(k, f, device=dev, seed=3)
        if kept:
            h, pre = block.forward_train(x)
            assert torch.equal(h, block.forward(x))
        else:
            block.forward(x)
            pre = None
        for t in between:
            block.forward(t)
        gx, norm = block.step(x, gh, 0.5, 0.25, pre) if kept else block.step(x, gh, 0.5, 0.25)
        results.append([gx, norm, *block.masters, *block.weights])
    for r in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], r))


def test_forward_keeps_no_buffer(dev):
    block = gated.GatedBlock(64, 64, device=dev)
    x = torch.zeros((1 << 16, 64), dtype=torch.bfloat16, device=dev)
    before = torch.cuda.memory_allocated()
    h = block.forward(x)
    del h
    assert torch.cuda.memory_allocated() == before
