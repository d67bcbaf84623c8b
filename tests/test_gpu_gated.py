"""The gated block trained, clipped, packed and served (run with -m gpu).

The training step is held against the same step in 64 bits from the same
16-bit weights and tokens: an SGD step of lr moves a weight by lr c g, whose
gradient carries two roundings to bf16 (2^-8 each, one of dg or du within a sum
over the tokens, one of the result) and whose coefficient c as much; so the
move is within 4 * 2^-8 of its size plus what the sum's cancellation leaves,
bounded by the sum of the products' magnitudes."""
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


def test_step_against_64_bits(dev):
    m, k, f, lr, top = 96, 40, 72, 0.5, 0.25
    block = gated.GatedBlock(k, f, device=dev, seed=3)
    gen = torch.Generator(device=dev)
    gen.manual_seed(1)
    x = torch.randn((m, k), generator=gen, device=dev).to(torch.bfloat16)
    gh = (torch.randn((m, f), generator=gen, device=dev) * 0.1).to(torch.bfloat16)
    before = [w.double() for w in block.masters]
    G, W = (w.double() for w in block.weights)
    block.forward(x)
    gx, norm = block.step(x, gh, lr, top)
    X, D = x.double(), gh.double()
    g, u = X @ G.t(), X @ W.t()
    p = torch.sigmoid(g)
    dg, du = D * u * p * (1 + g * (1 - p)), D * g * p
    grads = [dg.t() @ X, du.t() @ X]
    want = float(torch.cat([t.flatten() for t in grads]).norm())
    r = 2.0 ** -8
    assert abs(float(norm) - want) <= 4 * r * want
    assert want > top  # the case clips
    for w, master, b, t, d in zip(block.weights, block.masters, before, grads, (dg, du)):
        spread = d.abs().t() @ X.abs()
        bound = lr * top / want * (4 * r * t.abs() + 2 * r * spread) + 2.0 ** -22
        assert bool(((master.double() - (b - lr * top / want * t).clamp(-1, 1)).abs() <= bound).all())
        assert torch.equal(w, master.to(w.dtype))
    ref = dg @ G + du @ W
    bound = 4 * r * ref.abs() + 2 * r * (dg.abs() @ G.abs() + du.abs() @ W.abs())
    assert bool(((gx.double() - ref).abs() <= bound).all())


def test_trains_and_serves(dev):
    block, teacher, losses = gated.train(steps=80, device=dev)
    assert losses[-1] < 0.5 * losses[0]
    packed = block.packed(group=32)
    x = torch.randn((70, block.masters[0].shape[1]), device=dev).to(torch.bfloat16)
    full, many = block.forward(x).float(), packed.forward(x).float()
    # a normal value's rounding to 4 bits is off by about a tenth of the values' size, in both factors; twice that
    assert float((many - full).norm()) <= 0.34 * float(full.norm())
    # token by token, few at a time and all together: each rounded once (2^-9), the sums in another order (192 terms'
    # 2^-23 of sum |x||w| ~ 8, times the other factor, up to 4)
    for n in (1, 7, 40):
        part = torch.cat([packed.forward(x[i:i + n]) for i in range(0, 70, n)]).float()
        assert bool(((part - many).abs() <= 2.0 ** -8 * 1.01 * many.abs() + 1e-3).all())
