"""aqe_clip_grads into other tensors: which layouts pair up (run with -m gpu)."""
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


def _filled(t):
    gen = torch.Generator(device=t.device)
    gen.manual_seed(t.numel())
    return t.copy_(torch.randn(t.shape, generator=gen, device=t.device))


def test_dimensions_of_one_value(dev):
    """A channels-last gradient in the list does not bind the others' strides where a dimension has one value, nor the
    shape of those that are contiguous."""
    last = torch.channels_last
    grads = [_filled(torch.empty((8, 6, 5, 4), device=dev).contiguous(memory_format=last)),
             _filled(torch.empty((64, 32, 1, 1), device=dev).contiguous(memory_format=last)),
             _filled(torch.empty((60, 40), device=dev)), _filled(torch.empty((16, 1, 3, 3), device=dev))]
    out = [torch.empty_like(grads[0]), torch.empty((64, 32, 1, 1), device=dev), torch.empty(2400, device=dev),
           torch.empty((16, 1, 3, 3), device=dev).contiguous(memory_format=last)]
    norm = q.aqe_clip_grads(grads, 1.0, out=out)
    n = float(torch.cat([g.double().flatten() for g in grads]).norm())
    assert abs(float(norm) - n) <= 2.0 ** -23 * n
    for g, o in zip(grads, out):
        want = g.double() / n
        assert bool(((o.view(g.shape).double() if o.dim() != g.dim() else o.double()) - want).abs().max() <= 2.0 ** -21)


def test_other_orders_are_refused(dev):
    a = _filled(torch.empty((8, 6, 5, 4), device=dev))
    for o in (torch.empty((8, 6, 5, 4), device=dev).contiguous(memory_format=torch.channels_last),
              torch.empty((6, 8, 5, 4), device=dev).transpose(0, 1)):
        for g, t in ((a, o), (o, a)):
            with pytest.raises(ValueError):
                q.aqe_clip_grads([g], 1.0, out=[t])
    with pytest.raises(ValueError):  # equal strides, another shape
        q.aqe_clip_grads([torch.zeros((4, 6), device=dev).t()], 1.0, out=[torch.zeros((2, 2, 6), device=dev).permute(2, 0, 1)])
