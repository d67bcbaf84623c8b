"""How the operators for rows that go to different weights are called (run with
-m gpu): in captured graphs beside eager calls, on other streams, by tensors of
another device, with workspaces of the caller's, twice at once."""
import types

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


class Step:
    """A training step through experts and one through adapters on tensors of its own; run() returns every result."""

    def __init__(self, dev, seed, tokens=300, slots=2, groups=7, k=136, f=200, rank=12, rows_of_none=0.1):
        gen = torch.Generator(device=dev)
        gen.manual_seed(seed)
        draw = lambda *s: (torch.randn(s, generator=gen, device=dev) * 0.3).bfloat16()
        self.ids = torch.randint(0, groups, (tokens, slots), generator=gen, device=dev)
        self.ids[torch.rand(self.ids.shape, generator=gen, device=dev) < rows_of_none] = -1
        self.weights = torch.rand((tokens, slots), generator=gen, device=dev)
        self.x, self.gy = draw(tokens, k), draw(tokens, k)
        self.wg, self.wu, self.wd = draw(groups, f, k), draw(groups, f, k), draw(groups, k, f)
        self.a, self.b = draw(groups, rank, k), draw(groups, f, rank)
        self.base, self.gb = draw(tokens, f), draw(tokens, f)
        self.scale = torch.rand((groups,), generator=gen, device=dev)
        self.groups = groups

    def run(self, **kw):
        offsets, order, place = q.moe_sort(self.ids, self.groups, **kw)
        zeros = lambda *s: torch.zeros(s, dtype=self.x.dtype, device=self.x.device)
        n, k, f = self.ids.numel(), self.x.shape[1], self.wg.shape[1]
        stream = kw.get("stream")
        with torch.cuda.stream(stream) if stream is not None else torch.cuda.stream(torch.cuda.current_stream()):
            made = [zeros(n, k), zeros(n, f), zeros(n, k), zeros(n, f), zeros(n, k), zeros(n, k), self.base.clone()]
        xs = q.moe_gather(self.x, place, out=made[0], **kw)
        h, pre = q.moe_gated_forward(xs, self.wg, self.wu, offsets, keep_pre=True, out=made[1], **kw)
        ys = q.moe_linear_forward(h, self.wd, offsets, out=made[2], **kw)
        y = q.moe_combine(ys, place, self.weights, **kw)
        gys, gw = q.moe_combine_backward(self.gy, ys, place, self.weights, out=(made[5], None), **kw)
        gh, gwd = q.moe_linear_backward(h, self.wd, offsets, gys, out=(made[3], None), **kw)
        gxs, gwg, gwu = q.moe_gated_backward(xs, self.wg, self.wu, offsets, pre, gh, out=(made[4], None, None), **kw)
        gx = q.moe_gather_backward(gxs, place, **kw)
        mine = q.moe_sort(self.ids[:, 0], self.groups, **kw)
        out, mid = q.lora_forward(made[6], self.x, self.a, self.b, mine[0], mine[1], self.scale, keep_mid=True, **kw)
        grads = q.lora_backward(self.x, self.a, self.b, mine[0], mine[1], mid, self.gb, self.scale, **kw)
        return [offsets, order, place, xs, h, ys, y, gys, gw, gh, gwd, gxs, gwg, gwu, gx, out, *grads]


def _same(a, b):
    for i, (u, v) in enumerate(zip(a, b, strict=True)):
        assert torch.equal(u, v), i


def test_repeats_itself(dev):
    s = Step(dev, 1)
    first = s.run()
    for _ in range(3):
        _same(s.run(), first)


@pytest.mark.parametrize("sizes", [{}, dict(tokens=9000, groups=3, k=264, f=520), dict(tokens=5, slots=3, k=1032, f=72)])
def test_captured_and_replayed(dev, sizes):
    """Two graphs captured one after the other, replayed in turn with eager calls and new inputs between: every replay is
    what an eager call gives."""
    steps = [Step(dev, 2, **sizes), Step(dev, 3, **sizes)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        [s.run() for s in steps]
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for s in steps:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(s.run())
        graphs.append(g)
    for turn in range(3):
        for s, g, out in zip(steps, graphs, outs):
            s.ids.copy_(s.ids.roll(turn, 0))
            s.x.copy_(s.x.roll(1, 1))
            want = [t.clone() for t in s.run()]
            g.replay()
            torch.cuda.synchronize()
            _same(out, want)
    for g in graphs:
        g.replay()
    _same(steps[1].run(), outs[1])


def test_other_streams(dev):
    """Calls on a stream beside the current one, and two steps on two streams at once."""
    steps = [Step(dev, 4), Step(dev, 5, tokens=4000, k=264)]
    want = [s.run() for s in steps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [s.run(stream=t) for _ in range(3) for s, t in zip(steps, streams)]
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        _same(g, want[i % 2])


def test_workspaces(dev):
    """A workspace of the caller's, larger than asked and full of NaN, gives the same; one too small is refused."""
    gen = torch.Generator(device=dev)
    gen.manual_seed(1)
    ids = torch.randint(0, 5, (20000,), generator=gen, device=dev, dtype=torch.int32)
    ws = torch.full((1 << 25,), float("nan"), device=dev)
    for a, b in zip(q.moe_sort(ids, 5), q.moe_sort(ids, 5, workspace=ws)):
        assert torch.equal(a, b)
    s = Step(dev, 6, tokens=64, slots=1, groups=2, k=2048, f=64, rows_of_none=0)
    offsets, order, _ = q.moe_sort(s.ids, 2)
    xs = s.x[order.long()]
    calls = [lambda **kw: q.moe_linear_backward(xs, s.wg, offsets, s.gb, **kw),
             lambda **kw: q.moe_gated_backward(xs, s.wg, s.wu, offsets, pre, s.gb, **kw),
             lambda **kw: [q.lora_forward(s.base, s.x, s.a, s.b, offsets, order, out=torch.empty_like(s.base), **kw)[0]],
             lambda **kw: q.lora_backward(s.x, s.a, s.b, offsets, order, mid, s.gb, **kw)]
    pre = q.moe_gated_forward(xs, s.wg, s.wu, offsets, keep_pre=True)[1]
    mid = q.lora_forward(s.base, s.x, s.a, s.b, offsets, order, keep_mid=True, out=torch.empty_like(s.base))[1]
    for call in calls:
        for a, b in zip(call(), call(workspace=ws)):
            assert torch.equal(a, b)
    for call in (calls[1], calls[3]):
        with pytest.raises(q.QconvError):
            call(workspace=ws[:4])


def _calls(dev):
    x = torch.zeros((4, 32), dtype=torch.bfloat16, device=dev)
    w = torch.zeros((2, 8, 32), dtype=torch.bfloat16, device=dev)
    h = torch.zeros((4, 8), dtype=torch.bfloat16, device=dev)
    ids = torch.zeros(4, dtype=torch.int32, device=dev)
    offsets, order, place = q.moe_sort(ids, 2)
    _, pre = q.moe_gated_forward(x, w, w, offsets, keep_pre=True)
    b = torch.zeros((2, 8, 8), dtype=torch.bfloat16, device=dev)
    _, mid = q.lora_forward(h, x, w, b, offsets, order, keep_mid=True)
    return [lambda **s: q.moe_sort(ids, 2, **s), lambda **s: q.moe_gather(x, place, **s), lambda **s: q.moe_combine(x, place, **s),
            lambda **s: q.moe_gather_backward(x, place, **s), lambda **s: q.moe_combine_backward(x, x, place, **s),
            lambda **s: q.moe_gated_forward(x, w, w, offsets, **s), lambda **s: q.moe_linear_forward(x, w, offsets, **s),
            lambda **s: q.moe_gated_backward(x, w, w, offsets, pre, h, **s),
            lambda **s: q.moe_linear_backward(x, w, offsets, h, **s),
            lambda **s: q.lora_forward(h, x, w, b, offsets, order, **s),
            lambda **s: q.lora_backward(x, w, b, offsets, order, mid, h, **s)]


@pytest.mark.parametrize("i", range(11))
def test_other_device(dev, i, monkeypatch):
    """One device is enough: its number, and a stream's, are made to look like another's."""
    call = _calls(dev)[i]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(stream=side)
    torch.cuda.synchronize()
    with pytest.raises(ValueError, match="cuda:1"):
        call(stream=types.SimpleNamespace(device_index=1, cuda_stream=side.cuda_stream))
    monkeypatch.setattr(q, "_current_device", lambda: 1, raising=False)
    with pytest.raises(ValueError, match="cuda:1"):
        call()


def test_refusals(dev):
    x = torch.zeros((4, 32), dtype=torch.bfloat16, device=dev)
    w = torch.zeros((2, 8, 32), dtype=torch.bfloat16, device=dev)
    h, ids = torch.zeros((4, 8), dtype=torch.bfloat16, device=dev), torch.zeros(4, dtype=torch.int32, device=dev)
    offsets, order, place = q.moe_sort(ids, 2)
    pre, mid = torch.zeros(4 * 16, device=dev), torch.zeros(4 * 8, device=dev)
    b = torch.zeros((2, 8, 8), dtype=torch.bfloat16, device=dev)
    weights = torch.zeros(4, device=dev)
    bad = [
        lambda: q.moe_sort(ids.float(), 2), lambda: q.moe_sort(ids.view(2, 2, 1), 2), lambda: q.moe_sort(ids.view(2, 2).t(), 2),
        lambda: q.moe_sort(ids[:1].expand(4), 2), lambda: q.moe_sort(ids, 2, out=(offsets, order, place[:3])),
        lambda: q.moe_sort(ids, 2, out=(offsets, order)), lambda: q.moe_sort(torch.zeros((4, 0), dtype=torch.int32, device=dev), 2),
        lambda: q.moe_gather(x, place[:3]), lambda: q.moe_gather(x, place.long()), lambda: q.moe_gather(x[0], place),
        lambda: q.moe_gather(x, place, out=x[:3]), lambda: q.moe_gather(x, place, out=x.half()), lambda: q.moe_gather(x.t(), place),
        lambda: q.moe_combine(x[:3], place), lambda: q.moe_combine(x, place, weights.double()),
        lambda: q.moe_combine(x, place, weights[:3]), lambda: q.moe_combine(x, place, out=h),
        lambda: q.moe_combine_backward(x, x[:3], place), lambda: q.moe_combine_backward(x, x, place, out=(None, weights[:3])),
        lambda: q.moe_linear_forward(x, w[:, :, :16], offsets), lambda: q.moe_linear_forward(x, w.half(), offsets),
        lambda: q.moe_linear_forward(x, w, offsets[:2]), lambda: q.moe_linear_forward(x, w, offsets.long()),
        lambda: q.moe_linear_forward(x, w.transpose(0, 1).contiguous().transpose(0, 1), offsets),
        lambda: q.moe_linear_forward(x, w[0], offsets), lambda: q.moe_gated_forward(x, w, w[:, :4], offsets),
        lambda: q.moe_gated_forward(x, w, w, offsets, pre=pre[:60]), lambda: q.moe_gated_forward(x, w, w, offsets, out=x),
        lambda: q.moe_gated_backward(x, w, w, offsets, pre[:60], h), lambda: q.moe_gated_backward(x, w, w, offsets, pre, x),
        lambda: q.moe_linear_backward(x, w, offsets, h, out=(h, None)), lambda: q.moe_linear_backward(x, w, offsets, h[:3]),
        lambda: q.moe_linear_backward(x, w, offsets, h, out=(None,)),
        lambda: q.lora_forward(h, x, w, b[:1], offsets, order), lambda: q.lora_forward(h, x, w[:, :, :16], b, offsets, order),
        lambda: q.lora_forward(h, x, w, b.transpose(1, 2), offsets, order), lambda: q.lora_forward(x, x, w, b, offsets, order),
        lambda: q.lora_forward(h, x, w, b, offsets, order[:3]), lambda: q.lora_forward(h, x, w, b, offsets, order, weights),
        lambda: q.lora_forward(h, x, w, b, offsets, order, mid=mid[:20]), lambda: q.lora_forward(h, x.float(), w, b, offsets, order),
        lambda: q.lora_backward(x, w, b, offsets, order, mid[:20], h), lambda: q.lora_backward(x, w, b, offsets, order, mid, x),
    ]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, q.QconvError)):
            call()
            pytest.fail(f"call {i} went through")
    for call in (lambda: q.moe_sort(ids, 0), lambda: q.moe_sort(ids, 4097),
                 lambda: q.moe_linear_forward(x.float(), w.float(), offsets),
                 lambda: q.lora_forward(h, x, w.new_zeros((2, 257, 32)), w.new_zeros((2, 8, 257)), offsets, order)):
        with pytest.raises(q.QconvError):
            call()
