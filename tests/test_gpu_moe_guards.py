"""Offsets, places and tokens of no order or outside the tensors (run with -m gpu):
results, what is kept for the backward pass and workspaces lie inside larger buffers,
and what lies before and behind them stays as it was.  What the results hold then is
nobody's; sizes reach every kernel that joins partial sums."""
import ctypes

import pytest
import torch

import paper_2003_04296_amd as q
from test_gpu_lora import _problem as _lora_problem
from test_gpu_moe_products import _problem

pytestmark = pytest.mark.gpu
PAD = 1 << 20  # bytes before and behind


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    q.lib()
    yield torch.device("cuda:0")
    torch.cuda.empty_cache()


class Guarded:
    """Tensors inside larger ones, and whether what is around them is as it was."""

    def __init__(self, dev):
        self.dev, self.stores = dev, []

    def new(self, shape, dtype):
        n = torch.empty(shape, dtype=dtype, device="meta").numel() * torch.empty((), dtype=dtype).element_size()
        store = torch.full((n + 2 * PAD,), 0x5A, dtype=torch.uint8, device=self.dev)
        self.stores.append((store, n))
        return store[PAD:PAD + n].view(dtype).view(shape)

    def check(self, what):
        torch.cuda.synchronize()
        for i, (store, n) in enumerate(self.stores):
            assert bool((store[:PAD] == 0x5A).all()) and bool((store[PAD + n:] == 0x5A).all()), (what, i)


def _bad_offsets(rows, groups):
    """groups + 1 offsets that fall, lie outside, or give all rows to every other group."""
    for some in ([0, 2 * rows, rows // 2, rows], [-5, rows // 2, 1 << 30, 3], [rows, rows // 2, 0, -1],
                 [-(1 << 31), (1 << 31) - 1, 3, 7], [0, rows, 0, rows], [rows // 3, rows, rows - 1, rows + 1], [rows + 9, rows + 99, 5, 2]):
        yield some[:3] + [some[2 + i % 2] for i in range(groups - 2)]


@pytest.mark.parametrize("rows,groups,k,f", [(80, 2, 64, 48), (80, 5, 64, 48), (32, 3, 1100, 40), (2840, 3, 2048, 6000), (6100, 3, 2048, 4096), (2700, 2, 520, 1000),
                                             (192, 3, 4100, 120), (920, 2, 333, 250), (60, 300, 1030, 24)])
def test_products(dev, rows, groups, k, f):
    x, wg, wu, gh, _ = _problem(dev, [rows] + [0] * (groups - 1), 0, k, f, torch.bfloat16)
    d = ctypes.byref(q.qconv_moe_desc(rows, groups, k, f, q.DT_BF16, q.ACT_SILU, k, k, f))
    L, g = q.lib(), Guarded(dev)
    h, y, pre = g.new((rows, f), x.dtype), g.new((rows, f), x.dtype), g.new((L.qconv_ffn_pre_floats(rows, f),), torch.float32)
    grads = [g.new((rows, k), x.dtype), g.new((groups, f, k), x.dtype), g.new((groups, f, k), x.dtype)]
    linear = [g.new((rows, k), x.dtype), g.new((groups, f, k), x.dtype)]
    ws = [g.new((call(d, gated),), torch.uint8) for call in (L.qconv_moe_forward_bytes, L.qconv_moe_backward_bytes) for gated in (1, 0)]
    for bad in _bad_offsets(rows, groups):
        offsets = torch.tensor(bad, dtype=torch.int32, device=dev)
        q.moe_gated_forward(x, wg, wu, offsets, pre=pre, out=h, workspace=ws[0])
        g.check((bad[:5], "gated forward"))
        q.moe_gated_backward(x, wg, wu, offsets, pre, gh, out=grads, workspace=ws[2])
        g.check((bad[:5], "gated backward"))
        q.moe_linear_forward(x, wg, offsets, out=y, workspace=ws[1])
        q.moe_linear_backward(x, wg, offsets, gh, out=linear, workspace=ws[3])
        g.check((bad[:5], "linear"))


@pytest.mark.parametrize("m,groups,rank,k,n", [(30, 3, 8, 64, 72), (1500, 2, 20, 1100, 77), (8200, 5, 24, 264, 300), (100, 4, 40, 4096, 2500),
                                               (700, 2, 130, 2055, 3001), (300, 200, 4, 96, 40)])
def test_adapters(dev, m, groups, rank, k, n):
    s = _lora_problem(dev, m, groups, rank, k, n, torch.bfloat16, "mixed")
    d = ctypes.byref(q.qconv_lora_desc(m, groups, rank, k, n, q.DT_BF16, k, n, n))
    L, g = q.lib(), Guarded(dev)
    good, order, _ = q.moe_sort(s["ids"], groups)
    strange = order.clone()
    strange[::3], strange[1::7], strange[-1], strange[2] = m, -4, 0x7fffffff, -(1 << 31)
    out, mid = g.new((m, n), s["x"].dtype), g.new((L.qconv_lora_mid_floats(m, rank),), torch.float32)
    grads = [g.new((m, k), s["x"].dtype), g.new((groups, rank, k), s["x"].dtype), g.new((groups, n, rank), s["x"].dtype)]
    ws = [g.new((L.qconv_lora_forward_bytes(d, 1),), torch.uint8), g.new((L.qconv_lora_backward_bytes(d),), torch.uint8)]
    for bad in [good.tolist(), *_bad_offsets(m, groups)]:
        offsets = torch.tensor(bad, dtype=torch.int32, device=dev)
        for o in (order, strange):
            q.lora_forward(s["y"], s["x"], s["a"], s["b"], offsets, o, s["scale"], mid=mid, out=out, workspace=ws[0])
            g.check((bad[:5], "forward"))
            q.lora_backward(s["x"], s["a"], s["b"], offsets, o, mid, s["gy"], s["scale"], out=grads, workspace=ws[1])
            g.check((bad[:5], "backward"))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_places(dev, dtype):
    tokens, slots, width = 50, 3, 133
    g = Guarded(dev)
    x, rows = torch.randn((tokens, width), device=dev).to(dtype), torch.randn((tokens * slots, width), device=dev).to(dtype)
    w = torch.rand((tokens, slots), device=dev)
    place = torch.arange(tokens * slots, device=dev, dtype=torch.int32).view(tokens, slots) * 7 - 300
    place[0], place[7, 1], place[49, 2], place[3, 0] = tokens * slots, 0x7fffffff, -(1 << 31), tokens * slots + 1
    to, y = g.new((tokens * slots, width), dtype), g.new((tokens, width), dtype)
    grows, gw = g.new((tokens * slots, width), dtype), g.new((tokens, slots), torch.float32)
    q.moe_gather(x, place, out=to)
    q.moe_combine(rows, place, w, out=y)
    q.moe_combine_backward(x, rows, place, w, out=(grows, gw))
    g.check("rows")
