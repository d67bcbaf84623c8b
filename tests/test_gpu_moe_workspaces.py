"""Workspaces of exactly the stated bytes, full of NaN, for every way that the
operators for rows that go to different weights use one (run with -m gpu): results are
those of a call without one, nothing past the workspace is written, one byte
less is refused."""
import ctypes

import pytest
import torch

import paper_2003_04296_amd as q
from test_gpu_dense_forms import _expect, _launched
from test_gpu_lora import _problem as _lora_problem
from test_gpu_moe_products import _problem

pytestmark = pytest.mark.gpu
GUARD = 1 << 24


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    q.lib()
    yield torch.device("cuda:0")
    torch.cuda.empty_cache()


def _check(dev, call, need, kernels):
    assert need > 0
    want, names = _launched(call)
    _expect(names, kernels)
    store = torch.full((need + 2 * GUARD,), 0xFF, dtype=torch.uint8, device=dev)  # NaN in every type
    ws = store[GUARD:GUARD + need]
    for _ in range(2):  # the second finds what the first has left
        for i, (a, b) in enumerate(zip(call(workspace=ws), want, strict=True)):
            assert (a is None and b is None) or torch.equal(a, b), i
    assert bool((store[:GUARD] == 0xFF).all()) and bool((store[GUARD + need:] == 0xFF).all())
    with pytest.raises(q.QconvError):
        call(workspace=ws[:-1])


@pytest.mark.parametrize("tokens,slots,groups", [(20000, 1, 5), (4097, 1, 300), (70000, 4, 4096)])
def test_sort(dev, tokens, slots, groups):
    ids = torch.arange(tokens * slots, device=dev, dtype=torch.int32).view(tokens, slots) * 7919 % (groups + 1)
    _check(dev, lambda **kw: q.moe_sort(ids, groups, **kw), q.lib().qconv_moe_sort_bytes(tokens, slots, groups),
           [r"moe_count_kernel", r"moe_rank_kernel"])


BIG, SMALL, BIG_W, SMALL_W = r"moe_gemm_kernel<.*, 256>", r"moe_gemm_kernel<.*, 128>", r"moe_gemm_w_kernel<.*, 256>", \
    r"moe_gemm_w_kernel<.*, 128>"
JOIN, JOIN_W, TAIL, COPY, SLOPES = r"moe_join_kernel", r"moe_join_w_kernel", r"moe_tail_kernel", r"dense_realign_kernel", r"ffn_slopes"


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("counts,k,f,gated,kernels", [
    # the gated and the linear form: those of the forward, of the backward
    ([1500, 1300, 40], 2048, 6000, True, ([BIG, TAIL], [SLOPES, BIG, TAIL, BIG_W])),
    ([1500, 1300, 40], 2048, 6000, False, ([BIG, TAIL], [BIG, TAIL])),
    ([3400, 0, 2700], 2048, 4096, True, ([BIG, TAIL], [SLOPES, BIG, TAIL, BIG_W])),
    ([3400, 0, 2700], 2048, 4096, False, ([BIG, TAIL], [BIG, TAIL, BIG_W, JOIN_W])),
    ([2400, 300], 520, 1000, True, (None, [SLOPES, SMALL_W, JOIN_W])),
    ([2400, 300], 520, 1000, False, (None, [SMALL_W, JOIN_W])),
    ([2, 130, 60], 4100, 120, True, ([SMALL, JOIN], [COPY, SLOPES, SMALL, SMALL_W])),
    ([2, 130, 60], 4100, 120, False, ([SMALL, JOIN], [COPY, SMALL, SMALL_W])),
    # copies of operands off 16-byte rows
    ([500, 420], 333, 250, True, ([COPY], [COPY, SLOPES])),
    ([500, 420], 333, 250, False, ([COPY], [COPY])),
])
def test_products(dev, counts, k, f, gated, kernels, dtype):
    x, wg, wu, gh, offsets = _problem(dev, counts, 0, k, f, dtype)
    ws = (wg, wu) if gated else (wg,)
    forward = q.moe_gated_forward if gated else q.moe_linear_forward
    d = ctypes.byref(q.qconv_moe_desc(sum(counts), len(counts), k, f, q.DT_F16 if dtype is torch.float16 else q.DT_BF16, q.ACT_SILU,
                                      k, k, f))
    if kernels[0] is not None:
        call = lambda **kw: [forward(x, *ws, offsets, **kw)[0]] if gated else [forward(x, *ws, offsets, **kw)]
        _check(dev, call, q.lib().qconv_moe_forward_bytes(d, gated), kernels[0])
    if gated:
        pre = q.moe_gated_forward(x, wg, wu, offsets, keep_pre=True)[1]
        call = lambda **kw: q.moe_gated_backward(x, wg, wu, offsets, pre, gh, **kw)
    else:
        call = lambda **kw: q.moe_linear_backward(x, wg, offsets, gh, **kw)
    _check(dev, call, q.lib().qconv_moe_backward_bytes(d, gated), kernels[1])


SHRINK, EXPAND, GRAD, GRAD_JOIN, PARTS_JOIN, TRANSPOSE = r"lora_shrink_kernel", r"lora_expand_kernel", r"lora_grad_kernel", \
    r"lora_grad_join_kernel", r"lora_join_kernel", r"lora_transpose_kernel"


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("m,groups,rank,k,n,how,backward", [
    (1500, 2, 20, 1100, 77, "one", [TRANSPOSE, SHRINK, EXPAND, GRAD, GRAD_JOIN]),
    (8200, 5, 24, 264, 300, "mixed", [TRANSPOSE, SHRINK, EXPAND, GRAD, GRAD_JOIN]),
    (100, 4, 40, 4096, 2500, "runs", [TRANSPOSE, SHRINK, PARTS_JOIN, EXPAND, GRAD]),
    (700, 1, 130, 2055, 3001, "one", [TRANSPOSE, SHRINK, PARTS_JOIN, EXPAND, GRAD, GRAD_JOIN]),
])
def test_adapters(dev, m, groups, rank, k, n, how, backward, dtype):
    s = _lora_problem(dev, m, groups, rank, k, n, dtype, how)
    offsets, order, _ = q.moe_sort(s["ids"], groups)
    args = s["a"], s["b"], offsets, order
    d = ctypes.byref(q.qconv_lora_desc(m, groups, rank, k, n, q.DT_F16 if dtype is torch.float16 else q.DT_BF16, k, n, n))
    out = lambda: torch.empty_like(s["y"])
    _check(dev, lambda **kw: [q.lora_forward(s["y"], s["x"], *args, s["scale"], out=out(), **kw)[0]],
           q.lib().qconv_lora_forward_bytes(d, 0), [SHRINK, EXPAND])
    mid = q.lora_forward(s["y"], s["x"], *args, s["scale"], keep_mid=True, out=out())[1]
    kept = q.lib().qconv_lora_forward_bytes(d, 1)
    if kept:  # mid is joined from parts in the workspace
        named = order[:int(offsets[-1])].long()
        rows = lambda t: t.view(m, -1)[:len(named), :rank]

        def call(**kw):
            y, v = q.lora_forward(s["y"], s["x"], *args, s["scale"], keep_mid=True, out=out(), **kw)
            return y, rows(v)

        _check(dev, call, kept, [SHRINK, PARTS_JOIN, EXPAND])
    _check(dev, lambda **kw: q.lora_backward(s["x"], *args, mid, s["gy"], s["scale"], **kw), q.lib().qconv_lora_backward_bytes(d),
           backward)
