"""Argument checks of the operators for rows that go to different weights (CPU
only: every call here is refused before a launch, or only asks sizes)."""
import ctypes

import pytest
import torch

import paper_2003_04296_amd as q

P = 1 << 20  # an aligned address that no refused call touches


def test_sort_arguments():
    L = q.lib()
    ok = dict(ids=P, wide=0, tokens=4, slots=2, ld=2, groups=8, offsets=P, order=P, place=P, ws=None, nbytes=0)

    def call(**kw):
        return L.qconv_moe_sort(*{**ok, **kw}.values(), None)

    for bad in (dict(tokens=-1), dict(slots=0), dict(groups=0), dict(groups=-3), dict(ld=1), dict(ld=1 << 50), dict(ids=None),
                dict(offsets=None), dict(order=None), dict(place=None), dict(ids=P + 2), dict(ids=P + 4, wide=1),
                dict(offsets=P + 2), dict(order=P + 1), dict(place=P + 2), dict(ws=P + 8)):
        assert call(**bad) == q.QCONV_EINVAL, bad
    assert call(groups=4097) == q.QCONV_EUNSUPPORTED
    assert call(tokens=1 << 30, slots=4, ld=4) == q.QCONV_EUNSUPPORTED
    need = L.qconv_moe_sort_bytes(1 << 16, 2, 8)
    assert need > 0 and L.qconv_moe_sort_bytes(16, 2, 8) == 0 and L.qconv_moe_sort_bytes(16, 2, 5000) == 0
    assert call(tokens=1 << 16, ws=None) == q.QCONV_EINVAL
    assert call(tokens=1 << 16, ws=P, nbytes=need - 1) == q.QCONV_EWORKSPACE


def _rows(tokens=4, slots=2, width=16, dtype=q.DT_F16, ld_tokens=16, ld_rows=16):
    return ctypes.byref(q.qconv_moe_rows_desc(tokens, slots, width, dtype, ld_tokens, ld_rows))


@pytest.mark.parametrize("bad", [dict(tokens=-1), dict(slots=0), dict(width=0), dict(dtype=3), dict(dtype=-1),
                                 dict(ld_tokens=15), dict(ld_rows=15), dict(ld_rows=1 << 50)])
def test_rows_descriptors(bad):
    L, d = q.lib(), _rows(**bad)
    assert L.qconv_moe_gather(d, P, P, P, None) == q.QCONV_EINVAL
    assert L.qconv_moe_combine(d, P, P, P, P, None) == q.QCONV_EINVAL
    assert L.qconv_moe_combine_backward(d, P, P, P, P, P, 16, P, None) == q.QCONV_EINVAL


def test_rows_pointers():
    L = q.lib()
    big = _rows(tokens=1 << 30, slots=4)
    assert L.qconv_moe_gather(big, P, P, P, None) == q.QCONV_EUNSUPPORTED
    for a in ((None, P, P), (P, None, P), (P, P, None), (P + 1, P, P), (P, P + 2, P), (P, P, P + 1)):
        assert L.qconv_moe_gather(_rows(), *a, None) == q.QCONV_EINVAL, a
        assert L.qconv_moe_combine(_rows(), a[0], a[1], P, a[2], None) == q.QCONV_EINVAL, a
    assert L.qconv_moe_gather(_rows(dtype=q.DT_F32), P + 2, P, P, None) == q.QCONV_EINVAL
    assert L.qconv_moe_combine(_rows(), P, P, P + 2, P, None) == q.QCONV_EINVAL
    assert L.qconv_moe_gather(None, P, P, P, None) == q.QCONV_EINVAL
    for a in ((None, P, P, P, P, 16, P), (P, None, P, P, P, 16, P), (P, P, None, P, P, 16, P), (P, P, P, P, P, 15, P),
              (P, P, P, P, P + 1, 16, P), (P, P, P, P + 2, P, 16, P), (P, P, P, P, P, 16, P + 2)):
        assert L.qconv_moe_combine_backward(_rows(), *a, None) == q.QCONV_EINVAL, a
    # nothing to do, nothing read
    none = _rows(tokens=0)
    assert L.qconv_moe_gather(none, None, None, None, None) == q.QCONV_OK
    assert L.qconv_moe_combine(none, None, None, None, None, None) == q.QCONV_OK
    assert L.qconv_moe_combine_backward(none, None, None, None, None, None, 0, None, None) == q.QCONV_OK


def _moe(rows=4, groups=3, k=16, f=24, dtype=q.DT_BF16, act=q.ACT_SILU, ld_x=16, ld_w=16, ld_h=24):
    return ctypes.byref(q.qconv_moe_desc(rows, groups, k, f, dtype, act, ld_x, ld_w, ld_h))


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(groups=0), dict(k=0), dict(f=0), dict(dtype=3), dict(act=3), dict(act=-1),
                                 dict(ld_x=15), dict(ld_w=15), dict(ld_h=23), dict(ld_w=1 << 62)])
def test_products_descriptors(bad):
    L, d = q.lib(), _moe(**bad)
    assert L.qconv_moe_gated_forward(d, P, P, P, P, P, None, P, 1 << 40, None) == q.QCONV_EINVAL
    assert L.qconv_moe_linear_forward(d, P, P, P, P, P, 1 << 40, None) == q.QCONV_EINVAL
    assert L.qconv_moe_gated_backward(d, P, P, P, P, P, P, P, P, P, P, 1 << 40, None) == q.QCONV_EINVAL
    assert L.qconv_moe_linear_backward(d, P, P, P, P, P, P, P, 1 << 40, None) == q.QCONV_EINVAL
    assert L.qconv_moe_forward_bytes(d, 1) == 0 and L.qconv_moe_backward_bytes(d, 1) == 0


def test_products_pointers_and_types():
    L = q.lib()
    for d in (_moe(dtype=q.DT_F32), _moe(groups=4097)):
        assert L.qconv_moe_gated_forward(d, P, P, P, P, P, None, P, 1 << 40, None) == q.QCONV_EUNSUPPORTED
        assert L.qconv_moe_linear_backward(d, P, P, P, P, P, P, P, 1 << 40, None) == q.QCONV_EUNSUPPORTED
    for i in range(5):  # x, weights, offsets, h
        a = [P] * 5
        for v in (None, P + 1):
            a[i] = v
            assert L.qconv_moe_gated_forward(_moe(), *a, None, P, 1 << 40, None) == q.QCONV_EINVAL, (i, v)
            if i != 2:
                b = a[:2] + a[3:]
                assert L.qconv_moe_linear_forward(_moe(), *b, P, 1 << 40, None) == q.QCONV_EINVAL, (i, v)
    assert L.qconv_moe_gated_forward(_moe(), P, P, P, P, P, P + 4, P, 1 << 40, None) == q.QCONV_EINVAL
    need = L.qconv_moe_backward_bytes(_moe(), 1)
    assert need >= 4 * 2 * 24 * 2
    ok = [P] * 9
    for i in (0, 1, 2, 3, 4, 5, 7, 8):  # gx alone may be missing, the weight gradients only together
        a = list(ok)
        a[i] = None
        assert L.qconv_moe_gated_backward(_moe(), *a, P, need, None) == q.QCONV_EINVAL, i
    assert L.qconv_moe_gated_backward(_moe(), *ok, P, need - 1, None) == q.QCONV_EWORKSPACE
    assert L.qconv_moe_gated_backward(_moe(), *ok, None, need, None) == q.QCONV_EINVAL
    assert L.qconv_moe_gated_backward(_moe(), *ok, P + 8, need, None) == q.QCONV_EINVAL
    # odd rows of gy, x and w are copied
    odd = dict(f=25, ld_h=25)
    need = L.qconv_moe_backward_bytes(_moe(**odd), 0)
    assert need > 0 and L.qconv_moe_backward_bytes(_moe(), 0) == 0
    assert L.qconv_moe_linear_backward(_moe(**odd), P, P, P, P, P, P, P, need - 1, None) == q.QCONV_EWORKSPACE
    many = dict(rows=4096, k=17, ld_x=17, ld_w=17)
    need = L.qconv_moe_forward_bytes(_moe(**many), 0)
    assert need > 0 and L.qconv_moe_forward_bytes(_moe(**many), 1) > need
    assert L.qconv_moe_linear_forward(_moe(**many), P, P, P, P, P, need - 1, None) == q.QCONV_EWORKSPACE
    assert L.qconv_moe_linear_forward(_moe(**many), P, P, P, P, None, need, None) == q.QCONV_EINVAL
    assert L.qconv_moe_linear_forward(_moe(rows=0), None, P, P, None, None, 0, None) == q.QCONV_OK


def test_host_tensors_are_refused():
    x, w = torch.zeros((4, 16), dtype=torch.float16), torch.zeros((3, 8, 16), dtype=torch.float16)
    h, pre = torch.zeros((4, 8), dtype=torch.float16), torch.zeros(64)
    ids, offsets = torch.zeros(4, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    for bad in (lambda: q.moe_sort(ids, 3), lambda: q.moe_gather(x, ids), lambda: q.moe_combine(x, ids),
                lambda: q.moe_gather_backward(x, ids), lambda: q.moe_combine_backward(x, x, ids),
                lambda: q.moe_gated_forward(x, w, w, offsets), lambda: q.moe_linear_forward(x, w, offsets),
                lambda: q.moe_gated_backward(x, w, w, offsets, pre, h), lambda: q.moe_linear_backward(x, w, offsets, h)):
        with pytest.raises(ValueError):
            bad()


def _lora(m=4, groups=3, rank=8, k=16, n=24, dtype=q.DT_BF16, ld_x=16, ld_y=24, ld_out=24):
    return ctypes.byref(q.qconv_lora_desc(m, groups, rank, k, n, dtype, ld_x, ld_y, ld_out))


@pytest.mark.parametrize("bad", [dict(m=-1), dict(groups=0), dict(rank=0), dict(k=0), dict(n=0), dict(dtype=3), dict(ld_x=15),
                                 dict(ld_y=23), dict(ld_x=1 << 62)])
def test_lora_descriptors(bad):
    L, d = q.lib(), _lora(**bad)
    assert L.qconv_lora_forward(d, P, P, P, P, P, P, P, P, P, P, 1 << 40, None) == q.QCONV_EINVAL
    assert L.qconv_lora_backward(d, P, P, P, P, P, P, P, P, P, P, P, P, 1 << 40, None) == q.QCONV_EINVAL
    assert L.qconv_lora_forward_bytes(d, 0) == 0 and L.qconv_lora_backward_bytes(d) == 0


def test_lora_pointers_and_sizes():
    L = q.lib()
    for bad in (dict(dtype=q.DT_F32), dict(rank=257), dict(groups=4097)):
        assert L.qconv_lora_forward(_lora(**bad), P, P, P, P, P, P, P, P, P, P, 1 << 40, None) == q.QCONV_EUNSUPPORTED, bad
        assert L.qconv_lora_backward(_lora(**bad), P, P, P, P, P, P, P, P, P, P, P, P, 1 << 40, None) == q.QCONV_EUNSUPPORTED
    ok = [P] * 9  # x, a, b, offsets, order, scale, y, out, mid
    for i in range(9):
        for v in (None, P + 1):
            if v is None and i in (5, 8):
                continue
            a = list(ok)
            a[i] = v
            assert L.qconv_lora_forward(_lora(), *a, P, 1 << 40, None) == q.QCONV_EINVAL, (i, v)
    assert L.qconv_lora_forward(_lora(ld_out=25), *ok, P, 1 << 40, None) == q.QCONV_EINVAL  # y itself, by another stride
    assert L.qconv_lora_forward(_lora(ld_out=23), *ok, P, 1 << 40, None) == q.QCONV_EINVAL
    need = L.qconv_lora_forward_bytes(_lora(m=4096), 0)
    assert need > 0 and L.qconv_lora_forward_bytes(_lora(), 0) == 0
    assert L.qconv_lora_forward(_lora(m=4096), *ok[:8], None, P, need - 1, None) == q.QCONV_EWORKSPACE
    assert L.qconv_lora_forward(_lora(m=4096), *ok[:8], None, None, need, None) == q.QCONV_EINVAL
    assert L.qconv_lora_forward(_lora(m=4096), *ok[:8], None, P + 8, need, None) == q.QCONV_EINVAL
    ok = [P] * 11  # x, a, b, offsets, order, scale, mid, gy, gx, ga, gb
    for i in range(11):
        for v in (None, P + 1):
            if v is None and i in (5, 8):
                continue
            a = list(ok)
            a[i] = v
            assert L.qconv_lora_backward(_lora(), *a, P, 1 << 40, None) == q.QCONV_EINVAL, (i, v)
    need = L.qconv_lora_backward_bytes(_lora())
    assert need > 0 and L.qconv_lora_backward(_lora(), *ok, P, need - 1, None) == q.QCONV_EWORKSPACE
    assert L.qconv_lora_backward(_lora(), *ok, None, need, None) == q.QCONV_EINVAL
    assert L.qconv_lora_forward(_lora(m=0), None, P, P, P, None, None, None, None, None, None, 0, None) == q.QCONV_OK
    assert L.qconv_lora_mid_floats(3, 9) == 36 and L.qconv_lora_mid_floats(-1, 9) == 0 and L.qconv_lora_mid_floats(3, 300) == 0


def test_lora_host_tensors_are_refused():
    x, y = torch.zeros((4, 16), dtype=torch.float16), torch.zeros((4, 24), dtype=torch.float16)
    a, b = torch.zeros((3, 8, 16), dtype=torch.float16), torch.zeros((3, 24, 8), dtype=torch.float16)
    ids = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        q.lora_forward(y, x, a, b, ids, ids)
    with pytest.raises(ValueError):
        q.lora_backward(x, a, b, ids, ids, torch.zeros(32), y)
