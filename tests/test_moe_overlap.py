"""Results of the operators for rows that go to different weights that lie over what
the call still reads are refused (CPU only: every call here is refused before a launch)."""
import ctypes

import pytest

import paper_2003_04296_amd as q

P = 1 << 24  # addresses that no refused call touches, far apart
FAR = [P + (i << 28) for i in range(16)]


def _lora(m=100, groups=3, rank=8, k=40, n=40, ld_x=40, ld_y=40, ld_out=40):
    return ctypes.byref(q.qconv_lora_desc(m, groups, rank, k, n, q.DT_BF16, ld_x, ld_y, ld_out))


def _lora_forward(d, **at):
    a = dict(x=FAR[0], a=FAR[1], b=FAR[2], offsets=FAR[3], order=FAR[4], scale=FAR[5], y=FAR[6], out=FAR[7], mid=FAR[8])
    return q.lib().qconv_lora_forward(d, *{**a, **at}.values(), FAR[9], 1 << 20, None)


STARTS = [dict(out=FAR[0]), dict(out=FAR[0], y=FAR[0]), dict(out=FAR[6] + 2), dict(out=FAR[2]), dict(out=FAR[5])]
ENDS = [dict(out=FAR[0] + 99 * 80 + 78), dict(out=FAR[0] - 99 * 80 - 78), dict(out=FAR[6] - 80), dict(out=FAR[1] + 3 * 8 * 40 * 2 - 2),
        dict(out=FAR[3] + 12), dict(out=FAR[4] + 396), dict(out=FAR[8] + 3196)]


@pytest.mark.parametrize("m,at", [(m, at) for m in (1, 100, 5000) for at in STARTS] + [(m, at) for m in (100, 5000) for at in ENDS])
def test_adapters_over_their_inputs(m, at):
    """One launch for few tokens sums a row of x in every block of the result's columns."""
    assert _lora_forward(_lora(m=m), **at) == q.QCONV_EINVAL


def test_rows_of_one_tensor():
    """x and the result as columns of one tensor: they may not share columns, in rows of one stride or of two."""
    for off in (0, 2, 78, 200 - 78):
        assert _lora_forward(_lora(ld_x=100, ld_out=100), out=FAR[0] + off) == q.QCONV_EINVAL, off
    # rows of 200 and of 280 bytes: the third and the eighth meet
    assert _lora_forward(_lora(ld_x=100, ld_out=140), out=FAR[0] + 90) == q.QCONV_EINVAL


def test_sort_over_its_ids():
    def call(wide=0, tokens=50, slots=3, ld=3, **at):
        a = dict(ids=FAR[0], wide=wide, tokens=tokens, slots=slots, ld=ld, groups=8, offsets=FAR[1], order=FAR[2], place=FAR[3])
        return q.lib().qconv_moe_sort(*{**a, **at}.values(), FAR[4], 1 << 20, None)

    for at in (dict(order=FAR[0]), dict(offsets=FAR[0] + 596), dict(place=FAR[0] + 4), dict(place=FAR[0], wide=1),
               dict(place=FAR[0], ld=4), dict(order=FAR[0] - 596)):
        assert call(**at) == q.QCONV_EINVAL, at


def _rows(tokens=20, slots=2, width=16, ld_tokens=16, ld_rows=16):
    return ctypes.byref(q.qconv_moe_rows_desc(tokens, slots, width, q.DT_F16, ld_tokens, ld_rows))


def test_rows_over_their_inputs():
    L, bad = q.lib(), q.QCONV_EINVAL
    x, place, rows, w, y, gw = FAR[:6]
    for slots in (1, 2):
        d = _rows(slots=slots)
        assert L.qconv_moe_gather(d, x, place, x, None) == bad
        assert L.qconv_moe_gather(d, x, place, x + 19 * 32 + 30, None) == bad
        assert L.qconv_moe_gather(d, x, place, place, None) == bad
        assert L.qconv_moe_combine(d, rows, place, w, rows, None) == bad
        assert L.qconv_moe_combine(d, rows, place, w, rows - 20 * 32 + 2, None) == bad
        assert L.qconv_moe_combine(d, rows, place, w, w, None) == bad
        for grows, gweights in ((y, None), (y, gw), (rows + 2, gw), (place, gw), (w, gw), (x, y), (x, rows), (x, w + 4), (x, x),
                                (None, place)):
            assert L.qconv_moe_combine_backward(d, y, rows, place, w, grows, 16, gweights, None) == bad, (grows, gweights)
        assert L.qconv_moe_combine_backward(d, y, rows, place, w, rows, 17, gw, None) == bad


def _moe(rows=40, groups=3, k=16, f=16):
    return ctypes.byref(q.qconv_moe_desc(rows, groups, k, f, q.DT_BF16, q.ACT_SILU, k, k, f))


@pytest.mark.parametrize("rows", [1, 40, 3000])
def test_products_over_their_inputs(rows):
    L, bad, d = q.lib(), q.QCONV_EINVAL, _moe(rows)
    x, wg, wu, offsets, h, pre, gh, gx, gwg, gwu, ws = FAR[:11]
    for to, kept in ((x, None), (wg, None), (wu + 3 * 16 * 32 - 2, None), (offsets + 12, None), (h, h), (h, x), (h, wu), (pre, pre)):
        assert L.qconv_moe_gated_forward(d, x, wg, wu, offsets, to, kept, ws, 1 << 30, None) == bad, (to, kept)
    for to in (x, x + 30, wg, offsets):
        assert L.qconv_moe_linear_forward(d, x, wg, offsets, to, ws, 1 << 30, None) == bad, to
    for a in ((x, gwg, gwu), (gx, x, gwu), (gx, gwg, x), (wg, gwg, gwu), (wu, None, None), (gx, gx, gwu), (gx, gwg, gwg + 2),
              (gx, offsets, gwu)):
        assert L.qconv_moe_gated_backward(d, x, wg, wu, offsets, pre, gh, *a, ws, 1 << 30, None) == bad, a
    for a in ((x, gwg), (gh, None), (gx, gh), (gx, x), (wg, None), (gx, gx + 2), (offsets, None)):
        assert L.qconv_moe_linear_backward(d, x, wg, offsets, gh, *a, ws, 1 << 30, None) == bad, a


@pytest.mark.parametrize("m", [1, 100, 5000])
def test_adapters_gradients_over_their_inputs(m):
    x, a, b, offsets, order, scale, mid, gy, gx, ga, gb, ws = FAR[:12]
    for to in ((x, ga, gb), (gy, ga, gb), (gx, x, gb), (gx, gy, gb), (gx, ga, gy), (mid, ga, gb), (gx, mid, gb), (gx, ga, mid),
               (gx, gx, gb), (gx, ga, ga), (gx, ga, gx), (order, None, None), (gx, offsets, gb), (gx, ga, scale)):
        assert q.lib().qconv_lora_backward(_lora(m), x, a, b, offsets, order, scale, mid, gy, *to, ws, 1 << 30, None) == \
            q.QCONV_EINVAL, to
