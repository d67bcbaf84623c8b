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
