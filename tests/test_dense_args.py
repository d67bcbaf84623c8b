"""Argument checks of the fully connected operators and of the gradient norm
(CPU only: every call here is refused before a launch, or only asks sizes)."""
import ctypes

import pytest
import torch

import paper_2003_04296_amd as q

P = 1 << 20  # an aligned address that no refused call touches


def _ffn(m=4, k=16, f=24, dtype=q.DT_F16, act=q.ACT_SILU, ld_x=16, ld_w=16, ld_h=24):
    return ctypes.byref(q.qconv_ffn_desc(m, k, f, dtype, act, ld_x, ld_w, ld_h))


BAD_FFN = [dict(m=-1), dict(k=0), dict(f=0), dict(act=3), dict(act=-1), dict(dtype=3), dict(dtype=-1), dict(ld_x=15),
           dict(ld_w=0), dict(ld_h=23), dict(ld_x=1 << 62)]


@pytest.mark.parametrize("bad", BAD_FFN)
def test_ffn_descriptors(bad):
    L, d = q.lib(), _ffn(**bad)
    assert L.qconv_ffn_forward(d, P, P, P, P, None, P, 1 << 40, None) == q.QCONV_EINVAL
    assert L.qconv_ffn_backward(d, P, P, P, P, P, P, P, P, P, 1 << 30, None) == q.QCONV_EINVAL
    assert L.qconv_ffn_backward_bytes(d) == 0


def test_ffn_pointers_and_types():
    L = q.lib()
    for p in ((None, P, P, P, None), (P, None, P, P, None), (P, P, None, P, None), (P, P, P, None, None),
              (P + 1, P, P, P, None), (P, P, P, P + 1, None), (P, P, P, P, P + 4)):
        assert L.qconv_ffn_forward(_ffn(), *p, P, 1 << 40, None) == q.QCONV_EINVAL
    assert L.qconv_ffn_forward(None, P, P, P, P, None, P, 1 << 40, None) == q.QCONV_EINVAL
    assert L.qconv_ffn_forward(_ffn(dtype=q.DT_F32), P, P, P, P, None, P, 1 << 40, None) == q.QCONV_EUNSUPPORTED
    ok = [P] * 9
    for i in (0, 1, 2, 3, 4, 6, 7, 8):  # gx alone may be missing, the weight gradients only together
        a = list(ok)
        a[i] = None
        assert L.qconv_ffn_backward(_ffn(), *a, 1 << 30, None) == q.QCONV_EINVAL, i
    need = L.qconv_ffn_backward_bytes(_ffn())
    assert need >= 4 * 2 * 24 * 2
    assert L.qconv_ffn_backward(_ffn(), *ok, need - 1, None) == q.QCONV_EWORKSPACE
    assert L.qconv_ffn_forward(_ffn(m=0), None, P, P, None, None, None, 0, None) == q.QCONV_OK  # nothing to do, nothing read
    wide = dict(m=256, k=8192, f=64, ld_x=8192, ld_w=8192, ld_h=64)  # few tiles and a long sum: a split product
    need = L.qconv_ffn_forward_bytes(_ffn(**wide))
    assert need > 0 and L.qconv_ffn_forward_bytes(_ffn()) == 0
    assert L.qconv_ffn_forward(_ffn(**wide), P, P, P, P, None, P, need - 1, None) == q.QCONV_EWORKSPACE
    assert L.qconv_ffn_forward(_ffn(**wide), P, P, P, P, None, None, 0, None) == q.QCONV_EINVAL
    assert L.qconv_ffn_forward(_ffn(**wide), P, P, P, P, None, P + 8, need, None) == q.QCONV_EINVAL
    assert L.qconv_ffn_pre_floats(3, 20) == 3 * 2 * 24 and L.qconv_ffn_pre_floats(-1, 20) == 0


def _q4(m=4, n=24, k=100, group=32, dtype=q.DT_BF16, ld_x=100, ld_y=24):
    return ctypes.byref(q.qconv_q4_desc(m, n, k, group, dtype, ld_x, ld_y))


@pytest.mark.parametrize("bad", [dict(m=-1), dict(n=0), dict(k=0), dict(group=16), dict(group=48), dict(dtype=5),
                                 dict(ld_x=99), dict(ld_y=23)])
def test_q4_descriptors(bad):
    L, d = q.lib(), _q4(**bad)
    assert L.qconv_q4_linear(d, P, P, P, None, P, P, 1 << 40, None) == q.QCONV_EINVAL
    assert L.qconv_q4_gated(d, P, P, P, P, P, 0, P, P, 1 << 40, None) == q.QCONV_EINVAL


def test_q4_pointers_types_and_sizes():
    L = q.lib()
    for p in ((None, P, P, None, P), (P, None, P, None, P), (P, P, None, None, P), (P, P, P, None, None),
              (P + 1, P, P, None, P), (P, P + 8, P, None, P), (P, P, P + 8, None, P), (P, P, P, P + 2, P),
              (P, P, P, None, P + 1)):
        assert L.qconv_q4_linear(_q4(), *p, P, 1 << 40, None) == q.QCONV_EINVAL
    assert L.qconv_q4_linear(_q4(dtype=q.DT_F32), P, P, P, None, P, P, 1 << 40, None) == q.QCONV_EUNSUPPORTED
    assert L.qconv_q4_gated(_q4(), P, P, P, None, P, 0, P, P, 1 << 40, None) == q.QCONV_EINVAL
    assert L.qconv_q4_gated(_q4(), P, P, P, P, P, 4, P, P, 1 << 40, None) == q.QCONV_EINVAL
    assert L.qconv_q4_linear(_q4(m=0), None, P, P, None, None, None, 0, None) == q.QCONV_OK
    many = dict(m=256, n=64, k=8192, ld_x=8192, ld_y=64)
    need = L.qconv_q4_workspace_bytes(_q4(**many), 0)
    assert need > 0 and L.qconv_q4_workspace_bytes(_q4(), 1) == 0
    assert L.qconv_q4_linear(_q4(**many), P, P, P, None, P, P, need - 1, None) == q.QCONV_EWORKSPACE
    assert L.qconv_q4_linear(_q4(**many), P, P, P, None, P, None, need, None) == q.QCONV_EINVAL
    assert L.qconv_q4_gated(_q4(**many), P, P, P, P, P, 0, P, P, need - 1, None) == q.QCONV_EWORKSPACE
    assert L.qconv_q4_code_bytes(3, 100, 32) == 3 * 64 and L.qconv_q4_scale_bytes(3, 100, 32) == 3 * 4 * 2
    assert L.qconv_q4_code_bytes(3, 100, 33) == 0 and L.qconv_q4_scale_bytes(0, 100, 32) == 0
    ok = (P, q.DT_F32, 4, 100, 100, 32, 6, P, P, None)
    for i, v in ((0, None), (1, 3), (2, 0), (3, 0), (4, 99), (5, 16), (6, 5), (7, None), (8, None), (7, P + 8), (0, P + 2)):
        a = list(ok)
        a[i] = v
        assert L.qconv_q4_pack(*a) == q.QCONV_EINVAL, (i, v)


def _grads(sizes, types=None, ptrs=None):
    n = len(sizes)
    return (n, (ctypes.c_void_p * n)(*(ptrs or [P] * n)), (ctypes.c_int64 * n)(*sizes),
            (ctypes.c_int * n)(*(types or [q.DT_F32] * n)))


def test_grad_arguments():
    L = q.lib()
    n, p, s, t = _grads([5, 7])
    need = L.aqe_grad_norm_bytes(n, s)
    assert need >= 8
    for a in (_grads([5, -1]), _grads([5, 7], [0, 3]), _grads([5, 7], ptrs=[P, None]), _grads([5, 7], ptrs=[P, P + 2])):
        assert L.aqe_grad_norm(*a, P, P, 1 << 20, None) == q.QCONV_EINVAL
        assert L.aqe_clip_grads(a[0], a[1], p, a[2], a[3], 1.0, P, P, 1 << 20, None) == q.QCONV_EINVAL
    assert L.aqe_grad_norm(-1, p, s, t, P, P, 1 << 20, None) == q.QCONV_EINVAL
    assert L.aqe_grad_norm(n, None, s, t, P, P, 1 << 20, None) == q.QCONV_EINVAL
    assert L.aqe_grad_norm(n, p, s, t, None, P, 1 << 20, None) == q.QCONV_EINVAL
    assert L.aqe_grad_norm(n, p, s, t, P, None, 1 << 20, None) == q.QCONV_EINVAL
    assert L.aqe_grad_norm(n, p, s, t, P, P, need - 1, None) == q.QCONV_EWORKSPACE
    assert L.aqe_grad_norm(*_grads([1 << 40]), P, P, 1 << 40, None) == q.QCONV_EUNSUPPORTED
    for m in (-1.0, float("nan")):
        assert L.aqe_clip_grads(n, p, p, s, t, m, P, P, 1 << 20, None) == q.QCONV_EINVAL
    assert L.aqe_clip_grads(n, p, None, s, t, 1.0, P, P, 1 << 20, None) == q.QCONV_EINVAL
    bad = _grads([5, 7], ptrs=[P, None])[1]
    assert L.aqe_clip_grads(n, p, bad, s, t, 1.0, P, P, 1 << 20, None) == q.QCONV_EINVAL


def test_host_tensors_are_refused():
    x, w = torch.zeros((2, 32), dtype=torch.float16), torch.zeros((8, 32), dtype=torch.float16)
    codes, scales = torch.zeros((8, 16), dtype=torch.uint8), torch.zeros((8, 1), dtype=torch.bfloat16)
    for bad in (lambda: q.ffn_forward(x, w, w), lambda: q.ffn_backward(x, w, w, torch.zeros(32), x),
                lambda: q.q4_pack(w), lambda: q.q4_linear(x, codes, scales),
                lambda: q.q4_gated(x, codes, scales, codes, scales), lambda: q.aqe_grad_norm([w]),
                lambda: q.aqe_clip_grads([w], 1.0)):
        with pytest.raises(ValueError):
            bad()
