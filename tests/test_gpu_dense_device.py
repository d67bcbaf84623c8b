"""Tensors of another device than the one a call would go to (run with -m gpu).
One device is enough: the current device's number, and a stream's, are made to
look like another's."""
import types

import pytest
import torch

import paper_2003_04296_amd as q

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def calls():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    q.lib()
    dev = torch.device("cuda:0")
    x = torch.zeros((3, 32), dtype=torch.bfloat16, device=dev)
    w = torch.zeros((8, 32), dtype=torch.bfloat16, device=dev)
    codes, scales = q.q4_pack(w, 32)
    gh = torch.zeros((3, 8), dtype=torch.bfloat16, device=dev)
    _, pre = q.ffn_forward(x, w, w, keep_pre=True)
    norm = torch.zeros((), device=dev)
    return [lambda **s: q.ffn_forward(x, w, w, **s), lambda **s: q.ffn_backward(x, w, w, pre, gh, **s),
            lambda **s: q.q4_pack(w, 32, **s), lambda **s: q.q4_linear(x, codes, scales, **s),
            lambda **s: q.q4_gated(x, codes, scales, codes, scales, **s), lambda **s: q.aqe_grad_norm([x, w], **s),
            lambda **s: q.aqe_clip_grads([x.clone()], 1.0, **s), lambda **s: q.aqe_grad_norm([], norm=norm, **s)]


@pytest.mark.parametrize("i", range(8))
def test_other_current_device(calls, i, monkeypatch):
    calls[i]()
    monkeypatch.setattr(q, "_current_device", lambda: 1, raising=False)
    with pytest.raises(ValueError, match="cuda:1"):
        calls[i]()


@pytest.mark.parametrize("i", range(8))
def test_stream_of_another_device(calls, i):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    calls[i](stream=side)
    torch.cuda.synchronize()
    with pytest.raises(ValueError, match="cuda:1"):
        calls[i](stream=types.SimpleNamespace(device_index=1, cuda_stream=side.cuda_stream))
