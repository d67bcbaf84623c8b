"""Refusals of the fully connected operators' Python entry points that need no
GPU: host memory that would reach a kernel."""
import pytest
import torch

import paper_2003_04296_amd as q


@pytest.mark.parametrize("call", [lambda n: q.aqe_grad_norm([], norm=n), lambda n: q.aqe_clip_grads([], 1.0, norm=n),
                                  lambda n: q.aqe_clip_grads([], 1.0, out=[], norm=n)])
def test_host_norm_of_no_gradients(call):
    with pytest.raises(ValueError):
        call(torch.zeros(()))
