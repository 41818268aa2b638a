"""How the linear-attention layer's entry points stand in torch's autograd (CPU only: stand-ins for the library's calls)."""
import numpy as np
import pytest
import torch
from torch.autograd import forward_ad

from paper_2609_33133_amd import api, autograd
from paper_2609_33133_amd.api import GroupBatch

CU = ([0, 10, 25], [0, 2, 3], [0, 5, 12, 20])


def leaves(d=64):
    z = lambda t, h: torch.zeros(t, h, d, dtype=torch.bfloat16)
    return [z(25, 4), z(25, 2), z(25, 2), z(20, 4), z(20, 2), z(20, 2)]


@pytest.fixture
def stand_ins(monkeypatch):
    monkeypatch.setattr(api, "head_norm_fwd", lambda x, *a, **k: x.detach().clone())
    monkeypatch.setattr(api, "linear_fwd", lambda b, dec, q_p, k_p, v_p, q_r, *a, **k:
                        (q_p.detach().clone(), q_r.detach().clone(), None, None))


def dual(t):
    return forward_ad.make_dual(t, torch.ones_like(t))


@pytest.mark.parametrize("grad", [True, False])
@pytest.mark.parametrize("which", range(4))
def test_head_norm_has_no_forward_derivatives(stand_ins, which, grad):
    t = [torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.ones(2, 64), torch.zeros(2, 64),
         torch.zeros(3, 2, 64, dtype=torch.bfloat16)]
    with forward_ad.dual_level(), torch.set_grad_enabled(grad):
        autograd.head_norm(*t)
        t[which] = dual(t[which])
        with pytest.raises(NotImplementedError):
            autograd.head_norm(*t)


@pytest.mark.parametrize("grad", [True, False])
@pytest.mark.parametrize("which", range(7))
def test_linear_attention_has_no_forward_derivatives(stand_ins, which, grad):
    b, x, state = GroupBatch(*CU, 4, 2, 64), leaves(), torch.zeros(2, 2, 64, 64)
    with forward_ad.dual_level(), torch.set_grad_enabled(grad):
        autograd.group_linear_attention(*x, b, 0.9, state=state)
        if which < 6:
            x[which] = dual(x[which])
        else:
            state = dual(state)
        with pytest.raises(NotImplementedError):
            autograd.group_linear_attention(*x, b, 0.9, state=state)


def test_a_decay_has_no_forward_derivative(stand_ins):
    b, x = GroupBatch(*CU, 4, 2, 64), leaves()
    with forward_ad.dual_level(), pytest.raises(ValueError, match="constant"):
        autograd.group_linear_attention(*x, b, dual(torch.tensor([0.9, 0.9])))
