"""How the linear-attention layer's entry points stand in torch's autograd (CPU only: stand-ins for the library's calls)."""
import numpy as np
import pytest
import torch
from torch.autograd import forward_ad
from torch.utils._python_dispatch import TorchDispatchMode

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


class Reached(Exception):
    """A call went past the checks of its arguments."""


class FakeOn:
    """api._On for host tensors: the library is not reached."""

    def __init__(self, tensors, stream=None):
        pass

    def __enter__(self):
        raise Reached

    def __exit__(self, *exc):
        pass


def step_args():
    z = lambda *s: torch.zeros(3, *s, 64, dtype=torch.bfloat16)
    return dict(q=z(4), k=z(2), v=z(2), state=torch.zeros(3, 2, 64, 64), state_out=torch.zeros(3, 2, 64, 64), o=z(4))


def step(a):
    return api.linear_step(a["q"], a["k"], a["v"], 0.9, a["state"], state_out=a["state_out"], o=a["o"])


@pytest.mark.parametrize("name", ["q", "k", "v", "state", "state_out", "o"])
def test_a_step_forms_no_gradient_and_says_so(monkeypatch, name):
    monkeypatch.setattr(api, "_On", FakeOn)
    monkeypatch.setattr(api, "_need", lambda *a: None)  # (it asks for device tensors)
    a = step_args()
    with pytest.raises(Reached):
        step(a)
    a[name].requires_grad_(True)
    with pytest.raises(ValueError, match="no_grad"):
        step(a)
    with torch.no_grad(), pytest.raises(Reached):
        step(a)
    with torch.inference_mode(), pytest.raises(Reached):
        step(a)
    for grad in (True, False):
        a = step_args()
        with forward_ad.dual_level(), torch.set_grad_enabled(grad):
            a[name] = dual(a[name])
            with pytest.raises(ValueError, match="tangent"):
                step(a)


@pytest.fixture
def library(monkeypatch):
    """Calls that pass the checks of their arguments and write nothing."""
    class On:
        def __init__(self, tensors, stream=None):
            self.device = torch.device("cpu")

        def __enter__(self):
            return 0

        def __exit__(self, *exc):
            pass

    class Lib:
        def __getattr__(self, name):
            return lambda *a: 1024 if name.endswith("workspace_size") else 0
    monkeypatch.setattr(api, "_On", On)
    monkeypatch.setattr(api._lib, "load", lambda: Lib())


def written(call, given, *unwritten):
    """Every tensor in `given` counts as written by the call, none of the others does."""
    for t in given.values():
        assert t._version == 0
    before = [t._version for t in unwritten]
    call(**given)
    assert not [n for n, t in given.items() if t._version == 0]
    assert [t._version for t in unwritten] == before


def test_what_a_call_writes_counts_as_written(library):
    """A tensor that another op has saved for its backward is not replaced unnoticed."""
    b, x = GroupBatch(*CU, 4, 2, 64), leaves()
    do = [x[0].clone(), x[3].clone()]
    like = lambda *names: {n: x[{"q": 0, "k": 1, "v": 2, "o": 0}[n.lstrip("d")[0]] + 3 * n.endswith("_r")].clone() for n in names}
    ws = lambda: torch.zeros(1024, dtype=torch.uint8)
    states = dict(state_p=torch.zeros(2, 2, 64, 64), state_r=torch.zeros(3, 2, 64, 64))
    written(lambda **k: api.linear_fwd(b, 0.9, *x, **k), dict(like("o_p", "o_r"), ws=ws(), **states), *x)
    kept = ws()
    written(lambda **k: api.linear_bwd(b, 0.9, *x[:3], do[0], *x[3:], do[1], fwd_ws=kept, **k),
            dict(like("dq_p", "dk_p", "dv_p", "dq_r", "dk_r", "dv_r"), ws=ws()), *x, *do, kept)
    a = step_args()
    written(lambda **k: api.linear_step(a["q"], a["k"], a["v"], 0.9, a["state"], **k),
            {n: a[n] for n in ("state_out", "o")}, a["q"], a["k"], a["v"], a["state"])
    w = lambda: torch.zeros(4, 64)
    written(lambda **k: api.head_norm_fwd(x[0], **k), {"y": x[0].clone()}, x[0])
    written(lambda **k: api.head_norm_bwd(x[0], do[0], w(), w(), x[0].clone(), **k),
            {"dx": x[0].clone(), "dgate": x[0].clone(), "dweight": w(), "dbias": w(), "ws": ws()}, x[0], do[0])


def test_a_state_saved_for_a_backward_is_not_updated_in_place_unnoticed(library):
    a = step_args()
    weight = torch.ones(1, requires_grad=True)
    loss = (a["state"] * weight).sum()  # saves the state
    with torch.no_grad():
        api.linear_step(a["q"], a["k"], a["v"], 0.9, a["state"], state_out=a["state"])
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_what_a_refused_call_would_have_written_does_not(library):
    a = step_args()
    with pytest.raises((ValueError, TypeError)):
        api.linear_step(a["q"], a["k"], a["v"].float(), 0.9, a["state"], state_out=a["state_out"])
    assert a["state_out"]._version == 0


def test_a_learned_state_and_decay_serve_inference(stand_ins):
    """Refused where a gradient could be asked for, constants as any other where it cannot."""
    b, x = GroupBatch(*CU, 4, 2, 64), leaves()
    state = torch.nn.Parameter(torch.zeros(2, 2, 64, 64))
    decay = torch.nn.Parameter(torch.tensor([0.9, 0.8]))
    for kw in (dict(decay=0.9, state=state), dict(decay=decay)):
        with pytest.raises(ValueError, match="constant"):
            autograd.group_linear_attention(*x, b, **kw)
    for off in (torch.no_grad, torch.inference_mode):
        with off():
            o_p, o_r = autograd.group_linear_attention(*x, b, decay, state=state)
            assert o_p.shape == x[0].shape and o_r.shape == x[3].shape
            assert api._decay(decay, 2).tolist() == [np.float32(0.9), np.float32(0.8)]


def train(monkeypatch, state, return_state=False):
    """A step of group_linear_attention on stand-ins; what _linear_bwd was handed is kept."""
    b, x = GroupBatch(*CU, 4, 2, 64), [t.requires_grad_(True) for t in leaves()]
    states = (torch.zeros(2, 2, 64, 64), torch.zeros(3, 2, 64, 64)) if return_state else (None, None)
    handed = []

    class On:
        def __init__(self, tensors, stream=None):
            pass

        def __enter__(self):
            return 0

        def __exit__(self, *exc):
            pass
    monkeypatch.setattr(api, "linear_fwd", lambda b, dec, q_p, k_p, v_p, q_r, *a, **k:
                        (q_p.detach().clone(), q_r.detach().clone(), *states))
    monkeypatch.setattr(api, "_On", On)
    monkeypatch.setattr(api, "_linear_bwd", lambda *a: handed.append(a))
    return x, autograd.group_linear_attention(*x, b, 0.9, state=state, return_state=return_state), handed


def test_a_state_may_be_updated_between_forward_and_backward(monkeypatch):
    """The backward reads the states that the forward left in its workspace, not the one it began from."""
    state = torch.zeros(2, 2, 64, 64)
    x, (o_p, o_r), handed = train(monkeypatch, state)
    state.add_(1)
    torch.autograd.grad((o_p, o_r), x, (torch.zeros_like(o_p), torch.zeros_like(o_r)))
    (_, _, tensors, fwd_ws, _, _), = handed
    assert tensors[8] is None and fwd_ws is not None


def test_states_returned_in_training_get_no_gradients_made_of_zeros(monkeypatch):
    """A state is [d, d] per head, tree and branch in fp32: nothing of that size is filled with zeros for the backward. An
    output outside the loss still has a gradient of zeros."""
    x, (o_p, o_r, state_p, state_r), handed = train(monkeypatch, None, return_state=True)
    assert not state_p.requires_grad and not state_r.requires_grad
    made = []

    class Sizes(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            r = func(*args, **(kwargs or {}))
            if isinstance(r, torch.Tensor):
                made.append(r.shape)
            return r
    with Sizes(), torch.autograd.set_multithreading_enabled(False):
        torch.autograd.grad(o_r, x, torch.ones_like(o_r))
    assert made and not [s for s in made if len(s) == 4]
    (_, _, tensors, _, _, _), = handed
    do_p, do_r = tensors[3], tensors[7]
    assert do_p.shape == o_p.shape and not do_p.any() and do_p.dtype == torch.bfloat16 and (do_r == 1).all()
