"""Training steps of the linear-attention layer as a program interleaves them with its other work."""
import pytest
import torch

from paper_2609_33133_amd.autograd import group_linear_attention

from linear_helpers import LEAVES, batch, decays, inputs, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def test_a_state_updated_between_forward_and_backward():
    b, dec = batch([(200, [70, 131]), (33, [5])], 4, 2, 128), decays(2)
    x = inputs(b, 71)
    state = torch.randn(2, 2, 128, 128, generator=torch.Generator().manual_seed(5)).cuda()
    want = run(b, dec, x, state=state)
    leaf = [x[n].clone().requires_grad_(True) for n in LEAVES]
    outs = group_linear_attention(*leaf, b, dec, state=state)
    state.zero_()  # the buffer of the next piece
    for n, g in zip(LEAVES, torch.autograd.grad(outs, leaf, (x["do_p"], x["do_r"]))):
        assert torch.equal(g, want["d" + n]), n
