"""Linear attention where a block is several chunks of 64 rows, d = 128 above all: what one chunk hands to the next inside
a block. A block's length is chosen by a rule, so the lengths that these batches get are read back (on the CPU) first."""
import pytest
import torch

from paper_2609_33133_amd import api

from linear_helpers import LEAVES, batch, check, decays, inputs, oracle, run

# name: trees, query heads, KV heads, head dimension, least rows of a block on average
CASES = {
    "two_chunks_group_4": ([(1000, [300, 77])], 64, 16, 128, 110),
    "three_chunks": ([(1000, [300, 77])], 64, 32, 128, 190),
    "five_chunks_one_head_each": ([(900, [333])], 64, 64, 128, 300),
    "two_trees": ([(700, [201]), (650, [300, 129])], 48, 48, 128, 200),
    "d64": ([(2100, [1500, 61])], 64, 32, 64, 200),
}


def up(n):
    return (n + 255) // 256 * 256


def blocks(b):
    """Blocks of a batch, from the workspace that holds a state for each of them and KV head (besides a table of five
    words a segment and a state a tree)."""
    state = b.hkv * b.d * b.d * 4
    n = api.linear_workspace_size(b) - up(20 * (b.num_groups + b.num_branches)) - up(state * b.num_groups)
    assert n % state == 0
    return n // state


@pytest.mark.parametrize("name", list(CASES))
def test_the_blocks_have_several_chunks(name):
    trees, hq, hkv, d, rows = CASES[name]
    b = batch(trees, hq, hkv, d)
    assert (b.tp + b.tr) / blocks(b) >= rows > 64


def gpu(f):
    return pytest.mark.gpu(pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")(f))


@gpu
@pytest.mark.parametrize("state", [False, True], ids=["from_zero", "from_a_state"])
@pytest.mark.parametrize("name", list(CASES))
def test_matches_reference(name, state):
    trees, hq, hkv, d, _ = CASES[name]
    b, dec = batch(trees, hq, hkv, d), decays(hkv, 3.0, 14.0)
    x = inputs(b, 61)
    s0 = None
    if state:
        s0 = torch.randn(len(trees), hkv, d, d, generator=torch.Generator().manual_seed(62)).mul(4).cuda()
    check(run(b, dec, x, state=s0), oracle(b, dec, x, state=s0), name)


@gpu
@pytest.mark.parametrize("decay", [1.0, 0.5, 1e-30], ids=str)
def test_decays_over_several_chunks(decay):
    trees, hq, hkv, d, _ = CASES["three_chunks"]
    b = batch(trees, hq, hkv, d)
    dec = torch.full((hkv,), decay).numpy()
    x = inputs(b, 63)
    check(run(b, dec, x), oracle(b, dec, x), f"decay {decay}")


@gpu
def test_backward_from_the_forwards_workspace():
    trees, hq, hkv, d, _ = CASES["three_chunks"]
    b, dec = batch(trees, hq, hkv, d), decays(hkv)
    x = inputs(b, 64)
    ws = torch.empty(api.linear_workspace_size(b), dtype=torch.uint8, device="cuda")
    api.linear_fwd(b, dec, *(x[n] for n in LEAVES), ws=ws)
    args = (b, dec, x["q_p"], x["k_p"], x["v_p"], x["do_p"], x["q_r"], x["k_r"], x["v_r"], x["do_r"])
    for g, w in zip(api.linear_bwd(*args, fwd_ws=ws), api.linear_bwd(*args)):
        assert torch.equal(g, w)
