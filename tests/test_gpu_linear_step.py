"""One token of linear attention (linear_step) on the GPU against the recurrence in fp64.

Bounds per element: states are fp32 (one multiply-add each, 2^-22 of the magnitudes); outputs are fp32 sums over the
head dimension (2^-17 of the magnitudes, d = 128 terms), rounded once to bf16 (2^-8)."""
import numpy as np
import pytest
import torch

from oracle import linear as L
from paper_2609_33133_amd import api

from linear_helpers import decays, to64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def make(rows, hq, hkv, d, slots, seed):
    gen = torch.Generator().manual_seed(seed)
    bf = lambda *s: torch.randn(*s, generator=gen).to(torch.bfloat16).cuda()
    return bf(rows, hq, d), bf(rows, hkv, d), bf(rows, hkv, d), (3 * torch.randn(slots, hkv, d, d, generator=gen)).cuda()


def check(o, new, q, k, v, dec, scale, start):
    want, state, mag = L.recurrence(to64(q), to64(k), to64(v), dec.astype(np.float64), scale, start)
    terms = abs(start) + abs(to64(k))[..., :, None] * abs(to64(v))[..., None, :]
    assert (abs(to64(new) - state) <= 2.0 ** -22 * terms).all()
    assert (abs(to64(o) - want) <= 2.0 ** -8 * abs(want) + 2.0 ** -17 * mag).all()


@pytest.mark.parametrize("rows,hq,hkv,d", [(1, 1, 1, 64), (1, 32, 8, 128), (3, 7, 1, 128), (5, 12, 4, 64), (130, 4, 2, 128),
                                           (9, 20, 2, 64)])
def test_matches_the_recurrence(rows, hq, hkv, d):
    q, k, v, s = make(rows, hq, hkv, d, rows, rows)
    dec = decays(hkv, 1.0, 12.0)
    o, new = api.linear_step(q, k, v, dec, s)
    check(o, new, q, k, v, dec, d ** -0.5, to64(s))


def test_forks_repeats_and_empty_slots():
    q, k, v, s = make(7, 4, 2, 128, 3, 1)
    dec = decays(2)
    src = torch.tensor([2, 0, 0, -1, 3, 2, -2 ** 31], dtype=torch.int32, device="cuda")
    keep = s.clone()
    o, new = api.linear_step(q, k, v, dec, s, src=src, scale=0.3)
    assert torch.equal(s, keep)
    start = np.stack([to64(s)[i] if 0 <= i < 3 else np.zeros_like(to64(s)[0]) for i in src.tolist()])
    check(o, new, q, k, v, dec, 0.3, start)


def test_in_place_and_rows_behind_the_last_one():
    q, k, v, s = make(4, 4, 2, 64, 6, 2)
    dec = decays(2)
    want, new = api.linear_step(q, k, v, dec, s)
    buf = s.clone()
    o, out = api.linear_step(q, k, v, dec, buf, state_out=buf[:4])
    assert torch.equal(o, want) and torch.equal(buf[:4], new) and torch.equal(buf[4:], s[4:])


def test_no_rows():
    q, k, v, s = make(0, 4, 2, 64, 2, 3)
    o, new = api.linear_step(q, k, v, decays(2), s, src=torch.zeros(0, dtype=torch.int32, device="cuda"))
    assert o.shape == (0, 4, 64) and new.shape == (0, 2, 64, 64)


def test_captured_steps_replay():
    q, k, v, s = make(5, 4, 2, 128, 5, 4)
    dec = decays(2)
    state, want = s.clone(), s.clone()
    g = torch.cuda.CUDAGraph()
    api.linear_step(q, k, v, dec, state.clone())
    with torch.cuda.graph(g):
        o, _ = api.linear_step(q, k, v, dec, state, state_out=state)
    for i in range(4):
        q.copy_(q.roll(1, 0))
        g.replay()
        torch.cuda.synchronize()
        o2, want = api.linear_step(q, k, v, dec, want)
        assert torch.equal(o, o2) and torch.equal(state, want), i


def test_offsets_past_32_bits():
    """Rows behind 4 GiB of states, as on their own."""
    rows, tail = 2 ** 32 // (128 * 128 * 4) + 40, 30
    gen = torch.Generator(device="cuda").manual_seed(5)
    bf = lambda h: torch.empty(rows, h, 128, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    q, k, v = bf(2), bf(1), bf(1)
    s = torch.empty(rows, 1, 128, 128, device="cuda").normal_(generator=gen)
    dec = decays(1)
    src = torch.arange(rows - 1, -1, -1, dtype=torch.int32, device="cuda")
    last = [t[-tail:].contiguous() for t in (q, k, v)]
    o, new = api.linear_step(q, k, v, dec, s, src=src)
    want = api.linear_step(*last, dec, s[:tail].flip(0).contiguous())
    assert torch.equal(o[-tail:], want[0]) and torch.equal(new[-tail:], want[1])
    want = api.linear_step(*last, dec, s[-tail:].contiguous())
    o, new = api.linear_step(q, k, v, dec, s, state_out=s)
    assert torch.equal(o[-tail:], want[0]) and torch.equal(s[-tail:], want[1])
