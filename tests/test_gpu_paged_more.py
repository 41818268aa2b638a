"""More of the paged KV cache on the GPU."""
import numpy as np
import pytest
import torch

from oracle import paged as P
from paper_2609_33133_amd import _lib, api

from paged_helpers import Step, to64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("seqs", [40, 1025, 2500, 4096])
def test_new_tokens_past_32_bits_are_refused(seqs):
    """Each sequence asks for more tokens than the plan has rows; of 2500 and more their sum passes 2^31."""
    rows = 1 << 20
    pages = api.PageTable.empty(seqs, rows // 256, 30, 256)
    new = torch.full((seqs,), rows if seqs > 2048 else 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    keep = [t.clone() for t in (pages.table, pages.length, pages.free_pages, pages.free_state)]
    plan = api.page_plan(pages, new, rows, 2, 1)
    assert int(plan.status) & (_lib.PAGES_ROWS | _lib.PAGES_SHORT) == _lib.PAGES_ROWS | _lib.PAGES_SHORT
    for a, b in zip(keep, (pages.table, pages.length, pages.free_pages, pages.free_state)):
        assert torch.equal(a, b)
    assert (plan.slots == -1).all() and (plan.cu_rows == 0).all()


NAN, INF = float("nan"), float("inf")
# The most tokens before a new token of whose V a NaN may reach a row: 31 rows of a wavefront and the 63 keys behind the
# last of them.
REACH = 94


def bounds(s):
    """How far o and lse may be off (paged_helpers)."""
    k, v = s.held("k"), s.held("v")
    ref, rlse, mag, size = P.attention(to64(s.q), lambda i: s.tokens(k, i), lambda i: s.tokens(v, i), s.t["parent"],
                                       s.t["length"], s.t["new"], s.d ** -0.5, s.hq // s.hkv)
    return (2.0 ** -8 * abs(ref) + (2.0 ** -8 + 2.0 ** -13) * mag, 2.0 ** -17 * size + 2.0 ** -16 + 2.0 ** -21 * abs(rlse))


@pytest.mark.parametrize("fp8,bad", [(False, NAN), (False, INF), (True, NAN)])
@pytest.mark.parametrize("heads", [(2, 2, 128), (2, 2, 64), (8, 2, 128), (14, 2, 64)])
@pytest.mark.parametrize("cached", [0, 1, 6, 70])
def test_a_bad_new_token(heads, cached, fp8, bad):
    """A new token of a chunk alone, and of one behind a parent. In K: the rows that see it. In V: these, and rows of the
    same sequence at most REACH tokens before it, in the bad value's channel. Not: other KV heads, other sequences, earlier
    rows than that, whose results are the same bit for bit. But of an infinity in K, whose score a row sees: the rows
    computed together with it move the reference of their exponents with it. By the formula the reference cancels, so
    their results before and after are both within `bound` of the exact one, and within twice that of one another."""
    new, hq = 300, heads[0]
    s = Step([(-1, cached, new), (-1, 150, 0), (1, cached, new), (1, 9, 1)], heads, 64, seed=cached, fp8=fp8)
    plan = s.plan()
    want = s.attend(plan)
    cu, mine = s.want[4], slice(hq // 2, hq)  # the query heads of KV head 1
    bound, lbound = (torch.from_numpy(b).cuda() for b in bounds(s))
    for seq in (0, 2):
        for at in sorted({cached, 63, 127, 128, 250, cached + new - 1} & set(range(cached, cached + new))):
            slot = int(s.want[0][seq, at // 64]) * 64 + at % 64
            for where in "kv":
                c = getattr(s, where + "_cache")
                place = (slot // 64, 1, slot % 64, 7)
                keep = c.view(torch.uint8 if fp8 else torch.int16)[place].clone()
                if fp8:
                    c.view(torch.uint8)[place] = 0xFF
                else:
                    c[place] = bad
                o, lse = s.attend(plan)
                c.view(torch.uint8 if fp8 else torch.int16)[place] = keep
                first = int(cu[seq]) + at - cached  # the first row that sees it
                from_ = first if where == "k" else max(int(cu[seq]), first - REACH)
                same = torch.ones(o.shape, dtype=torch.bool, device="cuda")
                same[from_:int(cu[seq + 1]), mine, 7 if where == "v" else slice(None)] = False
                moved = where == "k" and bad == INF
                err = (o.double() - want[0].double()).abs()[same]
                assert (err <= (2 * bound[same] if moved else 0)).all(), (seq, at, where)
                rows = torch.ones(lse.shape, dtype=torch.bool, device="cuda")
                if where == "k":
                    rows[mine, from_:int(cu[seq + 1])] = False
                err = (lse.double() - want[1].double()).abs()[rows]
                assert (err <= (2 * lbound[rows] if moved else 0)).all(), (seq, at, where)
                if where == "v":
                    assert not torch.isfinite(o[first:int(cu[seq + 1]), mine, 7]).any()
    assert all(torch.equal(a, b) for a, b in zip(s.attend(plan), want))


def forest(seqs, seed):
    """Trees one after the other, most of whose branches take a token: runs that cross the 64 lanes of a wavefront, its
    steps and the wavefronts; some branches rest, end or take more tokens."""
    rng, rows, root, left = np.random.RandomState(seed), [], -1, 0
    for i in range(seqs):
        if left == 0:
            root, left = i, rng.randint(0, 150)
            rows.append((-1, rng.randint(0, 200), 0 if rng.rand() < 0.8 else rng.randint(1, 30)))
        else:
            left -= 1
            kind = rng.rand()
            new = 1 if kind < 0.8 else rng.randint(2, 6) if kind < 0.9 else 0 if kind < 0.94 else -1 if kind < 0.97 else rng.randint(20, 80)
            rows.append((root, rng.randint(0, 90), new))
    return rows


def check_items(s, plan):
    """The plan's items lie inside its room and meet, for every (row, head) pair, each block of 64 keys that it sees once."""
    w, n, r, g = plan.data.cpu().numpy(), s.pages.num_seqs, s.rows, s.hq // s.hkv
    up = lambda x: -(-x // 4) * 4
    slots = 32 + up(n + 1) + up(18 * n + 1)
    np.testing.assert_array_equal(w[slots:slots + r], s.want[5])  # (the layout that is read here)
    at, items = slots + 2 * up(r) + up(12 * r), int(w[9])
    assert at + 16 * items <= len(w)
    cu, new = s.want[4], np.maximum(s.t["new"], 0)
    total, parent = s.t["length"] + new, s.t["parent"]
    blocks = lambda t: -(-t // 64)
    met_a, met_b = (np.zeros((s.live, g), np.int64) for _ in range(2))
    used = []
    for row0, rows, pair0, a_seq, a_len, b_seq, b_len, b_pos, blk0, blk1, slot in w[at:at + 16 * items].reshape(-1, 16)[:, :11]:
        assert 0 <= row0 and rows > 0 and row0 + rows <= s.live and 0 <= pair0 < rows * g and pair0 % 128 == 0
        assert 0 <= blk0 <= blk1 <= blocks(a_len) + blocks(b_len)
        assert a_len == (total[a_seq] if a_seq >= 0 else 0) and b_len == (total[b_seq] if b_seq >= 0 else 0)
        pairs = np.arange(pair0, min(pair0 + 128, rows * g))
        row, head = row0 + pairs // g, pairs % g
        seq = np.searchsorted(cu, row, side="right") - 1
        n_a = blocks(a_len)
        if a_seq >= 0:
            assert (parent[seq] == a_seq).all()
            met_a[row, head] += max(0, min(blk1, n_a) - blk0)
        if b_seq >= 0:
            assert (seq == b_seq).all() and b_pos == s.t["length"][b_seq]
            seen = (b_pos + pairs // g) // 64 + 1  # blocks that the pair sees
            met_b[row, head] += np.maximum(0, np.minimum(blk1 - n_a, seen) - max(blk0 - n_a, 0))
        if slot >= 0:
            used += range(slot, slot + -(-len(pairs) // 32))
    seq = np.searchsorted(cu, np.arange(s.live), side="right") - 1
    own = (s.t["length"][seq] + np.arange(s.live) - cu[seq]) // 64 + 1
    above = np.where(parent[seq] >= 0, blocks(total[parent[seq]]), 0)
    assert (met_a == above[:, None]).all() and (met_b == own[:, None]).all()
    assert len(set(used)) == len(used) and (max(used, default=0) + 1) * s.hkv * 32 * (s.d + 1) * 4 <= plan.workspace_size(s.d)


@pytest.mark.parametrize("seqs,heads,page,spare,fp8", [
    (1000, (4, 2, 64), 16, 7, False),     # one launch
    (1100, (8, 2, 128), 64, 7, False),    # two, of more than 1024 sequences
    (3000, (4, 4, 64), 32, 0, True),
    (3000, (7, 1, 128), 16, 50, False),
    (200, (8, 2, 128), 32, 2100, True),   # two, of more than 2048 rows
    (900, (6, 1, 64), 64, 2100, False),
])
def test_attention_of_many_sequences(seqs, heads, page, spare, fp8):
    s = Step(forest(seqs, seqs + page), heads, page, seed=seqs, fp8=fp8, spare_rows=spare)
    plan = s.plan()
    plan.check()
    check_items(s, plan)
    o, lse = s.attend(plan)
    s.check_attention(o, lse)
    o2, lse2 = s.attend(plan)
    assert torch.equal(o[:s.live], o2[:s.live]) and torch.equal(lse[:, :s.live], lse2[:, :s.live])
