"""More of the paged KV cache on the GPU."""
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
