"""The paged KV cache on the GPU: plans, writes and attention against oracle/paged.py, alone and as a rollout runs them."""
import numpy as np
import pytest
import torch

from oracle import paged as P
from paper_2609_33133_amd import _lib, api

from paged_helpers import FP8, Step, gpu, random_tables, to64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# (parent, cached, new): lonely sequences at the borders of blocks and pages
ALONE = [(-1, 0, 1), (-1, 1, 1), (-1, 62, 1), (-1, 63, 1), (-1, 64, 1), (-1, 65, 2), (-1, 0, 0), (-1, 255, 3), (-1, 1000, 1)]
# a prompt that sits, its branches (two runs, cut by a long one and by one that rests), a prompt that grows with its own
TREES = [(-1, 300, 0), (0, 0, 1), (0, 63, 1), (0, 10, 0), (0, 500, 2), (0, 70, 90), (0, 5, 1), (0, 128, 1), (-1, 40, 33),
         (8, 7, 1), (8, 0, 4), (-1, 77, 1), (8, 200, 1)]
# chunks: from nothing, over cached tokens, of a tile and one row more
CHUNKS = [(-1, 0, 130), (-1, 190, 64), (-1, 500, 33), (-1, 31, 200), (-1, 3, 1)]
SETS = {"alone": ALONE, "trees": TREES, "chunks": CHUNKS}
HEADS = [(1, 1, 64), (4, 2, 128), (7, 1, 128), (32, 8, 128), (12, 4, 64), (6, 6, 128)]


def check_plan(step, plan, length, state):
    table, total, ring, st, cu, slots, positions = step.want
    host = lambda t: t.cpu().numpy().astype(np.int64)
    assert int(plan.status) == 0
    plan.check()
    for got, want in ((step.pages.table, table), (length, total), (step.pages.free_pages, ring), (state, st),
                      (plan.cu_rows, cu), (plan.slots, slots), (plan.positions, positions)):
        np.testing.assert_array_equal(host(got), want)


@pytest.mark.parametrize("name", SETS)
@pytest.mark.parametrize("page", [16, 64, 256])
def test_plan(name, page):
    s = Step(SETS[name], (4, 2, 64), page, seed=page, spare_rows=5)
    length, state = torch.empty_like(s.pages.length), torch.empty_like(s.pages.free_state)
    before = s.pages.length.clone(), s.pages.free_state.clone()
    for _ in range(2):  # the same step again gives the same
        check_plan(s, s.plan(length_out=length, free_state_out=state), length, state)
    assert torch.equal(s.pages.length, before[0]) and torch.equal(s.pages.free_state, before[1])
    check_plan(s, s.plan(), s.pages.length, s.pages.free_state)  # in place


@pytest.mark.parametrize("seqs,new", [(3000, 2), (40, 700), (1024, 2), (1025, 1), (5000, 9)])
def test_plan_of_many(seqs, new):
    rng = np.random.RandomState(seqs)
    roots = seqs // 9
    rows = [(-1, rng.randint(0, 400), rng.randint(0, new + 1)) for _ in range(roots)]
    rows += [(int(rng.randint(roots)) if rng.rand() < 0.8 else -1, rng.randint(0, 200),
              -1 if rng.rand() < 0.1 else rng.randint(0, new + 1)) for _ in range(seqs - roots)]
    s = Step(rows, (4, 4, 64), 32, seed=new, spare_rows=11)
    check_plan(s, s.plan(), s.pages.length, s.pages.free_state)


def test_plan_of_ended_sequences_only():
    s = Step([(-1, 100, -1), (-1, 0, -1), (-1, 5, -3), (-1, 64, 0)], (2, 1, 64), 16)
    plan = s.plan()
    check_plan(s, plan, s.pages.length, s.pages.free_state)
    o, _ = s.attend(plan)
    assert o.shape == (0, 2, 64)


@pytest.mark.parametrize("change,bits,text", [
    (lambda s: s.pages.free_state.copy_(gpu([0, 1])), _lib.PAGES_SHORT, "free pages"),
    (lambda s: s.new.__setitem__(0, 10 ** 6), _lib.PAGES_LONG | _lib.PAGES_ROWS, "outgrows"),
    (lambda s: s.new.__setitem__(0, s.rows), _lib.PAGES_ROWS, "rows"),
    (lambda s: s.pages.length.__setitem__(3, -1), _lib.PAGES_LENGTH, "length"),
    (lambda s: s.pages.parent.__setitem__(1, 1), _lib.PAGES_PARENT, "parent"),
    (lambda s: s.pages.parent.__setitem__(1, 99), _lib.PAGES_PARENT, "parent"),
    (lambda s: s.pages.parent.__setitem__(1, 4), _lib.PAGES_PARENT, "parent"),
    (lambda s: s.new.__setitem__(0, -1), _lib.PAGES_PARENT, "parent"),
])
def test_steps_that_do_not_fit_change_nothing(change, bits, text):
    s = Step(TREES, (4, 2, 128), 32, seed=3)
    change(s)
    keep = [t.clone() for t in (s.pages.table, s.pages.length, s.pages.free_pages, s.pages.free_state)]
    plan = s.plan()
    assert int(plan.status) & bits == bits
    with pytest.raises(RuntimeError, match=text):
        plan.check()
    for a, b in zip(keep, (s.pages.table, s.pages.length, s.pages.free_pages, s.pages.free_state)):
        assert torch.equal(a, b)
    assert (plan.slots == -1).all() and (plan.cu_rows == 0).all()
    # the calls that take it do nothing
    cache = [s.k_cache.view(torch.int16).clone(), s.v_cache.view(torch.int16).clone()]
    o, lse = torch.full_like(s.q, 7.0), torch.full((s.hq, s.rows), 7.0, device="cuda")
    kv = torch.zeros(s.rows, s.hkv, s.d, dtype=torch.bfloat16, device="cuda")
    api.cache_write(kv, kv, s.k_cache, s.v_cache, plan)
    s.attend(plan, o=o, lse=lse)
    assert (o == 7).all() and (lse == 7).all()
    assert torch.equal(cache[0], s.k_cache.view(torch.int16)) and torch.equal(cache[1], s.v_cache.view(torch.int16))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("heads,page", list(zip(HEADS, [16, 32, 64, 128, 256, 16])))
def test_write(heads, page, fp8):
    s = Step(TREES + [(-1, 0, 70)], heads, page, seed=5, fp8=fp8, spare_rows=3, joint=page == 32)
    plan = s.plan()
    gen = torch.Generator().manual_seed(9)
    k, v = ((30 * torch.randn(s.rows, s.hkv, s.d, generator=gen)).to(torch.bfloat16) for _ in range(2))
    odd = [float("nan"), float("inf"), -float("inf"), 0.0, -0.0, 3e38, -3e38, 1e-30, 448 * 0.02, 464 * 0.02]
    k.view(-1)[:len(odd)] = torch.tensor(odd)
    k, v = k.cuda(), v.cuda()
    want = {n: getattr(s, n + "_cache").clone() for n in "kv"}
    slot = torch.from_numpy(s.want[5][:s.live]).cuda()
    at, off = torch.div(slot, page, rounding_mode="floor"), slot % page
    for n, x in (("k", k), ("v", v)):
        y = x[:s.live]
        if fp8:
            y = (y.float() / s.scales[n + "_scale"][:, None]).clamp(-448, 448).to(FP8).view(torch.uint8)
            want[n].view(torch.uint8)[at, :, off] = y
        else:
            want[n][at, :, off] = y
    api.cache_write(k, v, s.k_cache, s.v_cache, plan, **s.scales)
    for n in "kv":  # bit for bit, but that any NaN is a NaN
        got = getattr(s, n + "_cache")
        a, b = (t.float() for t in (got, want[n]))
        same = (a == b) & (torch.signbit(a) == torch.signbit(b))
        assert (same | (a.isnan() & b.isnan())).all()


@pytest.mark.parametrize("scales", [(0.02, 1 / 3), (1.0, 0.0078125), (7e-5, 123.456), (3e-30, 4e25), (1e-38, 1e30)])
def test_every_bf16_value_in_8_bits(scales):
    """All 65536 bf16 patterns divided by a scale, bit for bit; NaN as NaN."""
    rows = 65536 // 64
    pages = api.PageTable.empty(1, rows // 16, rows // 16, 16)
    plan = api.page_plan(pages, gpu([rows]), rows, 2, 2)
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).view(rows, 1, 64).expand(rows, 2, 64).contiguous().cuda()
    kc, vc = (torch.zeros(rows // 16, 2, 16, 64, device="cuda").to(FP8) for _ in range(2))
    s = torch.tensor(scales, dtype=torch.float32, device="cuda")
    api.cache_write(x, x, kc, vc, plan, k_scale=s, v_scale=s)
    want = (x.float() / s[:, None]).clamp(-448, 448).to(FP8).float().view(rows // 16, 16, 2, 64).transpose(1, 2)
    for got in (kc.float(), vc.float()):
        same = (got == want) & (torch.signbit(got) == torch.signbit(want))
        assert (same | (got.isnan() & want.isnan())).all()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("name", SETS)
def test_attention(name, page, fp8):
    heads = HEADS[(page // 16 + 2 * fp8 + len(name)) % len(HEADS)]
    s = Step(SETS[name], heads, page, seed=page + fp8, fp8=fp8, spare_rows=2)
    o, lse = s.attend(s.plan())
    s.check_attention(o, lse)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("heads", HEADS + [(130, 1, 64), (300, 2, 128), (28, 4, 128)])
def test_attention_heads(heads, fp8):
    s = Step(TREES[:8], heads, 64, seed=heads[0], fp8=fp8, joint=True)
    o, lse = s.attend(s.plan(), scale=0.07)
    s.check_attention(o, lse, 0.07)


@pytest.mark.parametrize("seqs", [
    [(-1, 20000, 1)],                                                      # one long sequence: many parts
    [(-1, 9000, 0)] + [(0, 40 * i, 1) for i in range(17)],                 # a run of more than one tile
    [(-1, 5000, 0), (0, 3000, 1), (0, 0, 1)],
    [(-1, 4000, 300)],                                                     # a chunk with parts
    [(-1, 3000, 0), (0, 50, 120), (0, 2000, 45)],                          # long rows behind a parent, with parts
    [(-1, 0, 0), (0, 10, 1), (0, 20, 1), (-1, 33, 1)],                     # a parent without tokens
    [(-1, i * 37 % 900, 1) for i in range(300)],
    [(-1, 3000, 70), (-1, 17000, 1), (-1, 900, 40)],                       # rows of few parts beside one of many
    [(-1, 12000, 0), (0, 9000, 1), (0, 100, 1), (-1, 30, 1)],              # many parts in both units
])
def test_attention_in_parts(seqs):
    for heads, page in (((8, 2, 128), 64), ((4, 4, 64), 16)):
        s = Step(seqs, heads, page, seed=len(seqs))
        o, lse = s.attend(s.plan())
        s.check_attention(o, lse)


def test_sharp_scores():
    s = Step(TREES, (8, 2, 128), 32, seed=8, amp=6.0)
    o, lse = s.attend(s.plan())
    s.check_attention(o, lse)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("where", ["q", "k", "v"])
def test_nan_and_infinity_stay_with_their_sequence(where, value):
    """In one row of Q: that row alone. In a token of K or V: the rows of its own sequence (a parent's: its branches)."""
    s = Step(TREES, (8, 2, 128), 64, seed=14)
    plan = s.plan()
    want = s.attend(plan)
    cu = s.want[4]
    if where == "q":
        touched = [int(cu[5]) + 3]
        s.q[touched[0], 2] = value
    else:
        seq = 5
        at = 20  # a cached token
        slot = int(s.want[0][seq, at // 64]) * 64 + at % 64
        (s.k_cache if where == "k" else s.v_cache)[slot // 64, 1, slot % 64, 7] = value
        touched = range(cu[seq], cu[seq + 1])
    got = s.attend(plan)
    keep = torch.ones(s.rows, dtype=torch.bool)
    keep[list(touched)] = False
    keep = keep.cuda()
    assert torch.equal(got[0][keep], want[0][keep]) and torch.equal(got[1][:, keep], want[1][:, keep])
    heads = [h for h in range(8) if (h != 2 if where == "q" else h < 4)]  # other heads, heads of the other KV head
    assert torch.equal(got[0][:, heads], want[0][:, heads])


@pytest.mark.parametrize("where", ["k", "v"])
@pytest.mark.parametrize("seqs,seq", [(TREES, 5), (CHUNKS, 1)])
def test_nan_in_8_bits_stays_with_its_sequence(where, seqs, seq):
    s = Step(seqs, (8, 2, 128), 64, seed=15, fp8=True)
    plan = s.plan()
    want = s.attend(plan)
    cu, at = s.want[4], 20  # a cached token
    slot = int(s.want[0][seq, at // 64]) * 64 + at % 64
    (s.k_cache if where == "k" else s.v_cache).view(torch.uint8)[slot // 64, 1, slot % 64, 7] = 0xFF
    got = s.attend(plan)
    mine = slice(int(cu[seq]), int(cu[seq + 1]))
    if where == "v":
        assert got[0][mine, 4:, 7].isnan().all()
    for x, y in zip(got, want):  # the other rows, and the other KV head's heads
        rows = 1 if x.dim() == 2 else 0
        heads = 1 - rows
        assert torch.equal(x.narrow(heads, 0, 4), y.narrow(heads, 0, 4))
        for part in (slice(0, mine.start), slice(mine.stop, s.live)):
            assert torch.equal(x[:, part] if rows else x[part], y[:, part] if rows else y[part])


@pytest.mark.parametrize("fp8", [False, True])
def test_two_layers_at_once_share_a_plan(fp8):
    """On two streams, each with a workspace and outputs of its own."""
    a, b = (Step(TREES + CHUNKS, (8, 2, 128), 64, seed=21, fp8=fp8) for _ in range(2))
    b.q, b.k_cache, b.v_cache = b.q.flip(2), b.v_cache, b.k_cache
    plan = a.plan()
    want = [x.attend(plan) for x in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[x.attend(plan, stream=st) for _ in range(4)] for x, st in zip((a, b), streams)]
    torch.cuda.synchronize()
    for tries, w in zip(got, want):
        for o, lse in tries:
            assert torch.equal(o[:a.live], w[0][:a.live]) and torch.equal(lse[:, :a.live], w[1][:, :a.live])


def test_rows_behind_the_last_are_left_and_results_repeat():
    s = Step(TREES, (8, 2, 128), 64, seed=2, spare_rows=40)
    plan = s.plan()
    o, lse = torch.full_like(s.q, 3.0), torch.full((s.hq, s.rows), 3.0, device="cuda")
    s.attend(plan, o=o, lse=lse)
    assert (o[s.live:] == 3).all() and (lse[:, s.live:] == 3).all()
    o2, lse2 = s.attend(plan, ws=torch.full((plan.workspace_size(s.d),), 0xFF, dtype=torch.uint8, device="cuda"))
    assert torch.equal(o[:s.live], o2[:s.live]) and torch.equal(lse[:, :s.live], lse2[:, :s.live])


def test_tables_are_written_not_exchanged():
    pages = api.PageTable.empty(2, 3, 8, 16)
    for name in ("length", "table", "parent", "free_state", "page_size"):
        with pytest.raises(AttributeError, match=name):
            setattr(pages, name, None)
    assert api.page_plan(pages, gpu([1, 0]), 1, 1, 1).positions.tolist() == [0]


def test_no_parents_tensor_and_other_stream():
    s = Step([(-1, 100, 1), (-1, 7, 20)], (4, 1, 64), 16, seed=6, parents=False)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    plan = s.plan(stream=side)
    o, lse = s.attend(plan, stream=side)
    side.synchronize()
    s.check_attention(o, lse)


def test_pages_outside_the_pool_read_as_zeros():
    """Table entries outside the pool: their keys and values count as zeros, and nothing faults."""
    s = Step([(-1, 200, 1), (-1, 130, 40)], (4, 2, 128), 64, seed=4)
    plan = s.plan()
    num = s.pages.num_pages
    for bad in (-1, num, 2 ** 31 - 1, -2 ** 31):
        t = s.pages.table.clone()
        s.pages.table[0, 1] = s.pages.table[1, 0] = bad
        o, lse = s.attend(plan)
        s.pages.table.copy_(t)
        kc, vc, table = s.k_cache.clone(), s.v_cache.clone(), s.want[0].copy()
        for i, k in ((0, 1), (1, 0)):
            s.k_cache[int(t[i, k])] = 0
            s.v_cache[int(t[i, k])] = 0
        s.check_attention(o, lse)
        s.k_cache, s.v_cache = kc, vc


def test_ring_pages_outside_the_pool_are_reported():
    s = Step([(-1, 10, 100)], (4, 2, 64), 16, seed=4)
    s.pages.free_pages.fill_(10 ** 6)
    plan = s.plan()
    assert int(plan.status) == _lib.PAGES_PAGE
    assert (plan.slots[:6] >= 0).all() and (plan.slots[6:] == -1).all()
    kv = torch.ones(s.rows, s.hkv, s.d, dtype=torch.bfloat16, device="cuda")
    api.cache_write(kv, kv, s.k_cache, s.v_cache, plan)
    o, lse = s.attend(plan)
    assert torch.isfinite(o.float()).all()


def test_a_plan_of_other_sizes_does_nothing():
    """The kernels compare the plan's sizes with the call's: through the C ABI a caller may hand over another's."""
    s = Step([(-1, 100, 3)], (4, 2, 128), 64, seed=1)
    plan = s.plan()
    other = api.PagePlan(s.pages, 5, 4, 2)
    other.data.fill_(0)
    other.data[:plan.data.numel()].copy_(plan.data[:other.data.numel()])
    q = torch.zeros(5, 4, 128, dtype=torch.bfloat16, device="cuda")
    o = torch.full_like(q, 7.0)
    before = s.k_cache.view(torch.int16).clone()
    narrow = api.PagePlan(api.PageTable(s.pages.table[:, :1].contiguous(), s.pages.length, s.pages.parent, s.pages.free_pages,
                                        s.pages.free_state, 64), 3, 4, 2)  # a table with fewer entries
    narrow.data[:min(narrow.data.numel(), plan.data.numel())] = plan.data[:narrow.data.numel()]
    api.paged_fwd(q[:3], s.k_cache, s.v_cache, narrow, o=o[:3])
    api.paged_fwd(q, s.k_cache, s.v_cache, other, o=o)
    kv = torch.zeros(5, 2, 128, dtype=torch.bfloat16, device="cuda")
    api.cache_write(kv, kv, s.k_cache, s.v_cache, other)
    assert (o == 7).all() and torch.equal(before, s.k_cache.view(torch.int16))


def test_offsets_past_32_bits():
    """A cache of 5 GiB: pages at its end as pages at its beginning."""
    page, d, num = 64, 128, 5 * 2 ** 30 // (64 * 128 * 2)
    k = torch.zeros(num, 1, page, d, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    gen = torch.Generator(device="cuda").manual_seed(2)
    q = torch.randn(2, 4, d, generator=gen, device="cuda").to(torch.bfloat16)
    kv = torch.randn(2, 70, 1, d, generator=gen, device="cuda").to(torch.bfloat16)
    out = []
    for first in (0, num - 4):
        pages = api.PageTable.empty(2, 4, num, page)
        pages.free_state[0] = first
        new = gpu([69, 1])
        plan = api.page_plan(pages, new, 70, 4, 1)
        plan.check()
        api.cache_write(kv[0], kv[1], k, v, plan)
        plan = api.page_plan(pages, gpu([1, 1]), 2, 4, 1)
        api.cache_write(kv[0, :2].contiguous(), kv[1, :2].contiguous(), k, v, plan)
        o, lse = api.paged_fwd(q, k, v, plan, want_lse=True)
        assert int(plan.slots[0]) // page == first + 1
        out.append((o, lse, k[first:first + 3].clone()))
    assert all(torch.equal(a, b) for a, b in zip(*out))


@pytest.mark.parametrize("fp8", [False, True])
def test_rollout_of_trees_meets_group_attention(fp8):
    """Prompts in chunks, then branches token by token and in turns, all through the cache: the outputs are those of
    group attention over the finished trees (bf16 cache; with 8 bits, over the keys and values that the cache holds)."""
    hq, hkv, d, page = 8, 2, 128, 32
    prompts, branches = [150, 70], [[20, 33, 9], [41, 5]]
    batch = api.GroupBatch(np.cumsum([0] + prompts), np.cumsum([0] + [len(b) for b in branches]),
                           np.cumsum([0] + sum(branches, [])), hq, hkv, d)
    gen = torch.Generator().manual_seed(3)
    mk = lambda t, h: torch.randn(t, h, d, generator=gen).to(torch.bfloat16).cuda()
    x = {s: (mk(t, hq), mk(t, hkv), mk(t, hkv)) for s, t in (("p", batch.tp), ("r", batch.tr))}
    lens = prompts + sum(branches, [])
    parent = [-1, -1] + [i for i, b in enumerate(branches) for _ in b]
    starts = [("p", int(a)) for a in batch.cu_prompt[:-1]] + [("r", int(a)) for a in batch.cu_resp[:-1]]
    pages = api.PageTable.empty(len(lens), 8, 40, page)
    pages.parent.copy_(gpu(parent))
    shape = (40, hkv, page, d)
    kc, vc = (torch.full(shape, float("nan"), device="cuda").to(FP8 if fp8 else torch.bfloat16) for _ in range(2))
    scales = {n: torch.tensor([0.02, 0.03], device="cuda") for n in ("k_scale", "v_scale")} if fp8 else {}
    o = {s: torch.zeros_like(x[s][0]) for s in x}
    lse = {s: torch.zeros(hq, x[s][0].shape[0], device="cuda") for s in x}
    done, rng = [0] * len(lens), np.random.RandomState(0)
    steps = 0
    while done != lens:
        grow = [0] * len(lens)
        for i, n in enumerate(lens):
            if parent[i] < 0:
                grow[i] = min(n - done[i], int(rng.choice([0, 1, 64, 33])))
            elif done[parent[i]] == lens[parent[i]]:
                grow[i] = min(n - done[i], int(rng.choice([0, 1, 1, 1, 12])))
        at = torch.cat([torch.arange(starts[i][1] + done[i], starts[i][1] + done[i] + g) + (0 if starts[i][0] == "p" else batch.tp)
                        for i, g in enumerate(grow)]).cuda()
        rows = [torch.cat([a, b])[at] for a, b in zip(x["p"], x["r"])]
        plan = api.page_plan(pages, gpu(grow), sum(grow), hq, hkv)
        plan.check()
        api.cache_write(rows[1], rows[2], kc, vc, plan, **scales)
        y, z = api.paged_fwd(rows[0], kc, vc, plan, want_lse=True, **scales)
        for s, sel in (("p", at < batch.tp), ("r", at >= batch.tp)):
            i = at[sel] - (0 if s == "p" else batch.tp)
            o[s][i], lse[s][:, i] = y[sel], z[:, sel]
        done = [a + b for a, b in zip(done, grow)]
        steps += 1
    assert steps > 10 and pages.length.tolist() == lens
    if fp8:
        held = lambda t, s: ((t.float() / s[:, None]).clamp(-448, 448).to(FP8).float() * s[:, None])
        x = {s: (q, held(k, scales["k_scale"]), held(v, scales["v_scale"])) for s, (q, k, v) in x.items()}
    ref, rlse, mag, size = [], [], [], []
    seqs = {i: [x[s][j][a:a + n] for j in range(3)] for i, ((s, a), n) in enumerate(zip(starts, lens))}
    args = lambda ids, new: P.attention(np.concatenate([to64(seqs[i][0]) for i in ids]), lambda i: to64(seqs[i][1].float()),
                                        lambda i: to64(seqs[i][2].float()), np.array(parent), np.zeros(len(lens)), np.array(new),
                                        d ** -0.5, hq // hkv)
    for s, ids in (("p", [0, 1]), ("r", range(2, len(lens)))):
        r, rl, mg, sz = args(ids, [n if i in ids else 0 for i, n in enumerate(lens)])
        assert (abs(to64(o[s]) - r) <= 2.0 ** -8 * abs(r) + (2.0 ** -8 + 2.0 ** -13) * mg).all()
        assert (abs(to64(lse[s]) - rl) <= 2.0 ** -17 * sz + 2.0 ** -16 + 2.0 ** -21 * abs(rl)).all()
    if not fp8:
        o_p, lse_p, o_r, lse_r, *_ = api.tree_fwd(batch, *x["p"], *x["r"])
        for a, b in ((o["p"], o_p), (o["r"], o_r)):
            assert (a.float() - b.float()).norm() <= 2.0 ** -7 * b.float().norm()
        for a, b in ((lse["p"], lse_p), (lse["r"], lse_r)):
            assert (a - b).abs().max() <= 1e-4


def test_captured_prefill_replays():
    """A captured step of more rows than one workgroup plans: prompts of changing lengths in a room of 2300 rows."""
    hq, hkv, d, page, rows = 4, 2, 64, 32, 2300
    lens = [[900, 1200, 1], [0, 2300, 0], [5, 7, 1500], [64, 0, 0]]
    gen = torch.Generator().manual_seed(6)
    mk = lambda h: torch.randn(rows, h, d, generator=gen).to(torch.bfloat16).cuda()
    q, k, v = mk(hq), mk(hkv), mk(hkv)
    pages = [api.PageTable.empty(3, 120, 200, page) for _ in range(2)]
    caches = [[torch.zeros(200, hkv, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)] for _ in range(2)]
    new = gpu(lens[0])

    def take(n, plan):
        plan = api.page_plan(pages[n], new, rows, hq, hkv, plan=plan)
        api.cache_write(k, v, *caches[n], plan)
        return plan, *api.paged_fwd(q, *caches[n], plan, want_lse=True)

    warm = api.PageTable.empty(3, 120, 200, page)
    api.paged_fwd(q, *caches[1], api.page_plan(warm, new, rows, hq, hkv))
    plan = api.PagePlan(pages[1], rows, hq, hkv)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _, o, lse = take(1, plan)
    for n in lens:
        new.copy_(gpu(n))
        p, o_want, lse_want = take(0, None)
        p.check()
        g.replay()
        torch.cuda.synchronize()
        live = sum(n)
        assert torch.equal(o[:live], o_want[:live]) and torch.equal(lse[:, :live], lse_want[:, :live])
        assert torch.equal(pages[0].table, pages[1].table) and torch.equal(pages[0].length, pages[1].length)
        assert all(torch.equal(a, b) for a, b in zip(*caches))


def test_captured_decode_replays():
    """A decode step captured once: every replay takes a token, pages and lengths advance on the GPU, a branch ends."""
    heads, page = (8, 2, 128), 16
    seqs = [(-1, 100, 0), (0, 14, 1), (0, 3, 1), (0, 40, 1), (-1, 9, 1)]

    def start():
        s = Step(seqs, heads, page, seed=12)
        big = api.PageTable.empty(len(seqs), 12, 60, page)
        num = s.pages.num_pages
        big.table[:, :s.pages.max_pages] = s.pages.table
        big.length.copy_(s.pages.length)
        big.parent.copy_(s.pages.parent)
        first, spare = s.pages.free_state.tolist()
        used = set(s.pages.table[i, k].item() for i, n in enumerate(s.t["length"]) for k in range(-(-n // page)))
        free = [p for p in range(60) if p not in used]
        big.free_pages[:len(free)] = gpu(free)
        big.free_state.copy_(gpu([0, len(free)]))
        s.pages = big
        pad = lambda t: torch.cat([torch.nan_to_num(t), torch.zeros(60 - num, *t.shape[1:], dtype=t.dtype, device="cuda")])
        s.k_cache, s.v_cache = pad(s.k_cache), pad(s.v_cache)
        return s

    gen = torch.Generator().manual_seed(5)
    data = [[torch.randn(6, h, 128, generator=gen).to(torch.bfloat16).cuda() for h in (8, 2, 2)] for _ in range(25)]

    def take(s, x, plan):
        plan = api.page_plan(s.pages, s.new, 6, 8, 2, plan=plan)
        api.cache_write(x[1], x[2], s.k_cache, s.v_cache, plan)
        return plan, *api.paged_fwd(x[0], s.k_cache, s.v_cache, plan, want_lse=True)

    def changes(s, i):
        if i == 9:
            s.new[2] = -1
        if i == 10:
            s.new[2] = 0

    want, a = [], start()
    for i, x in enumerate(data):
        changes(a, i)
        plan, o, lse = take(a, x, None)
        plan.check()
        n = int(plan.cu_rows[-1])
        want.append((o[:n].clone(), lse[:, :n].clone(), plan.slots.clone()))
    b, x = start(), [t.clone() for t in data[0]]
    warm = start()
    take(warm, x, None)
    plan = api.PagePlan(b.pages, 6, 8, 2)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _, o, lse = take(b, x, plan)
    for i, d in enumerate(data):
        changes(b, i)
        for t, src in zip(x, d):
            t.copy_(src)
        g.replay()
        torch.cuda.synchronize()
        n = int(plan.cu_rows[-1])
        assert int(plan.status) == 0
        assert torch.equal(o[:n], want[i][0]) and torch.equal(lse[:, :n], want[i][1]) and torch.equal(plan.slots, want[i][2]), i
    for n in ("table", "length", "free_pages", "free_state"):
        assert torch.equal(getattr(a.pages, n), getattr(b.pages, n))
