"""The operators of a paged KV cache under replay trees, as cases that can be timed and compared.

Rollout fills the trees that group attention later trains on. Its keys and values live in pages of a pool; a prompt's
pages are read, in place, by all branches of its tree. Kinds ("op"):

* ``plan``   page_plan: from the lengths and the numbers of new tokens on the GPU, the page tables grown by new pages,
             finished sequences' pages given back, and the slots and positions of the new tokens.
* ``write``  cache_write: keys and values of the new tokens into their slots (bf16, or 8 bits with a scale per head).
* ``attend`` paged_fwd: attention of the new tokens, one or many per sequence, over the pages of the prompt and of the
             branch's own tokens, with the log-sum-exp.

A batch has ``trees`` prompts, ``branches`` branches of each, and ``alone`` sequences without a prompt. ``prompt``,
``own`` and ``alone_len`` are ranges of cached tokens, ``prompt_new``, ``own_new`` and ``alone_new`` of new ones, as
"lo:hi" (spread over their logarithm); ``done`` branches have ended and give their pages back. Head layouts come from
the named workloads of ``paper_2609_33133_amd.inputs`` and this repository's tests; lengths are generic, odd on purpose.
"""
import math

import numpy as np
import torch

own = False

# (query heads, KV heads, head dimension): a full 8-KV-head model, a 7B model's 28 / 4, one rank's share of the first
# under 4-way tensor parallelism, and a d = 64 model
HEADS = ((32, 8, 128), (28, 4, 128), (8, 2, 128), (16, 4, 64))
FP8 = torch.float8_e4m3fn


def _case(name, op, heads, page, fp8=False, trees=0, branches=0, alone=0, prompt="0:0", prompt_new="0:0", own="0:0",
          own_new="0:0", alone_len="0:0", alone_new="0:0", done=0, lengths=1):
    hq, hkv, d = heads
    return {"name": name, "op": op, "hq": hq, "hkv": hkv, "d": d, "page": page, "fp8": fp8, "trees": trees,
            "branches": branches, "alone": alone, "prompt": prompt, "prompt_new": prompt_new, "own": own,
            "own_new": own_new, "alone_len": alone_len, "alone_new": alone_new, "done": done, "lengths": lengths}


def listed():
    h32, h28, h8, h64 = HEADS
    return [
        # the step of a rollout server: 512 branches of 64 prompts, one token each, a few of them ended
        _case("plan_step", "plan", h32, 64, trees=64, branches=8, prompt="200:4000", own="1:3000", own_new="1:1", done=16),
        # a large server admits prompts in chunks while thousands of branches go on
        _case("plan_admit", "plan", h8, 16, trees=256, branches=16, prompt="1:700", prompt_new="1:900", own="1:1500",
              own_new="1:1", done=300),
        # the new token of 256 sequences
        _case("write_step", "write", h32, 64, alone=256, alone_len="100:5000", alone_new="1:1"),
        # the prompts of a rollout batch, cache in 8 bits
        _case("write_prompts_fp8", "write", h28, 32, fp8=True, trees=24, prompt="0:0", prompt_new="500:9000"),
        # one user waits for the next token: latency
        _case("attend_one", "attend", h32, 64, alone=1, alone_len="4096:4096", alone_new="1:1"),
        # eight answers to the headline workload's prompt
        _case("attend_tree", "attend", h32, 64, trees=1, branches=8, prompt="32768:32768", own="1:2047", own_new="1:1"),
        # a decode batch without shared prompts
        _case("attend_batch", "attend", h28, 64, alone=256, alone_len="500:8000", alone_new="1:1"),
        # a full rollout server, cache in 8 bits
        _case("attend_forest_fp8", "attend", h32, 64, fp8=True, trees=64, branches=8, prompt="300:4000", own="20:4000",
              own_new="1:1"),
        # five drafted tokens of each sequence are verified, d = 64, small pages
        _case("attend_draft_d64", "attend", h64, 16, alone=33, alone_len="150:3000", alone_new="5:5"),
        # a long prompt's next chunk and a short prompt whole
        _case("attend_chunk", "attend", h32, 128, trees=2, prompt="1200:21000", prompt_new="2900:4100", lengths=4),
        # one rank under tensor parallelism: a chunk of a prompt in a batch of single tokens
        _case("attend_mixed_tp", "attend", h8, 64, trees=1, alone=48, prompt="6001:6001", prompt_new="1500:1500",
              alone_len="200:7000", alone_new="1:1"),
        # the next turn of all branches, tool results of some hundred tokens, cache in 8 bits
        _case("attend_turn_fp8", "attend", h32, 32, fp8=True, trees=2, branches=8, prompt="5000:9001", own="300:900",
              own_new="150:700"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "write", "attend", "attend", "attend"])
    case = _case("", op, rng.choice(HEADS), rng.choice([16, 32, 64, 64, 128, 256]), fp8=rng.random() < 0.35,
                 lengths=rng.randrange(1 << 30))
    del case["name"]
    span = lambda lo, hi: "%d:%d" % (lo, max(lo, hi))
    if op == "plan":
        case.update(trees=_log(rng, 1, 256), branches=rng.choice([1, 2, 4, 8, 16]), alone=_log(rng, 1, 300),
                    prompt=span(rng.choice([0, 1, 50]), _log(rng, 50, 4000)), own=span(1, _log(rng, 1, 1500)),
                    own_new=span(1, rng.choice([1, 1, 1, 4])), alone_len=span(1, _log(rng, 1, 1500)),
                    alone_new=span(1, _log(rng, 1, 60)))
        case["done"] = rng.randrange(1 + case["trees"] * case["branches"] // 4)
        if rng.random() < 0.5:
            case["prompt_new"] = span(1, _log(rng, 1, 400))
    elif op == "write":
        case.update(alone=_log(rng, 1, 500), alone_len=span(0, _log(rng, 1, 500)),
                    alone_new=span(1, _log(rng, 1, 200)))
    else:
        kind = rng.choice(["alone", "tree", "tree", "chunk", "mixed"])
        if kind in ("alone", "mixed"):
            count, most = _log(rng, 1, 256), _log(rng, 1, 8000)
            case.update(alone=count, alone_len=span(rng.choice([0, 1, 1 + most // 8]), most),
                        alone_new=span(1, rng.choice([1, 1, 1, 2, 9]) if count * most < 600_000 else 1))
        if kind == "tree":
            case.update(trees=_log(rng, 1, 32), branches=rng.choice([1, 2, 4, 8, 16, 17]))
            count = case["trees"] * case["branches"]
            prompt, own_len = _log(rng, 1, min(32768, 1_500_000 // count)), _log(rng, 1, min(4000, 700_000 // count))
            new = _log(rng, 1, min(500, max(1, 60_000_000 // ((prompt + own_len) * count))))
            case.update(prompt=span(1 + prompt // 3, prompt), own=span(1, own_len), own_new=span(1, rng.choice([1, 1, new])))
        if kind in ("chunk", "mixed"):
            trees, most = rng.choice([1, 1, 2, 3]), _log(rng, 1, 16000)
            new = _log(rng, 17, max(20, min(4000, 60_000_000 // (trees * (most + 2000)))))
            case.update(trees=trees, prompt=span(rng.choice([0, most // 3]), most), prompt_new=span(1 + new // 2, new))
    return case


# ---------------------------------------------------------------------------------------------------- the batch


def _lengths(case):
    """Sequences in their order (prompts, branches, lonely ones): parent, cached tokens, new tokens (-1: has ended)."""
    rng = np.random.RandomState(case["lengths"])

    def span(text, count):
        lo, hi = (int(v) for v in text.split(":"))
        return np.floor(np.exp(rng.uniform(math.log(lo + 1), math.log(hi + 2), count)) - 1 + 1e-9).astype(np.int64).clip(lo, hi)

    t, b, a = case["trees"], case["trees"] * case["branches"], case["alone"]
    cached = np.concatenate([span(case["prompt"], t), span(case["own"], b), span(case["alone_len"], a)])
    new = np.concatenate([span(case["prompt_new"], t), span(case["own_new"], b), span(case["alone_new"], a)])
    parent = np.concatenate([np.full(t, -1), np.arange(b) // max(1, case["branches"]), np.full(a, -1)])
    if case["done"]:
        new[t + rng.permutation(b)[:case["done"]]] = -1
    return parent, cached, new


def _tables(case, seed):
    """A pool whose pages lie in random order: tables of the cached tokens, of all tokens, and the ring of free pages."""
    parent, cached, new = _lengths(case)
    page, rng = case["page"], np.random.RandomState(seed % (1 << 31))
    have, want = -(-cached // page), -(-(cached + new.clip(0)) // page)
    pages = int(want.sum()) + 5 + int(want.sum()) // 16
    ids = rng.permutation(pages).astype(np.int32)
    width = int(want.max()) + 2
    col = np.arange(width)[None]
    cached_at, new_at = col < have[:, None], (col >= have[:, None]) & (col < want[:, None])
    table = rng.randint(0, pages, (len(cached), width)).astype(np.int32)  # what earlier sequences left
    table[cached_at] = ids[:have.sum()]
    full = table.copy()
    full[new_at] = ids[have.sum():want.sum()]
    first, spare = int(rng.randint(pages)), pages - int(have.sum())
    ring = rng.randint(0, pages, pages).astype(np.int32)
    ring[(first + np.arange(spare)) % pages] = ids[have.sum():]
    return {"parent": parent, "cached": cached, "new": new, "table": table, "full": full, "pages": pages, "ring": ring,
            "state": np.array([first, spare])}


def _gpu(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(1_000_003 * int(seed) + 31)
    normal = lambda *s: torch.randn(*s, generator=gen, device="cuda", dtype=torch.bfloat16)
    t = _tables(case, int(seed))
    hq, hkv, d, page = case["hq"], case["hkv"], case["d"], case["page"]
    rows = int(t["new"].clip(0).sum())
    x = {"length": _gpu(t["cached"]), "new": _gpu(t["new"]), "parent": _gpu(t["parent"]), "free": _gpu(t["ring"]),
         "state": _gpu(t["state"])}
    if case["op"] == "plan":
        x["table"] = _gpu(t["table"])
        return x, t, rows
    x["table"] = _gpu(t["full"])
    shape = (t["pages"], hkv, page, d)
    for n in ("k_cache", "v_cache"):
        x[n] = normal(*shape)
        if case["fp8"]:  # what lies in the cache already: unit values times 1 / scale, which fills the type's range
            x[n] = (x[n] * 64.0).to(FP8)
    if case["fp8"]:
        x["k_scale"] = 2.0 ** -6 * torch.linspace(0.8, 1.25, hkv, device="cuda")
        x["v_scale"] = 2.0 ** -6 * torch.linspace(1.2, 0.75, hkv, device="cuda")
    if case["op"] == "write":
        x["k"], x["v"] = normal(rows, hkv, d), normal(rows, hkv, d)
    else:
        x["q"] = normal(rows, hq, d)
    return x, t, rows


def prepare(case, seed):
    x, t, rows = _inputs(case, seed)
    s = {"case": case, "x": x, "rows": rows}
    if case["op"] == "plan":
        s["length_out"], s["state_out"] = torch.empty_like(x["length"]), torch.empty_like(x["state"])
    elif case["op"] == "write":
        s["slots"] = _gpu(_slots(case, t), torch.int64)
    else:
        s["few"], s["many"] = _classes(case, t)
    if own:  # the tables of the cache, and the plan that a program makes once for all layers of a step
        from paper_2609_33133_amd import api
        s["pages"] = api.PageTable(x["table"], x["length"], x["parent"], x["free"], x["state"], case["page"])
        if case["op"] != "plan":
            s["plan"] = api.page_plan(s["pages"], x["new"], rows, case["hq"], case["hkv"],
                                      length_out=torch.empty_like(x["length"]), free_state_out=torch.empty_like(x["state"]))
    return s


def run(state):
    return _own(state) if own else _plain(state)


def _own(state):
    from paper_2609_33133_amd import api
    case, x = state["case"], state["x"]
    if case["op"] == "plan":
        pages = state["pages"]
        plan = api.page_plan(pages, x["new"], state["rows"], case["hq"], case["hkv"], length_out=state["length_out"],
                             free_state_out=state["state_out"])
        return {"table": pages.table, "length": state["length_out"], "free": pages.free_pages, "state": state["state_out"],
                "cu": plan.cu_rows, "slots": plan.slots, "positions": plan.positions}
    if case["op"] == "write":
        api.cache_write(x["k"], x["v"], x["k_cache"], x["v_cache"], state["plan"], k_scale=x.get("k_scale"),
                        v_scale=x.get("v_scale"))
        return {"k_cache": x["k_cache"], "v_cache": x["v_cache"]}
    o, lse = api.paged_fwd(x["q"], x["k_cache"], x["v_cache"], state["plan"], k_scale=x.get("k_scale"),
                           v_scale=x.get("v_scale"), want_lse=True)
    return {"o": o, "lse": lse}


# ---------------------------------------------------------------------------------------------------- the plain form


def _slots(case, t):
    """Slots of the new tokens, in order."""
    new, page = t["new"].clip(0), case["page"]
    seq = np.repeat(np.arange(len(new)), new)
    at = np.arange(len(seq)) - np.repeat(np.cumsum(new) - new, new) + t["cached"][seq]
    return t["full"][seq, at // page].astype(np.int64) * page + at % page


def _classes(case, t):
    """The sequences with new tokens, those with a few and those with many apart, each padded to its longest: rows
    [n, r] (one past the end: padding), their positions, the keys' pages and places in them [n, keys], and how many of
    the keys are seen by all rows."""
    new, cached, parent, page = t["new"].clip(0), t["cached"], t["parent"], case["page"]
    total, start = cached + new, np.cumsum(new) - new
    shared = np.where(parent >= 0, total[parent], 0)

    def padded(ids):
        r, n = np.arange(new[ids].max())[None], int((shared + total)[ids].max())
        rows = np.where(r < new[ids, None], start[ids, None] + r, new.sum())
        key = np.arange(n)[None]
        seq = np.where(key < shared[ids, None], parent[ids, None], ids[:, None])
        at = np.where(key < shared[ids, None], key, np.minimum(key - shared[ids, None], total[ids, None] - 1))
        return {"rows": _gpu(rows, torch.int64), "last": _gpu(shared[ids, None] + cached[ids, None] + r),
                "seq": _gpu(seq), "at": _gpu(at)}

    ids = np.arange(len(new))
    few, many = ids[(new > 0) & (new <= 16)], ids[new > 16]
    return padded(few) if len(few) else None, padded(many) if len(many) else None


def _plain(state):
    case, x = state["case"], state["x"]
    return {"plan": _plain_plan, "write": _plain_write, "attend": _plain_attend}[case["op"]](state, case, x)


def _plain_plan(state, case, x):
    page, rows, pages = case["page"], state["rows"], x["free"].numel()
    new, length, table, parent = (x[n].long() for n in ("new", "length", "table", "parent"))
    first, spare = x["state"].long()
    n, gone = new.clamp(min=0), new < 0
    cu = torch.nn.functional.pad(n.cumsum(0), (1, 0))
    have, want = (length + page - 1) // page, (length + n + page - 1) // page
    need = want - have
    taken = need.cumsum(0)
    col = torch.arange(table.shape[1], device="cuda")[None]
    fresh = (col >= have[:, None]) & (col < want[:, None])
    at = (first + (taken - need - have)[:, None] + col) % pages
    table_out = torch.where(fresh, x["free"].long()[at], table)
    back = gone[:, None] & (col < have[:, None])
    rank = back.flatten().cumsum(0).view(back.shape)
    to = torch.where(back, (first + spare + rank - 1) % pages, pages)
    free = torch.nn.functional.pad(x["free"].long(), (0, 1)).scatter(0, to.flatten(), table.flatten())[:pages]
    row = torch.arange(rows, device="cuda")
    seq = torch.searchsorted(cu, row, right=True) - 1
    pos = length[seq] + row - cu[seq]
    slots = table_out[seq, pos // page] * page + pos % page
    total = length + n
    before = torch.where(parent >= 0, total[parent.clamp(min=0)], 0)
    out = {"table": table_out, "length": torch.where(gone, 0, total), "free": free,
           "state": torch.stack([(first + taken[-1]) % pages, spare - taken[-1] + rank.flatten()[-1]]), "cu": cu,
           "slots": slots, "positions": pos + before[seq]}
    return {k: v.to(torch.int32) for k, v in out.items()}


def _plain_write(state, case, x):
    page, slot = case["page"], state["slots"]
    at, off = slot // page, slot % page
    if case["fp8"]:
        k, v = ((x[n].float() / x[n + "_scale"][:, None]).clamp(-448.0, 448.0).to(FP8) for n in "kv")
        x["k_cache"].view(torch.uint8)[at, :, off] = k.view(torch.uint8)
        x["v_cache"].view(torch.uint8)[at, :, off] = v.view(torch.uint8)
    else:
        x["k_cache"][at, :, off] = x["k"]
        x["v_cache"][at, :, off] = x["v"]
    return {"k_cache": x["k_cache"], "v_cache": x["v_cache"]}


def _plain_attend(state, case, x):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    q = torch.cat([x["q"], x["q"].new_zeros(1, hq, d)]).float()
    o, lse = q.new_zeros(q.shape), q.new_zeros(len(q), hq)
    if state["few"]:  # each class writes its own rows (padding: one past the end)
        _plain_class(case, x, state["few"], q, o, lse)
    if state["many"]:
        _plain_class(case, x, state["many"], q, o, lse)
    return {"o": o[:-1].to(torch.bfloat16), "lse": lse[:-1].t().contiguous()}


def _plain_class(case, x, c, q, o, lse):
    hq, hkv, d, page = case["hq"], case["hkv"], case["d"], case["page"]
    n, r = c["rows"].shape
    at = c["at"].long()
    pg, off = x["table"].long()[c["seq"].long(), at // page], at % page
    k, v = (x[m + "_cache"][pg, :, off].float().transpose(1, 2).contiguous() for m in "kv")   # [n, hkv, keys, d]
    if case["fp8"]:
        k.mul_(x["k_scale"][:, None, None])
        v.mul_(x["v_scale"][:, None, None])
    qg = q[c["rows"]].view(n, r, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(n, hkv, -1, d)
    s = torch.matmul(qg, k.transpose(-1, -2)).mul_(1.0 / math.sqrt(d)).view(n, hkv, hq // hkv, r, -1)
    hidden = torch.arange(s.shape[-1], device="cuda") > c["last"][..., None]                  # [n, r, keys]
    s.masked_fill_(hidden[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    s.sub_(top).exp_()
    total = s.sum(-1, keepdim=True)
    y = torch.matmul(s.view(n, hkv, -1, s.shape[-1]), v).view(n, hkv, hq // hkv, r, d) / total
    o[c["rows"].flatten()] = y.permute(0, 3, 1, 2, 4).reshape(n * r, hq, d)
    lse[c["rows"].flatten()] = (top + total.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(n * r, hq)


# ---------------------------------------------------------------------------------------------------- what it costs


def work(case):
    parent, cached, new = _lengths(case)
    n, page = new.clip(0), case["page"]
    total, rows = cached + n, int(n.sum())
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    size = 1 if case["fp8"] else 2
    if case["op"] == "plan":
        have, want = -(-cached // page), -(-total // page)
        moved = int((want - have).sum()) + int(have[new < 0].sum())  # a free page read, a table entry written, or back
        return {"bytes": 4 * (5 * len(new) + 2 * rows + 2 * moved + 4), "flops": 10 * (len(new) + rows)}
    if case["op"] == "write":
        return {"bytes": rows * (4 + 2 * hkv * d * (2 + size)), "flops": 2 * rows * hkv * d}
    used = n > 0
    shared = np.where(parent >= 0, total[parent], 0)
    read = used.copy()
    read[parent[used & (parent >= 0)]] = True
    pairs = int((n * (shared + cached) + n * (n + 1) // 2).sum())
    return {"bytes": 2 * int(total[read].sum()) * hkv * d * size + rows * hq * (4 * d + 4), "flops": 4 * d * hq * pairs}


# ---------------------------------------------------------------------------------------------------- in 64 bits


def exact(case, seed):
    """From the definition, in 64 bits, one sequence and one KV head at a time."""
    if case["op"] == "plan":
        return None  # whole numbers only
    x, t, rows = _inputs(case, seed)
    page, g, hkv, d = case["page"], case["hq"] // case["hkv"], case["hkv"], case["d"]
    new, cached = t["new"].clip(0), t["cached"]
    if case["op"] == "write":
        out = {n: x[n].double() for n in ("k_cache", "v_cache")}
        slot = torch.from_numpy(_slots(case, t)).cuda()
        at, off = torch.div(slot, page, rounding_mode="floor"), torch.remainder(slot, page)
        for n in "kv":
            y = x[n].double()
            if case["fp8"]:
                y = torch.clamp(y / x[n + "_scale"].double().view(1, -1, 1), min=-448.0, max=448.0)
            out[n + "_cache"][at, :, off] = y
        return out
    o = torch.zeros(rows, case["hq"], d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(case["hq"], rows, dtype=torch.float64, device="cuda")

    def tokens(seq, count):
        """Keys and values of a sequence, [hkv, count, d]."""
        ids = x["table"][seq, :-(-count // page)].long()
        found = []
        for n in "kv":
            y = x[n + "_cache"][ids].double().transpose(0, 1).reshape(hkv, -1, d)[:, :count]
            found.append(y * x[n + "_scale"].double().view(-1, 1, 1) if case["fp8"] else y)
        return found

    row = 0
    for i in range(len(new)):
        r = int(new[i])
        if not r:
            continue
        k, v = tokens(i, int(cached[i]) + r)
        before = int(cached[i])
        if t["parent"][i] >= 0:
            p = int(t["parent"][i])
            kp, vp = tokens(p, int(cached[p] + new[p]))
            before += kp.shape[1]
            k, v = torch.cat([kp, k], 1), torch.cat([vp, v], 1)
        step = max(1, int(2e9) // (k.shape[1] * case["hq"] * 8))
        for a in range(0, r, step):
            e = min(r, a + step)
            seen = torch.arange(k.shape[1], device="cuda") <= before + torch.arange(a, e, device="cuda")[:, None]
            q = x["q"][row + a:row + e].double().reshape(e - a, hkv, g, d)
            for h in range(hkv):
                s = torch.matmul(q[:, h].reshape(-1, d), k[h].t().contiguous()).reshape(e - a, g, -1) / math.sqrt(d)
                s = torch.where(seen[:, None], s, -math.inf)
                z = torch.logsumexp(s, -1)
                o[row + a:row + e, h * g:h * g + g] = torch.matmul(torch.exp(s - z[..., None]), v[h])
                lse[h * g:h * g + g, row + a:row + e] = z.t()
        row += r
    return {"o": o, "lse": lse}
