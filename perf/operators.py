"""The operators of a linear-attention layer over replay trees, as cases that can be timed and compared.

Kinds ("op"):

* ``prefill``  group_linear_attention without gradients, with the states it ends in: what a rollout or a scoring pass
               runs over the prompts and the branches so far ("state": it begins from the state of an earlier piece).
* ``train``    the differentiable op and its backward: outputs and the gradients of all six tensors.
* ``step``     linear_step: one token of every running sequence, on states kept between steps. "fork": the first step
               after a prompt, every branch of a tree starting from the state of its prompt.
* ``norm``     head_norm without gradients (rollout, scoring): a norm over each head, and an activation or a gate.
* ``norm_train``  head_norm and its backward: output and the gradients of all that it reads.

Lengths are text, "P:R,R,R;P:R,R": one tree per ";", its prompt's length and its branches'. They come from the named
workloads of ``paper_2609_33133_amd.inputs`` or are generic chat-like ones, odd on purpose; so do the head layouts.
Decays are spread over the heads as 1 - 2^-5 .. 1 - 2^-12: windows of 32 to 4096 tokens.
"""
import math

import numpy as np
import torch

own = False

LEAVES = ("q_p", "k_p", "v_p", "q_r", "k_r", "v_r")
# (query heads, KV heads, head dimension): a full 8-KV-head model, a 7B model's 28 / 4, one rank's share of the first
# under 4-way tensor parallelism, a d = 64 model, and a small d = 64 layout without grouped heads
HEADS = ((32, 8, 128), (28, 4, 128), (8, 2, 128), (16, 4, 64), (4, 4, 64))
CHUNK = 128  # rows of a block of the plain form


def _tree(name, op, lengths, heads, **more):
    hq, hkv, d = heads
    return {"name": name, "op": op, "lengths": lengths, "hq": hq, "hkv": hkv, "d": d, **more}


def _step(name, rows, heads, fork):
    hq, hkv, d = heads
    return {"name": name, "op": "step", "rows": rows, "hq": hq, "hkv": hkv, "d": d, "fork": fork}


def _norm(name, op, rows, heads, width, act, gate, affine):
    return {"name": name, "op": op, "rows": rows, "heads": heads, "d": width, "act": act, "gate": gate, "affine": affine}


def listed():
    h32, h28, h8, h64, h4 = HEADS
    return [
        # a debugging run, the last layer of a toy model: launches and host time count
        _tree("train_tiny", "train", "256:128,128", h4),
        # a rollout server takes in a few chat prompts with the answers so far, on one rank under tensor parallelism
        _tree("prefill_chat_tp", "prefill", "905:1,731,288;384:290,17;1337:702,530,911,404", h8, state=True),
        # long contexts with short candidate continuations, going on from an earlier piece
        _tree("prefill_long", "prefill", "32768:64,64,64,64;8191:5,16,27,38,49", h32, state=False),
        # one rank's microbatch of a group-relative RL step on chat data
        _tree("train_chat", "train", "417:311,198,977,64,523,402;1130:640,87,333,1204;233:58,120,77,96,41,205,150,88;"
              "1811:455,702,391,128,260", h28),
        # the headline workload: long prompt, eight answers
        _tree("train_prompt_heavy", "train", "32768:" + ",".join(["2048"] * 8), h32),
        # long reasoning traces from a short prompt (the largest case)
        _tree("train_response_heavy", "train", "2048:" + ",".join(["16384"] * 16), h32),
        # the first token of eight branches of one prompt: latency
        _step("step_fork8", 8, h32, True),
        # a full decode batch
        _step("step_512", 512, h32, False),
        # the norm of one decode step
        _norm("norm_decode", "norm", 8, 32, 128, "silu", True, False),
        # scoring with the norm's own activation, an odd row count and a wide head
        _norm("norm_score", "norm", 12289, 16, 256, "silu", False, True),
        # the norm of the chat microbatch
        _norm("norm_train_chat", "norm_train", 8513, 28, 128, "silu", True, True),
        # the norm of the prompt-heavy step
        _norm("norm_train_large", "norm_train", 49152, 32, 128, "silu", True, True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["prefill", "train", "train", "step", "norm", "norm_train"])
    heads = rng.choice(HEADS)
    if op == "step":
        case = _step("", _log(rng, 1, 700), heads, rng.random() < 0.3)
    elif op in ("norm", "norm_train"):
        rows = _log(rng, 1, 49152)
        case = _norm("", op, rows, rng.choice([1, 3, 8, 16, 28, 32]), rng.choice([32, 64, 64, 80, 128, 128, 128, 256]),
                     rng.choice(["silu", "silu", "none"]), rng.random() < 0.6, rng.random() < 0.5)
    else:
        cap = _log(rng, 200, 120_000)
        trees, tokens = [], 0
        for _ in range(rng.choice([1, 1, 2, 3, 5, 8])):
            p = _log(rng, 1, min(32768, cap))
            mid = _log(rng, 2, min(8192, cap))
            rs = [max(1, _log(rng, max(1, mid / 2), mid * 2)) for _ in range(rng.choice([1, 2, 4, 8, 16]))]
            if trees and tokens + p + sum(rs) > cap:
                break
            tokens += p + sum(rs)
            trees.append("%d:%s" % (p, ",".join(map(str, rs))))
        case = _tree("", op, ";".join(trees), heads)
        if op == "prefill":
            case["state"] = rng.random() < 0.5
    del case["name"]
    return case


def _lengths(text):
    ps, rs = [], []
    for tree in text.split(";"):
        p, r = tree.split(":")
        ps.append(int(p))
        rs.append([int(x) for x in r.split(",")])
    return ps, rs


def _decay(case):
    h = case["hkv"]
    return (1.0 - np.exp2(-np.linspace(5.0, 12.0, h))).astype(np.float32)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(1_000_003 * int(seed) + 29)

    def normal(*shape, dtype=torch.bfloat16):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)

    d, x = case["d"], {}
    if case["op"] in ("norm", "norm_train"):
        rows, h = case["rows"], case["heads"]
        # what linear attention leaves: heads of different windows differ in size, rows have a common part
        x["x"] = (normal(rows, h, d, dtype=torch.float32) * torch.logspace(-1, 1, h, device="cuda")[:, None] +
                  0.3 * normal(rows, h, 1, dtype=torch.float32)).to(torch.bfloat16)
        if case["gate"]:
            x["gate"] = normal(rows, h, d)
        if case["affine"]:
            x["weight"] = 1.0 + 0.2 * normal(h, d, dtype=torch.float32)
            x["bias"] = 0.2 * normal(h, d, dtype=torch.float32)
        if case["op"] == "norm_train":
            x["dy"] = normal(rows, h, d)
        return x
    hq, hkv = case["hq"], case["hkv"]
    if case["op"] == "step":
        n = case["rows"]
        x["q"], x["k"], x["v"] = normal(n, hq, d), normal(n, hkv, d), normal(n, hkv, d)
        slots = max(1, n // 8) if case["fork"] else n
        x["state"] = 4.0 * normal(slots, hkv, d, d, dtype=torch.float32)
        x["state_out"] = torch.empty(n, hkv, d, d, device="cuda")
        if case["fork"]:
            x["src"] = torch.arange(n, device="cuda", dtype=torch.int32) * slots // n
        return x
    ps, rs = _lengths(case["lengths"])
    for side, t in (("p", sum(ps)), ("r", sum(map(sum, rs)))):
        x["q_" + side], x["k_" + side], x["v_" + side] = normal(t, hq, d), normal(t, hkv, d), normal(t, hkv, d)
        if case["op"] == "train":
            x["do_" + side] = normal(t, hq, d)
    if case.get("state"):
        x["state"] = 4.0 * normal(len(ps), hkv, d, d, dtype=torch.float32)
    return x


def prepare(case, seed):
    s = {"op": case["op"], "case": case, "x": _inputs(case, seed)}
    x = s["x"]
    if "hkv" in case:
        s["decay"] = _decay(case)
    if "lengths" in case:
        s["plan"] = _plan(case)
        if own:  # the offsets object that a program makes once for a batch and hands to every layer
            from paper_2609_33133_amd.api import GroupBatch
            ps, rs = _lengths(case["lengths"])
            cu = [np.concatenate([[0], np.cumsum(v)]) for v in (ps, [len(r) for r in rs], [n for r in rs for n in r])]
            s["batch"] = GroupBatch(*cu, case["hq"], case["hkv"], case["d"])
    if case["op"] == "train":
        for n in LEAVES:
            x[n].requires_grad_(True)
    if case["op"] == "norm_train":
        for n in ("x", "gate", "weight", "bias"):
            if n in x:
                x[n].requires_grad_(True)
    return s


def run(state):
    return _own(state) if own else _plain(state)


def _own(state):
    from paper_2609_33133_amd import api
    from paper_2609_33133_amd.autograd import group_linear_attention, head_norm
    op, x, case = state["op"], state["x"], state["case"]
    if op == "step":
        o, s = api.linear_step(x["q"], x["k"], x["v"], state["decay"], x["state"], src=x.get("src"),
                               state_out=x["state_out"])
        return {"o": o, "state": s}
    if op in ("norm", "norm_train"):
        y = head_norm(x["x"], x.get("weight"), x.get("bias"), gate=x.get("gate"), activation=case["act"])
        if op == "norm":
            return {"y": y}
        names = [n for n in ("x", "gate", "weight", "bias") if n in x]
        grads = torch.autograd.grad(y, [x[n] for n in names], x["dy"])
        return {"y": y.detach(), **{"d" + n: g for n, g in zip(names, grads)}}
    leaves = [x[n] for n in LEAVES]
    if op == "prefill":
        o_p, o_r, s_p, s_r = group_linear_attention(*leaves, state["batch"], state["decay"], state=x.get("state"),
                                                    return_state=True)
        return {"o_p": o_p, "o_r": o_r, "state_p": s_p, "state_r": s_r}
    o_p, o_r = group_linear_attention(*leaves, state["batch"], state["decay"])
    grads = torch.autograd.grad((o_p, o_r), leaves, (x["do_p"], x["do_r"]))
    return {"o_p": o_p.detach(), "o_r": o_r.detach(), **{"d" + n: g for n, g in zip(LEAVES, grads)}}


# ---------------------------------------------------------------------------------------------------- the plain form
# Linear attention in blocks of CHUNK rows: inside a block by its matrix of decayed products, between blocks by one
# matrix product of the blocks' own states with the decays between blocks (zero where one is no ancestor of the other).


def _plan(case):
    """The blocks of a batch: their rows (of prompts and responses laid end to end; one past the end is padding), depth,
    length, tree, the last block of each prompt and branch, and which block is an ancestor of which."""
    ps, rs = _lengths(case["lengths"])
    tp, total = sum(ps), sum(ps) + sum(map(sum, rs))
    r_at = np.concatenate([[0], np.cumsum([sum(r) for r in rs])])
    p_at = np.concatenate([[0], np.cumsum(ps)])
    segs = [(p_at[g], p, 0, g, -1) for g, p in enumerate(ps)]
    for g, r in enumerate(rs):
        at = np.concatenate([[0], np.cumsum(r)])
        segs += [(tp + r_at[g] + at[i], n, ps[g], g, i) for i, n in enumerate(r)]
    row0, length, depth, tree, branch = (np.array(c, dtype=np.int64) for c in zip(*segs))
    count = -(-length // CHUNK)
    seg = np.repeat(np.arange(len(segs)), count)
    off = (np.arange(len(seg)) - np.repeat(np.cumsum(count) - count, count)) * CHUNK
    n = np.minimum(CHUNK, length[seg] - off)
    rows = (row0[seg] + off)[:, None] + np.arange(CHUNK)[None]
    rows = np.where(np.arange(CHUNK)[None] < n[:, None], rows, total)
    start = depth[seg] + off
    gpu = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return {"rows": gpu(rows), "start": gpu(start), "n": gpu(n), "tree": gpu(tree[seg]), "branch": gpu(branch[seg]),
            "last": gpu(np.cumsum(count) - 1), "tp": tp, "total": total, "trees": len(ps)}


def _weights(plan, decay):
    """log decay per head, the decays inside a block [hkv, C, C], to a block's end and from its start [hkv, n, C], and
    from block m's end to block n's start [hkv, n, m]; all from 64-bit exponents."""
    lg = torch.from_numpy(np.log(decay.astype(np.float64))).cuda()
    i = torch.arange(CHUNK, device="cuda")
    far = i[:, None] - i[None]
    inner = torch.where(far >= 0, torch.exp(lg[:, None, None] * far.clamp(min=0)), 0.0).float()
    to_end = torch.exp(lg[:, None, None] * (plan["n"][:, None] - 1 - i).clamp(min=0)).float()
    from_start = torch.exp(lg[:, None] * (i + 1)).float()
    s, e = plan["start"], plan["start"] + plan["n"]
    same = plan["tree"][:, None] == plan["tree"][None]
    kin = (plan["branch"][:, None] == plan["branch"][None]) | (plan["branch"][None] < 0)
    gap = s[:, None] - e[None]
    between = torch.where(same & kin & (gap >= 0), torch.exp(lg[:, None, None] * gap.clamp(min=0)), 0.0).float()
    return lg, inner, to_end, from_start, between


def _blocks(plan, p, r):
    """[n, heads, C, d] in 32 bits, zeros in the padding."""
    t = torch.cat([p, r, p.new_zeros(1, *p.shape[1:])]).float()
    return t[plan["rows"]].transpose(1, 2)


def _unblock(plan, t, dtype):
    out = t.new_zeros(plan["total"] + 1, t.shape[1], t.shape[3])
    out[plan["rows"].reshape(-1)] = t.transpose(1, 2).reshape(-1, t.shape[1], t.shape[3])
    out = out.to(dtype)
    return out[:plan["tp"]], out[plan["tp"]:plan["total"]]


def _per_kv(t, hkv):
    """[n, hq, C, d] -> [n, hkv, g C, d]"""
    n, h, c, d = t.shape
    return t.reshape(n, hkv, h // hkv * c, d)


def _between(w, states):
    """[hkv, n, m] decays, [m, hkv, a, b] states -> [n, hkv, a, b]"""
    m, h, a, b = states.shape
    return torch.matmul(w, states.permute(1, 0, 2, 3).reshape(h, m, a * b)).reshape(h, -1, a, b).transpose(0, 1)


def _plain(state):
    op, x, case = state["op"], state["x"], state["case"]
    if op == "step":
        return _plain_step(state)
    if op in ("norm", "norm_train"):
        return _plain_norm(op, x, case)
    with torch.no_grad():
        return _plain_linear(op, x, case, state)


def _plain_linear(op, x, case, state):
    plan, hkv, d = state["plan"], case["hkv"], case["d"]
    g, scale = case["hq"] // hkv, 1.0 / math.sqrt(d)
    lg, inner, to_end, from_start, between = _weights(plan, state["decay"])
    rep = lambda w: w.repeat(1, g, 1)                                    # [hkv, C, C] -> [hkv, g C, C]
    q, k, v = (_blocks(plan, x[n + "_p"], x[n + "_r"]) for n in "qkv")
    qg, kt = _per_kv(q, hkv), k.transpose(-1, -2)
    own_state = torch.matmul(kt, to_end.transpose(0, 1)[..., None] * v)  # [n, hkv, d, d]
    s = _between(between, own_state)
    if "state" in x:
        s = s + torch.exp(lg[None, :] * plan["start"][:, None]).float()[..., None, None] * x["state"][plan["tree"]]
    lead = from_start.repeat(1, g)[..., None]                            # [hkv, g C, 1]
    a = torch.matmul(qg, kt).mul_(rep(inner))
    o = (torch.matmul(a, v) + lead * torch.matmul(qg, s)).mul_(scale).reshape(q.shape)
    out = dict(zip(("o_p", "o_r"), _unblock(plan, o, torch.bfloat16)))
    if op == "prefill":
        last = plan["last"]
        end = torch.exp(lg[None, :] * plan["n"][last][:, None]).float()[..., None, None] * s[last] + own_state[last]
        return {**out, "state_p": end[:plan["trees"]], "state_r": end[plan["trees"]:]}
    do = _per_kv(_blocks(plan, x["do_p"], x["do_r"]), hkv)
    b = torch.matmul(do, v.transpose(-1, -2)).mul_(rep(inner))
    dq = (torch.matmul(b, k) + lead * torch.matmul(do, s.transpose(-1, -2))).mul_(scale).reshape(q.shape)
    # backwards in time: the state of what comes after a block, seen from its end
    first = (from_start / from_start[:, :1]).repeat(1, g)[..., None]     # gamma^i from the block's first row
    r = _between(between.transpose(1, 2), torch.matmul(qg.transpose(-1, -2), first * do))
    tail = (to_end * from_start[:, None, :1]).transpose(0, 1)[..., None]  # gamma^(n - j)
    dk = (torch.matmul(b.transpose(-1, -2), qg) + tail * torch.matmul(v, r.transpose(-1, -2))).mul_(scale)
    dv = (torch.matmul(a.transpose(-1, -2), do) + tail * torch.matmul(k, r)).mul_(scale)
    for n, t in (("q", dq), ("k", dk), ("v", dv)):
        out["d" + n + "_p"], out["d" + n + "_r"] = _unblock(plan, t, torch.bfloat16)
    return {n: out[n] for n in ("o_p", "o_r", *("d" + m for m in LEAVES))}


def _plain_step(state):
    x, case = state["x"], state["case"]
    n, hkv, d = x["k"].shape
    q, k, v = (x[m].float() for m in "qkv")
    gamma = torch.from_numpy(state["decay"]).cuda()[:, None, None]
    old = x["state"][x["src"].long()] if "src" in x else x["state"]
    new = gamma * old + k[..., None] * v[..., None, :]
    o = torch.matmul(q.reshape(n, hkv, -1, d), new).reshape(q.shape) / math.sqrt(d)
    return {"o": o.to(torch.bfloat16), "state": new}


def _plain_norm(op, x, case):
    with torch.no_grad():
        t = x["x"].float()
        w = x["weight"] if "weight" in x else 1.0
        b = x["bias"] if "bias" in x else 0.0
        mean = t.mean(-1, keepdim=True)
        rstd = torch.rsqrt((t - mean).square().mean(-1, keepdim=True) + 1e-5)
        n = (t - mean) * rstd
        a = n * w + b
        u = x["gate"].float() if "gate" in x else a
        sig = 1.0 / (1.0 + torch.exp(-u)) if case["act"] == "silu" else torch.ones_like(u)
        act = u * sig
        slope = sig * (1.0 + u * (1.0 - sig))
        y = (a * act if "gate" in x else act).to(torch.bfloat16)
        if op == "norm":
            return {"y": y}
        dy, out = x["dy"].float(), {"y": y}
        da = dy * (act if "gate" in x else slope)
        dn = da * w
        out["dx"] = (rstd * (dn - dn.mean(-1, keepdim=True) - n * (dn * n).mean(-1, keepdim=True))).to(torch.bfloat16)
        if "gate" in x:
            out["dgate"] = (dy * a * slope).to(torch.bfloat16)
        if "weight" in x:
            out["dweight"], out["dbias"] = (da * n).sum(0), da.sum(0)
        return out


# ---------------------------------------------------------------------------------------------------- what it costs


def work(case):
    d = case["d"]
    if case["op"] in ("norm", "norm_train"):
        e = case["rows"] * case["heads"] * d
        tensors = 2 + (1 if case["gate"] else 0)
        if case["op"] == "norm_train":  # x, gate, dy in; y, dx, dgate out
            tensors = 4 + (2 if case["gate"] else 0)
        params = (8 if case["op"] == "norm" else 16) * case["heads"] * d if case["affine"] else 0
        return {"bytes": 2 * e * tensors + params, "flops": e * (15 if case["op"] == "norm" else 40)}
    hq, hkv = case["hq"], case["hkv"]
    if case["op"] == "step":
        n = case["rows"]
        slots = max(1, n // 8) if case["fork"] else n
        return {"bytes": 4 * (n + slots) * hkv * d * d + 2 * n * d * (2 * hq + 2 * hkv),
                "flops": n * d * d * (3 * hkv + 2 * hq)}
    ps, rs = _lengths(case["lengths"])
    t = sum(ps) + sum(map(sum, rs))
    if case["op"] == "prefill":
        states = (2 if case["state"] else 1) * len(ps) + sum(map(len, rs))
        return {"bytes": 2 * t * d * (2 * hq + 2 * hkv) + 4 * states * hkv * d * d,
                "flops": t * d * d * (2 * hq + 2 * hkv)}
    return {"bytes": 2 * t * d * (4 * hq + 4 * hkv), "flops": t * d * d * (6 * hq + 6 * hkv)}


# ---------------------------------------------------------------------------------------------------- in 64 bits


def exact(case, seed):
    """From the definition, in 64 bits: every row against every ancestor row, in blocks of rows, one KV head at a time."""
    if case["op"] == "step":
        return _exact_step(case, seed)
    if case["op"] in ("norm", "norm_train"):
        return _exact_norm(case, seed)
    ps, rs = _lengths(case["lengths"])
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    pairs = sum(p * p / 2 + sum(r * (p + r / 2) for r in b) for p, b in zip(ps, rs))
    if pairs * d * hq * (10 if case["op"] == "train" else 4) > 3e14:
        return None
    x, g, scale = _inputs(case, seed), hq // hkv, 1.0 / math.sqrt(d)
    lg = np.log(_decay(case).astype(np.float64))
    train = case["op"] == "train"
    zeros = lambda *s: torch.zeros(*s, dtype=torch.float64, device="cuda")
    out = {}
    for side in "pr":
        t = x["q_" + side].shape[0]
        out["o_" + side] = zeros(t, hq, d)
        for n, h in (("dq", hq), ("dk", hkv), ("dv", hkv)) if train else ():
            out[n + "_" + side] = zeros(t, h, d)
    if not train:
        out["state_p"], out["state_r"] = zeros(len(ps), hkv, d, d), zeros(sum(map(len, rs)), hkv, d, d)

    def sequence(h, tree, segs, index):
        """The last segment's rows against all segments' (side, first row, length)."""
        side, at, length = segs[-1]
        before = sum(n for _, _, n in segs[:-1])
        k = torch.cat([x["k_" + s][a:a + n, h].double() for s, a, n in segs])
        v = torch.cat([x["v_" + s][a:a + n, h].double() for s, a, n in segs])
        hs, pos = slice(h * g, h * g + g), torch.arange(before + length, device="cuda", dtype=torch.float64)
        if train:
            dk, dv = torch.zeros_like(k), torch.zeros_like(v)
        step = max(64, int(1.2e8 / (g * (before + length))))
        for a in range(0, length, step):
            e = min(length, a + step)
            seen = before + e
            far = pos[before + a:before + e, None] - pos[None, :seen]
            w = torch.exp(far.clamp(min=0) * lg[h]).mul_(scale).masked_fill_(far < 0, 0.0)
            q = x["q_" + side][at + a:at + e, hs].double().transpose(0, 1).contiguous()
            s = torch.matmul(q, k[:seen].t().contiguous()).mul_(w)
            o = torch.matmul(s, v[:seen])
            if "state" in x:
                lead = torch.exp((pos[before + a:before + e] + 1) * lg[h]) * scale
                o += lead[:, None] * torch.matmul(q, x["state"][tree, h].double())
            out["o_" + side][at + a:at + e, hs] = o.transpose(0, 1)
            if not train:
                continue
            do = x["do_" + side][at + a:at + e, hs].double().transpose(0, 1).contiguous()
            b = torch.matmul(do, v[:seen].t().contiguous()).mul_(w)
            out["dq_" + side][at + a:at + e, hs] = torch.matmul(b, k[:seen]).transpose(0, 1)
            dk[:seen] += torch.matmul(b.reshape(-1, seen).t().contiguous(), q.reshape(-1, d))
            dv[:seen] += torch.matmul(s.reshape(-1, seen).t().contiguous(), do.reshape(-1, d))
        if train:
            c = 0
            for sd, a, n in segs:
                out["dk_" + sd][a:a + n, h] += dk[c:c + n]
                out["dv_" + sd][a:a + n, h] += dv[c:c + n]
                c += n
        else:
            w = torch.exp((before + length - 1 - pos) * lg[h])
            end = torch.matmul((k * w[:, None]).t().contiguous(), v)
            if "state" in x:
                end += math.exp(lg[h] * (before + length)) * x["state"][tree, h].double()
            out["state_" + side][index, h] = end

    for h in range(hkv):
        p0 = r0 = index = 0
        for tree, (p, br) in enumerate(zip(ps, rs)):
            sequence(h, tree, [("p", p0, p)], tree)
            for r in br:
                sequence(h, tree, [("p", p0, p), ("r", r0, r)], index)
                r0, index = r0 + r, index + 1
            p0 += p
    names = ("o_p", "o_r", *("d" + m for m in LEAVES)) if train else ("o_p", "o_r", "state_p", "state_r")
    return {n: out[n] for n in names}


def _exact_step(case, seed):
    x, d, g = _inputs(case, seed), case["d"], case["hq"] // case["hkv"]
    gamma = torch.from_numpy(_decay(case).astype(np.float64)).cuda()
    old = x["state"].double()
    if "src" in x:
        old = old[x["src"].long()]
    new = old * gamma.view(1, -1, 1, 1) + x["k"].double().unsqueeze(3) * x["v"].double().unsqueeze(2)
    o = (x["q"].double().unsqueeze(3) * new.repeat_interleave(g, dim=1)).sum(2) / math.sqrt(d)
    return {"o": o, "state": new}


def _exact_norm(case, seed):
    x = {n: t.double() for n, t in _inputs(case, seed).items()}
    for n in ("x", "gate", "weight", "bias"):
        if n in x:
            x[n].requires_grad_(case["op"] == "norm_train")
    t = x["x"]
    var, mean = torch.var_mean(t, dim=-1, unbiased=False, keepdim=True)
    a = (t - mean) / torch.sqrt(var + 1e-5)
    if "weight" in x:
        a = a * x["weight"] + x["bias"]
    act = (lambda u: u * torch.sigmoid(u)) if case["act"] == "silu" else (lambda u: u)
    y = a * act(x["gate"]) if "gate" in x else act(a)
    if case["op"] == "norm":
        return {"y": y}
    names = [n for n in ("x", "gate", "weight", "bias") if n in x]
    grads = torch.autograd.grad(y, [x[n] for n in names], x["dy"])
    return {"y": y.detach(), **{"d" + n: gr for n, gr in zip(names, grads)}}
