"""fp64 reference of the linear-attention layer over replay trees (test infrastructure only).

Written from the definitions: every row against every row of its own prompt and branch, no chunks and no states
(`attention`), the recurrence token by token (`recurrence`), and the norm over each head (`norm`). `attention` also
returns, for every output element, the sums of magnitudes that the tests' error bounds are made of.
"""
from __future__ import annotations

import numpy as np


def segments(cu_prompt, cu_branch, cu_resp):
    """(tree, prompt rows, branch index or None, branch rows) of every sequence that ends in a prompt or a branch."""
    for g in range(len(cu_prompt) - 1):
        p = range(cu_prompt[g], cu_prompt[g + 1])
        yield g, p, None, range(0)
        for b in range(cu_branch[g], cu_branch[g + 1]) if len(cu_branch) > g + 1 else ():
            yield g, p, b, range(cu_resp[b], cu_resp[b + 1])


def attention(cu_prompt, cu_branch, cu_resp, decay, scale, x, state=None, grads=True):
    """x: q_p, k_p, v_p, q_r, k_r, v_r (and do_p, do_r) fp64 [rows, heads, d]. Returns {name: (value, sum over the rows
    of |x| |y| |z|)} for o, dq, dk, dv of both sides, and {state_p, state_r: (value, sum of |k| |v|)}."""
    hq, hkv, d = x["q_p"].shape[1], x["k_p"].shape[1], x["q_p"].shape[2]
    g = hq // hkv
    out = {}
    names = ("o", "dq", "dk", "dv") if grads else ("o",)
    for n in names:
        for s in "pr":
            like = x[("q_" if n in ("o", "dq") else "k_") + s]
            out[n + "_" + s] = tuple(np.zeros(like.shape) for _ in range(2))
    trees, branches = len(cu_prompt) - 1, len(cu_resp) - 1
    out["state_p"] = tuple(np.zeros((trees, hkv, d, d)) for _ in range(2))
    out["state_r"] = tuple(np.zeros((branches, hkv, d, d)) for _ in range(2))

    for tree, p, branch, r in segments(cu_prompt, cu_branch, cu_resp):
        side, at = ("p", p) if branch is None else ("r", r)
        before, n = (0, len(p)) if branch is None else (len(p), len(r))
        total = before + n
        cat = lambda t: np.concatenate([x[t + "_p"][p.start:p.stop]] + ([x[t + "_r"][r.start:r.stop]] if n != total else []))
        k, v = cat("k"), cat("v")
        dist = np.arange(before, total)[:, None] - np.arange(total)[None]
        for h in range(hkv):
            w = np.where(dist >= 0, np.exp(np.log(float(decay[h])) * np.maximum(dist, 0)), 0.0)
            kh, vh = k[:, h], v[:, h]
            lead = np.exp(np.log(float(decay[h])) * (np.arange(before, total) + 1))[:, None]
            s0 = None if state is None else state[tree, h]
            for hh in range(h * g, h * g + g):
                q = x["q_" + side][at.start:at.stop, hh]

                def add(name, rows_of, value, mag):
                    arr = out[name + "_" + rows_of[0]]
                    for t, u in zip(arr, (value, mag)):
                        t[rows_of[1]:rows_of[2], hh if name in ("o", "dq") else h] += scale * u

                me = (side, at.start, at.stop)
                pm, pa = w * (q @ kh.T), w * (abs(q) @ abs(kh).T)
                o, oa = pm @ vh, pa @ abs(vh)
                if s0 is not None:
                    o, oa = o + lead * (q @ s0), oa + lead * (abs(q) @ abs(s0))
                add("o", me, o, oa)
                if not grads:
                    continue
                do = x["do_" + side][at.start:at.stop, hh]
                bm, ba = w * (do @ vh.T), w * (abs(do) @ abs(vh).T)
                dq, qa = bm @ kh, ba @ abs(kh)
                if s0 is not None:
                    dq, qa = dq + lead * (do @ s0.T), qa + lead * (abs(do) @ abs(s0).T)
                add("dq", me, dq, qa)
                for name, m, ma, z in (("dk", bm, ba, q), ("dv", pm, pa, do)):
                    value, mag = m.T @ z, ma.T @ abs(z)
                    add(name, ("p", p.start, p.stop), value[:len(p)], mag[:len(p)])
                    if branch is not None:
                        add(name, me, value[before:], mag[before:])
            end = np.exp(np.log(float(decay[h])) * np.arange(total - 1, -1, -1.0))[:, None]
            s, sa = (end * kh).T @ vh, (end * abs(kh)).T @ abs(vh)
            if s0 is not None:
                s, sa = s + float(decay[h]) ** total * s0, sa + float(decay[h]) ** total * abs(s0)
            i = tree if branch is None else branch
            out["state_" + side][0][i, h], out["state_" + side][1][i, h] = s, sa
    return out


def recurrence(q, k, v, decay, scale, state):
    """One token: (o, new state, sum of |q| |state|); state [rows, hkv, d, d] is what each row goes on from."""
    g = q.shape[1] // k.shape[1]
    new = state * np.asarray(decay, np.float64)[None, :, None, None] + k[..., :, None] * v[..., None, :]
    wide = np.repeat(new, g, axis=1)
    return (scale * np.einsum("rhi,rhij->rhj", q, wide), new,
            scale * np.einsum("rhi,rhij->rhj", abs(q), abs(wide)))


def norm(x, dy=None, weight=None, bias=None, gate=None, silu=False, eps=1e-5):
    """y and, with dy, dx, dgate, dweight, dbias of the norm over the last axis with an activation or a gate."""
    mean = x.mean(-1, keepdims=True)
    rstd = 1.0 / np.sqrt(((x - mean) ** 2).mean(-1, keepdims=True) + eps)
    n = (x - mean) * rstd
    w = np.ones(x.shape[1:]) if weight is None else weight
    a = n * w + (0.0 if bias is None else bias)
    u = a if gate is None else gate
    with np.errstate(over="ignore"):
        sig = 1.0 / (1.0 + np.exp(-u)) if silu else np.ones_like(u)
    act, slope = u * sig, sig * (1.0 + u * (1.0 - sig)) if silu else np.ones_like(u)
    res = {"y": act if gate is None else a * act}
    if dy is None:
        return res
    da = dy * (slope if gate is None else act)
    dn = da * w
    res["dx"] = rstd * (dn - dn.mean(-1, keepdims=True) - n * (dn * n).mean(-1, keepdims=True))
    res["dx_terms"] = rstd * (abs(dn) + abs(dn).mean(-1, keepdims=True) + abs(n) * abs(dn * n).mean(-1, keepdims=True))
    if gate is not None:
        res["dgate"] = dy * a * slope
    res["dweight"], res["dbias"] = (da * n).sum(0), da.sum(0)
    res["dweight_terms"], res["dbias_terms"] = abs(da * n).sum(0), abs(da).sum(0)
    return res
