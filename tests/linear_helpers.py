"""Inputs, runs and error bounds of the linear-attention tests.

Bounds (per element, from the kernels' roundings; a bf16 rounding is off by at most 2^-8 of the value):
  outputs and gradients: 2^-8 |result| (the rounding of the result) + 2^-14 sum |x| |y| |z|: P, the state as an operand
  and the decayed z are two bf16 terms each, off by 2^-16 at most, and at most three of them meet in one term of the
  sum; the fp32 decays are off by about 2^-20 each, fp32 sums of up to a few thousand terms, in a tree of chunks,
  by 2^-17;
  states handed out: (2^-18) sum |k| |v| (three bf16 terms, 2^-24; decays and fp32 sums as above).
"""
import numpy as np
import torch

from oracle import linear as L
from paper_2609_33133_amd import api
from paper_2609_33133_amd.api import GroupBatch

LEAVES = ("q_p", "k_p", "v_p", "q_r", "k_r", "v_r")


def batch(trees, hq, hkv, d, scale=None):
    """trees: [(prompt length, [branch lengths])]; no branches at all where every list is empty."""
    cu = lambda v: np.concatenate([[0], np.cumsum(v)])
    rs = [r for _, br in trees for r in br]
    return GroupBatch(cu([p for p, _ in trees]), cu([len(br) for _, br in trees]), cu(rs), hq, hkv, d, scale)


def decays(h, lo=5.0, hi=12.0):
    return (1.0 - np.exp2(-np.linspace(lo, hi, h))).astype(np.float32)


def inputs(b, seed, device="cuda", amp=1.0):
    gen = torch.Generator().manual_seed(seed)
    x = {}
    for side, t in (("p", b.tp), ("r", b.tr)):
        for n, h in (("q", b.hq), ("k", b.hkv), ("v", b.hkv), ("do", b.hq)):
            x[f"{n}_{side}"] = (amp * torch.randn(t, h, b.d, generator=gen)).to(torch.bfloat16).to(device)
    return x


def to64(t):
    return t.detach().double().cpu().numpy()


def oracle(b, decay, x, state=None, grads=True):
    cu_branch = b.cu_branch if b.num_branches else np.zeros(1, np.int32)
    return L.attention(b.cu_prompt, cu_branch, b.cu_resp, np.asarray(decay, np.float64), b.scale,
                       {k: to64(v) for k, v in x.items()}, None if state is None else to64(state), grads)


def run(b, decay, x, state=None, grads=True, ws=None, stream=None):
    o_p, o_r, s_p, s_r = api.linear_fwd(b, decay, *(x[n] for n in LEAVES), state=state, want_states=True, stream=stream)
    got = {"o_p": o_p, "o_r": o_r, "state_p": s_p, "state_r": s_r}
    if grads:
        g = api.linear_bwd(b, decay, x["q_p"], x["k_p"], x["v_p"], x["do_p"], x["q_r"], x["k_r"], x["v_r"], x["do_r"],
                           state=state, stream=stream)
        got.update(zip(("dq_p", "dk_p", "dv_p", "dq_r", "dk_r", "dv_r"), g))
    return got


def check(got, ref, label=""):
    bad = []
    for n, r in ref.items():
        if n not in got or r[0].size == 0:
            continue
        g = to64(got[n])
        assert g.shape == r[0].shape, (n, g.shape, r[0].shape)
        err = abs(g - r[0])
        bound = 2.0 ** -18 * r[1] if n.startswith("state") else 2.0 ** -8 * abs(r[0]) + 2.0 ** -14 * r[1]
        worst = float((err / np.maximum(bound, 1e-30)).max()) if np.isfinite(err).all() else np.inf
        norm = float(np.linalg.norm(err) / max(np.linalg.norm(r[0]), 1e-30))
        print(f"[{label}] {n}: error / bound {worst:.3f}, relative norm {norm:.2e}", flush=True)
        if not worst <= 1.0:
            bad.append((n, worst, norm))
    assert not bad, (label, bad)
