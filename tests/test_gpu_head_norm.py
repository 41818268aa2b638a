"""The norm over each head with an activation or a gate, and its gradients, against fp64 (oracle/linear.py).

Bounds per element: a result in bf16 is rounded once (2^-8 of it). The fp32 arithmetic before it is off by at most
2^-16 of the magnitudes that enter: n by 2^-18 (mean and variance are fp32 sums of up to 1024 terms in a tree; inputs
here have a mean of at most a few of their own deviations), the activation's exp by a few 2^-23, sums of products by
2^-18. For weight and bias gradients: 2^-16 of the sum of magnitudes."""
import numpy as np
import pytest
import torch

from oracle import linear as L
from paper_2609_33133_amd import api
from paper_2609_33133_amd.autograd import head_norm

from linear_helpers import to64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def make(rows, heads, d, gate, affine, seed=0):
    gen = torch.Generator().manual_seed(seed)
    bf = lambda t: t.to(torch.bfloat16).cuda()
    x = torch.randn(rows, heads, d, generator=gen) * torch.logspace(-1, 1, heads)[:, None] + \
        0.5 * torch.randn(rows, heads, 1, generator=gen)
    t = {"x": bf(x), "dy": bf(torch.randn(rows, heads, d, generator=gen))}
    if gate:
        t["gate"] = bf(2 * torch.randn(rows, heads, d, generator=gen))
    if affine:
        t["weight"] = (1 + 0.3 * torch.randn(heads, d, generator=gen)).cuda()
        t["bias"] = (0.3 * torch.randn(heads, d, generator=gen)).cuda()
    return t


def check(t, silu, eps=1e-5):
    ref = L.norm(**{n: to64(v) for n, v in t.items()}, silu=silu, eps=eps)
    leaf = {n: v.clone().requires_grad_(True) for n, v in t.items() if n != "dy"}
    y = head_norm(leaf["x"], leaf.get("weight"), leaf.get("bias"), gate=leaf.get("gate"),
                  activation="silu" if silu else "none", eps=eps)
    grads = dict(zip(leaf, torch.autograd.grad(y, list(leaf.values()), t["dy"])))
    a_mag = 1 + abs(to64(y)).max() + (abs(to64(t["gate"])).max() if "gate" in t else 0)

    def near(name, got, terms):
        err = abs(to64(got) - ref[name])
        r = abs(ref[name])
        bound = terms + (2.0 ** -8 * r if got.dtype == torch.bfloat16 else 2.0 ** -24 * r)
        worst = float((err / np.maximum(bound, 1e-30)).max())
        print(name, f"error / bound {worst:.3f}", flush=True)
        assert worst <= 1.0, (name, worst)

    near("y", y, 2.0 ** -16 * a_mag)
    near("dx", grads["x"], 2.0 ** -14 * ref["dx_terms"].max(-1, keepdims=True))
    if "gate" in t:
        near("dgate", grads["gate"], 2.0 ** -16 * abs(to64(t["dy"])) * a_mag)
    if "weight" in t:
        near("dweight", grads["weight"], 2.0 ** -16 * ref["dweight_terms"])
        near("dbias", grads["bias"], 2.0 ** -16 * ref["dbias_terms"])


@pytest.mark.parametrize("rows,heads,d", [(1, 1, 8), (7, 3, 16), (33, 5, 24), (65, 28, 128), (130, 4, 64), (9, 2, 80),
                                          (40, 3, 256), (5, 2, 512), (6, 2, 520), (3, 1, 1024), (2049, 1, 32),
                                          (300, 70, 8)])
@pytest.mark.parametrize("gate,silu,affine", [(True, True, True), (False, True, True), (False, False, False),
                                              (True, False, False), (True, True, False)])
def test_matches_reference(rows, heads, d, gate, silu, affine):
    check(make(rows, heads, d, gate, affine, rows + d), silu)


def test_weight_alone_and_bias_alone():
    t = make(50, 4, 64, True, True)
    for drop in ("weight", "bias"):
        u = {n: v for n, v in t.items() if n != drop}
        ref = L.norm(**{n: to64(v) for n, v in u.items()}, silu=True)
        args = {n: u.get(n) for n in ("weight", "bias", "gate")}
        y = api.head_norm_fwd(u["x"], **args, activation=api.ACT_SILU)
        assert (abs(to64(y) - ref["y"]) <= 2.0 ** -8 * abs(ref["y"]) + 2.0 ** -16 * (1 + abs(ref["y"]).max())).all()
        dx, dgate, dweight, dbias = api.head_norm_bwd(u["x"], u["dy"], **args, activation=api.ACT_SILU,
                                                      want_dweight=drop == "bias", want_dbias=drop == "weight")
        kept, gone = (dweight, dbias) if drop == "bias" else (dbias, dweight)
        name = "dweight" if drop == "bias" else "dbias"
        assert gone is None and (abs(to64(kept) - ref[name]) <= 2.0 ** -16 * ref[name + "_terms"]).all()


def test_constant_rows_and_large_gates():
    """A head without variance gives the bias; gates far from zero neither overflow nor turn into NaN."""
    t = make(6, 2, 64, True, True)
    t["x"][:] = 3.0
    t["gate"][0], t["gate"][1] = 300.0, -300.0
    check(t, True)


def test_in_place():
    t = make(300, 4, 128, True, True)
    args = dict(weight=t["weight"], bias=t["bias"], activation=api.ACT_SILU)
    y = api.head_norm_fwd(t["x"], gate=t["gate"], **args)
    dx, dgate, _, _ = api.head_norm_bwd(t["x"], t["dy"], gate=t["gate"], **args)
    for n in ("x", "gate"):
        c = {k: v.clone() for k, v in t.items()}
        assert torch.equal(api.head_norm_fwd(c["x"], gate=c["gate"], y=c[n], **args), y)
    c = {k: v.clone() for k, v in t.items()}
    api.head_norm_bwd(c["x"], c["dy"], gate=c["gate"], dx=c["dy"], dgate=c["gate"], **args)
    assert torch.equal(c["dy"], dx) and torch.equal(c["gate"], dgate)


def test_no_rows():
    t = make(0, 3, 64, True, True)
    y = api.head_norm_fwd(t["x"], t["weight"], t["bias"], t["gate"])
    dx, dgate, dw, db = api.head_norm_bwd(t["x"], t["dy"], t["weight"], t["bias"], t["gate"], want_dweight=True,
                                          want_dbias=True)
    assert y.numel() == dx.numel() == 0 and not dw.any() and not db.any()


def test_runs_repeat_and_replay():
    t = make(5000, 4, 128, True, True)
    args = (t["x"], t["dy"], t["weight"], t["bias"], t["gate"], api.ACT_SILU)
    a = api.head_norm_bwd(*args, want_dweight=True, want_dbias=True)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b = api.head_norm_bwd(*args, want_dweight=True, want_dbias=True)
    for _ in range(3):
        g.replay()
        torch.cuda.synchronize()
        c = api.head_norm_bwd(*args, want_dweight=True, want_dbias=True)
        for u, v, w in zip(a, b, c):
            assert torch.equal(u, v) and torch.equal(u, w)


def test_offsets_past_31_bits():
    """Rows behind 2^31 elements, as on their own."""
    rows, tail = 2 ** 31 // (16 * 128) + 50, 40
    gen = torch.Generator(device="cuda").manual_seed(6)
    x, dy, gate = (torch.empty(rows, 16, 128, dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for _ in range(3))
    w, b = (torch.empty(16, 128, device="cuda").normal_(generator=gen) for _ in range(2))
    last = [t[-tail:].contiguous() for t in (x, dy, gate)]
    assert torch.equal(api.head_norm_fwd(x, w, b, gate, api.ACT_SILU)[-tail:],
                       api.head_norm_fwd(last[0], w, b, last[2], api.ACT_SILU))
    got = api.head_norm_bwd(x, dy, w, b, gate, api.ACT_SILU)
    want = api.head_norm_bwd(*last[:2], w, b, last[2], api.ACT_SILU)
    assert torch.equal(got[0][-tail:], want[0]) and torch.equal(got[1][-tail:], want[1])
