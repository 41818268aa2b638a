"""Linear attention over replay trees on the GPU against the fp64 reference (oracle/linear.py), at the lengths, head
layouts and decays where the blocks, chunks and forks can go wrong."""
import numpy as np
import pytest
import torch

from paper_2609_33133_amd import api
from paper_2609_33133_amd.autograd import group_linear_attention

from linear_helpers import LEAVES, batch, check, decays, inputs, oracle, run, to64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


CASES = {
    "one_token": ([(1, [1])], 2, 2, 64),
    "chunk_edges": ([(63, [1, 64, 65]), (64, [63, 2]), (129, [128])], 4, 2, 64),
    "block_edges": ([(127, [129, 1]), (128, [128, 257]), (385, [384, 127])], 2, 1, 128),
    "many_blocks": ([(1000, [300, 77, 513])], 2, 2, 128),
    "grouped_heads": ([(200, [70, 131]), (33, [5])], 14, 2, 128),
    "one_kv_head": ([(150, [90])], 8, 1, 64),
    "d64_blocks": ([(700, [260, 3])], 4, 4, 64),
    "scan_groups": ([(1024, [512, 1088]), (1040, [1000])], 1, 1, 64),
    "long_blocks": ([(2100, [1500])], 64, 32, 64),
}


@pytest.mark.parametrize("name", list(CASES))
def test_matches_reference(name):
    trees, hq, hkv, d = CASES[name]
    b = batch(trees, hq, hkv, d)
    dec = decays(hkv)
    x = inputs(b, 11)
    check(run(b, dec, x), oracle(b, dec, x), name)


@pytest.mark.parametrize("decay", [1.0, 0.5, 1e-3, 1e-30], ids=str)
def test_decays_from_none_to_all(decay):
    b = batch([(150, [70, 65])], 4, 2, 64)
    dec = np.full(2, decay, np.float32)
    x = inputs(b, 12)
    check(run(b, dec, x), oracle(b, dec, x), f"decay {decay}")


def test_begins_from_a_state():
    b = batch([(200, [70, 131]), (33, [5])], 4, 2, 128)
    dec = decays(2)
    x = inputs(b, 13)
    state = torch.randn(2, 2, 128, 128, generator=torch.Generator().manual_seed(5)).mul(4).cuda()
    check(run(b, dec, x, state=state), oracle(b, dec, x, state=state), "state")


def test_backward_from_the_forwards_workspace():
    b = batch([(300, [70, 257]), (33, [5])], 4, 2, 128)
    dec = decays(2)
    x = inputs(b, 24)
    ws = torch.empty(api.linear_workspace_size(b), dtype=torch.uint8, device="cuda")
    api.linear_fwd(b, dec, *(x[n] for n in LEAVES), ws=ws)
    args = (b, dec, x["q_p"], x["k_p"], x["v_p"], x["do_p"], x["q_r"], x["k_r"], x["v_r"], x["do_r"])
    keep = ws.clone()
    for g, w in zip(api.linear_bwd(*args, fwd_ws=ws), api.linear_bwd(*args)):
        assert torch.equal(g, w)
    assert torch.equal(ws, keep)


def test_many_blocks_scan_branches_side_by_side():
    """More blocks in a tree than one scan launch takes (32)."""
    b = batch([(4500, [1300, 2500, 1]), (70, [300])], 1, 1, 64)
    dec = decays(1, 8.0, 8.0)
    x = inputs(b, 25)
    check(run(b, dec, x), oracle(b, dec, x), "two scan launches")


def test_pieces_of_a_sequence_in_place():
    """A prompt taken in pieces, its state updated in place, is the prompt taken at once."""
    whole = batch([(300, [])], 4, 2, 64)
    dec = decays(2)
    x = inputs(whole, 26)
    ref = oracle(whole, dec, x, grads=False)
    state = torch.zeros(1, 2, 64, 64, device="cuda")
    outs, a = [], 0
    for n in (130, 1, 169):
        b = batch([(n, [])], 4, 2, 64)
        part = [x[m + "_p"][a:a + n].contiguous() for m in "qkv"]
        o, _, s, _ = api.linear_fwd(b, dec, *part, *(x[m][:0] for m in ("q_r", "k_r", "v_r")), state=state, state_p=state)
        assert s is state
        outs.append(o)
        a += n
    check({"o_p": torch.cat(outs), "state_p": state}, {n: ref[n] for n in ("o_p", "state_p")}, "pieces")


def test_a_given_stream():
    """Memory that a call allocates belongs to the stream it is given."""
    b = batch([(2000, [700] * 4)], 4, 2, 128)
    dec = decays(2)
    x = inputs(b, 27)
    want = run(b, dec, x)
    s = torch.cuda.Stream()
    for _ in range(3):
        s.wait_stream(torch.cuda.current_stream())
        got = run(b, dec, x, stream=s)
        noise = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(8)]  # reuses what the calls freed
        torch.cuda.current_stream().wait_stream(s)
        for n in want:
            assert torch.equal(want[n], got[n]), n
        del noise


def test_sequences_without_branches():
    b = batch([(200, []), (1, []), (500, [])], 4, 2, 64)
    dec = decays(2)
    x = inputs(b, 14)
    got = run(b, dec, x)
    assert got["state_r"].shape[0] == 0
    check(got, oracle(b, dec, x), "no branches")


def test_more_segments_than_the_kernel_arguments_hold():
    rng = np.random.default_rng(3)
    trees = [(int(rng.integers(1, 140)), [int(r) for r in rng.integers(1, 70, 25)]) for _ in range(40)]
    b = batch(trees, 2, 1, 64)
    dec = decays(1)
    x = inputs(b, 15)
    check(run(b, dec, x), oracle(b, dec, x), "1040 segments")


def test_more_segments_than_two_looks_tell_apart():
    """Blocks find their segment by looking at 64 segments at once: 4096 take two looks."""
    b = batch([(1 + i % 3, [1 + i % 2]) for i in range(2100)], 1, 1, 64)
    dec = decays(1)
    x = inputs(b, 37)
    check(run(b, dec, x), oracle(b, dec, x), "4200 segments")


def test_outputs_do_not_depend_on_whether_states_are_asked_for():
    b = batch([(300, [70, 257])], 4, 2, 128)
    dec = decays(2)
    x = inputs(b, 16)
    a = run(b, dec, x)
    o_p, o_r, s_p, s_r = api.linear_fwd(b, dec, *(x[n] for n in LEAVES))
    assert s_p is None and s_r is None
    assert torch.equal(o_p, a["o_p"]) and torch.equal(o_r, a["o_r"])


def test_a_tree_does_not_depend_on_the_batch_and_runs_repeat():
    t1, t2 = (333, [120, 65]), (70, [200])
    both, alone = batch([t1, t2], 4, 2, 128), batch([t2], 4, 2, 128)
    dec = decays(2)
    x = inputs(both, 17)
    y = {n: t[(333 if n.endswith("p") else 185):].contiguous() for n, t in x.items()}
    a, a2, c = run(both, dec, x), run(both, dec, x), run(alone, dec, y)
    for n in a:
        assert torch.equal(a[n], a2[n]), n
        if not n.startswith("state"):
            assert torch.equal(a[n][333 if n.endswith("p") else 185:], c[n]), n


def test_prefill_then_steps_equal_one_longer_sequence():
    """Prompt, fork, single tokens: the outputs of linear_step are the branch rows of the chunked form."""
    P, G, R = 150, 3, 5
    b = batch([(P, [R] * G)], 4, 2, 128)
    dec = decays(2)
    x = inputs(b, 18)
    ref = oracle(b, dec, x, grads=False)
    prompt = batch([(P, [])], 4, 2, 128)
    empty = [x[n][:0] for n in ("q_r", "k_r", "v_r")]
    _, _, state, _ = api.linear_fwd(prompt, dec, x["q_p"], x["k_p"], x["v_p"], *empty, want_states=True)
    src = torch.zeros(G, dtype=torch.int32, device="cuda")
    rows = torch.arange(G, device="cuda") * R
    for t in range(R):
        q, k, v = (x[n][rows + t].contiguous() for n in ("q_r", "k_r", "v_r"))
        o, state = api.linear_step(q, k, v, dec, state, src=src if t == 0 else None,
                                   state_out=None if t == 0 else state)
        at = rows.cpu().numpy() + t
        want, mag = ref["o_r"][0][at], ref["o_r"][1][at]
        assert (abs(to64(o) - want) <= 2.0 ** -8 * abs(want) + 2.0 ** -17 * mag).all(), t
    assert (abs(to64(state) - ref["state_r"][0]) <= 2.0 ** -18 * ref["state_r"][1]).all()


def test_nan_stays_in_its_tree_and_branch():
    b = batch([(100, [50, 60]), (70, [33])], 2, 1, 64)
    dec = decays(1)
    x = inputs(b, 19)
    clean = run(b, dec, x)
    x["v_r"][10] = float("nan")  # in the first branch
    got = run(b, dec, x, grads=False)
    assert torch.equal(got["o_p"], clean["o_p"])
    assert torch.equal(got["o_r"][50:], clean["o_r"][50:])
    assert got["o_r"][10:50].isnan().all()


def test_autograd_and_differences():
    """Gradients that autograd returns are the explicit calls', and match differences of the loss."""
    b = batch([(90, [40, 67])], 4, 2, 64)
    dec = decays(2)
    x = inputs(b, 20)
    leaf = {n: x[n].clone().requires_grad_(True) for n in LEAVES}
    o_p, o_r = group_linear_attention(*(leaf[n] for n in LEAVES), b, dec)
    grads = torch.autograd.grad((o_p, o_r), [leaf[n] for n in LEAVES], (x["do_p"], x["do_r"]))
    got = run(b, dec, x)
    for n, g in zip(LEAVES, grads):
        assert torch.equal(g, got["d" + n]), n
    # the loss is linear in each tensor on its own: its difference along a direction is the gradient times it
    ref = oracle(b, dec, x)
    loss = lambda y: sum((oracle(b, dec, y, grads=False)["o_" + s][0] * to64(x["do_" + s])).sum() for s in "pr")
    for n in LEAVES:
        step = torch.randn(x[n].shape, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
        moved = dict(x, **{n: x[n].double() + step.double()})
        diff = loss(moved) - loss(x)
        along = (ref["d" + n][0] * to64(step)).sum()
        assert abs(diff - along) <= 1e-9 * (abs(ref["d" + n][0]) * abs(to64(step))).sum(), n


def test_no_second_derivatives():
    b = batch([(20, [4])], 2, 2, 64)
    x = inputs(b, 28)
    leaf = [x[n].requires_grad_(True) for n in LEAVES]
    o = group_linear_attention(*leaf, b, 0.9)
    g, = torch.autograd.grad(o[0].float().sum(), leaf[:1], create_graph=True)
    with pytest.raises(RuntimeError):
        g.float().sum().backward()


def test_strided_inputs_and_unused_outputs():
    """autograd takes views (a fused qkv projection's), and an output outside the loss has no gradient."""
    b = batch([(90, [40])], 4, 2, 64)
    dec = decays(2)
    x = inputs(b, 21)
    def fused(s):
        t = torch.cat([x["q_" + s], x["k_" + s], x["v_" + s]], 1).requires_grad_(True)
        return t, (t[:, :4], t[:, 4:6], t[:, 6:])
    (tp, vp), (tr, vr) = fused("p"), fused("r")
    o_p, o_r = group_linear_attention(*vp, *vr, b, dec)
    (o_r.float() * x["do_r"].float()).sum().backward()
    x["do_p"] = torch.zeros_like(x["do_p"])
    got = run(b, dec, x)
    assert torch.equal(o_p, got["o_p"]) and torch.equal(o_r, got["o_r"])
    assert torch.equal(tp.grad, torch.cat([got["dq_p"], got["dk_p"], got["dv_p"]], 1))
    assert torch.equal(tr.grad, torch.cat([got["dq_r"], got["dk_r"], got["dv_r"]], 1))


def test_graph_replays_and_other_streams():
    b = batch([(300, [70, 257])], 4, 2, 128)
    dec = decays(2)
    x = inputs(b, 22)
    state = torch.zeros(1, 2, 128, 128, device="cuda")
    want = run(b, dec, x, state=state)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run(b, dec, x, state=state)
    torch.cuda.synchronize()
    for n in want:
        assert torch.equal(want[n], got[n]), n
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = run(b, dec, x, state=state)
    y = inputs(b, 23)
    for k in range(4):
        for n in x:
            x[n].copy_(y[n] if k % 2 else inputs(b, 22)[n])
        g.replay()
        torch.cuda.synchronize()
        eager = run(b, dec, x, state=state)
        for n in want:
            assert torch.equal(eager[n], got[n]), (k, n)


def test_a_layer_trains_and_decodes():
    """The operators as a layer uses them: projections, linear attention over the tree, gated norm, a loss; against the
    same layer in fp64 through torch's own autograd; then two decoded tokens from the branches' states."""
    torch.manual_seed(7)
    hq, hkv, d, m = 4, 2, 64, 96
    trees = [(70, [20, 33]), (10, [9])]
    b = batch(trees, hq, hkv, d)
    dec = decays(hkv)
    from paper_2609_33133_amd.autograd import head_norm
    par = {"wq": torch.randn(m, hq * d) / m ** 0.5, "wk": torch.randn(m, hkv * d) / m ** 0.5,
           "wv": torch.randn(m, hkv * d) / m ** 0.5, "wg": torch.randn(m, hq * d) / m ** 0.5,
           "w": 1 + 0.1 * torch.randn(hq, d), "b": 0.1 * torch.randn(hq, d)}
    h = {"p": torch.randn(b.tp, m), "r": torch.randn(b.tr, m)}
    t = {"p": torch.randn(b.tp, hq * d), "r": torch.randn(b.tr, hq * d)}

    def layer(par, h, attend, norm):
        f = {s: {n: (h[s] @ par["w" + n]).reshape(len(h[s]), -1, d) for n in "qkvg"} for s in "pr"}
        o = attend(*(f[s][n] for s in "pr" for n in "qkv"))
        return {s: norm(o_s, par["w"], par["b"], f[s]["g"]) for s, o_s in zip("pr", o)}

    def plain_attend(qp, kp, vp, qr, kr, vr):
        lg = torch.from_numpy(np.log(dec.astype(np.float64)))
        def rows(q, k, v, pos_q):
            dist = (pos_q[:, None] - torch.arange(len(k))[None]).double()
            w = torch.where(dist >= 0, torch.exp(lg[:, None, None] * dist.clamp(min=0)), 0.0).repeat_interleave(hq // hkv, 0)
            k, v = (y.repeat_interleave(hq // hkv, 1).transpose(0, 1) for y in (k, v))
            return (((q.transpose(0, 1) @ k.transpose(1, 2)) * w * b.scale) @ v).transpose(0, 1)
        op, orr, pa, ra = [], [], 0, 0
        for p, br in trees:
            op.append(rows(qp[pa:pa + p], kp[pa:pa + p], vp[pa:pa + p], torch.arange(p)))
            for r in br:
                k, v = torch.cat([kp[pa:pa + p], kr[ra:ra + r]]), torch.cat([vp[pa:pa + p], vr[ra:ra + r]])
                orr.append(rows(qr[ra:ra + r], k, v, torch.arange(p, p + r)))
                ra += r
            pa += p
        return torch.cat(op), torch.cat(orr)

    def plain_norm(x, w, bias, g):
        n = (x - x.mean(-1, keepdim=True)) / torch.sqrt(x.var(-1, unbiased=False, keepdim=True) + 1e-5)
        return (n * w + bias) * torch.nn.functional.silu(g)

    ref = {k: v.double().requires_grad_(True) for k, v in par.items()}
    y = layer(ref, {s: v.double() for s, v in h.items()}, plain_attend, plain_norm)
    sum((y[s].flatten(1) * t[s].double()).sum() for s in "pr").backward()
    gpu = {k: v.cuda().requires_grad_(True) for k, v in par.items()}
    bf = lambda z: z.to(torch.bfloat16)
    got = layer(gpu, {s: v.cuda() for s, v in h.items()},
                lambda *a: group_linear_attention(*(bf(z) for z in a), b, dec),
                lambda o, w, bias, g: head_norm(o, w, bias, gate=bf(g), activation="silu"))
    sum((got[s].float().flatten(1) * t[s].cuda()).sum() for s in "pr").backward()
    # bf16 q, k, v, P, o, gate, y forward and as many roundings backward: some ten independent ones of 2^-8 at most
    for s in "pr":
        e = np.linalg.norm(to64(got[s]) - y[s].detach().numpy()) / np.linalg.norm(y[s].detach().numpy())
        assert e <= 10 * 2.0 ** -8, (s, e)
    for n in par:
        e = np.linalg.norm(to64(gpu[n].grad) - ref[n].grad.numpy()) / np.linalg.norm(ref[n].grad.numpy())
        assert e <= 10 * 2.0 ** -8, (n, e)


def test_a_tree_scanned_beside_a_longer_one():
    """The longer tree has its branches scanned by a launch of their own, and the short one with it; alone the short
    one's take one launch with its prompt."""
    t1, t2 = (2500, [300, 20]), (200, [70, 333])
    both, alone = batch([t1, t2], 2, 1, 128), batch([t2], 2, 1, 128)
    dec = decays(1)
    x = inputs(both, 29)
    y = {n: t[(2500 if n.endswith("p") else 320):].contiguous() for n, t in x.items()}
    a, c = run(both, dec, x), run(alone, dec, y)
    for n in a:
        at = (1 if n.endswith("p") else 2) if n.startswith("state") else 2500 if n.endswith("p") else 320
        assert torch.equal(a[n][at:], c[n]), n


def test_offsets_past_31_bits():
    """A small tree behind one whose query rows take 2^31 elements, of prompt and branch: as on its own."""
    n = 2 ** 31 // (16 * 128) + 65
    b, alone = batch([(n, [n - 1]), (100, [70])], 16, 1, 128), batch([(100, [70])], 16, 1, 128)
    dec = decays(1)
    gen = torch.Generator(device="cuda").manual_seed(31)
    x = {}
    for side, t in (("p", b.tp), ("r", b.tr)):
        for name, h in (("q", 16), ("k", 1), ("v", 1), ("do", 16)):
            x[f"{name}_{side}"] = torch.empty(t, h, 128, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    y = {k: t[n if k.endswith("p") else n - 1:].contiguous() for k, t in x.items()}
    got, want = run(b, dec, x), run(alone, dec, y)
    for k in want:
        at = 1 if k.startswith("state") else n if k.endswith("p") else n - 1
        assert torch.equal(got[k][at:], want[k]), k


def test_captured_training_step_replays():
    """Forward and backward through autograd in one graph. (No eager graph of the leaves is alive at the capture.)"""
    b = batch([(150, [70, 33])], 4, 2, 64)
    dec = decays(2)
    x = inputs(b, 41)

    def grads(leaves):
        o_p, o_r = group_linear_attention(*leaves, b, dec)
        return torch.autograd.grad((o_p, o_r), leaves, (x["do_p"], x["do_r"]))

    def leaves():
        return [x[n].clone().requires_grad_() for n in LEAVES]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        grads(leaves())
    torch.cuda.synchronize()
    static = leaves()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = grads(static)
    for k in range(3):
        y = inputs(b, 42 + k)
        with torch.no_grad():
            for n, t in zip(LEAVES, static):
                x[n].copy_(y[n])
                t.copy_(y[n])
        g.replay()
        torch.cuda.synchronize()
        for u, v in zip(got, grads(leaves())):
            assert torch.equal(u, v), k
