"""Refusals of the linear-attention layer's entry points (no GPU: every call fails before anything is enqueued)."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2609_33133_amd import _lib, api
from paper_2609_33133_amd.api import GroupBatch
from paper_2609_33133_amd.autograd import group_linear_attention, head_norm

OK, INVALID, UNSUPPORTED, MISALIGNED, WORKSPACE, DEVICE = range(6)


@pytest.fixture(scope="module")
def C():
    return _lib.load()


def fake(n=1 << 20):
    """A 256-byte-aligned address that is never dereferenced."""
    return ctypes.c_void_p(n * 256)


ODD = ctypes.c_void_p((1 << 28) + 2)
BIG = 1 << 40


def dec(*v):
    return np.array(v, np.float32)


def at(i):
    """Address i of tensors that lie apart."""
    return ctypes.c_void_p((1 << 50) + (i << 44))


FWD = ("q_p", "k_p", "v_p", "q_r", "k_r", "v_r", "state", "o_p", "o_r", "state_p", "state_r")
BWD = ("q_p", "k_p", "v_p", "do_p", "q_r", "k_r", "v_r", "do_r", "state", "dq_p", "dk_p", "dv_p", "dq_r", "dk_r", "dv_r")


def tensors(names, kw):
    optional = {"state": None, "state_p": None, "state_r": None}
    return [kw[n] if n in kw else optional.get(n, at(i)) for i, n in enumerate(names)]


def fwd(C, b, decay, ws=at(30), n=1 << 40, **kw):
    return C.augtree_linear_fwd(b.ref, decay.ctypes.data_as(ctypes.c_void_p), *tensors(FWD, kw), ws, n, None)


def bwd(C, b, decay, ws=at(30), n=1 << 40, fwd_ws=None, fwd_n=0, **kw):
    return C.augtree_linear_bwd(b.ref, decay.ctypes.data_as(ctypes.c_void_p), *tensors(BWD, kw), fwd_ws, fwd_n, ws, n, None)


GOOD = ([0, 10, 25], [0, 2, 3], [0, 5, 12, 20])


def test_valid_calls_reach_the_device_check(C):
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    b = GroupBatch(*GOOD, 4, 2, 64)
    assert fwd(C, b, dec(0.9, 1.0)) == DEVICE and bwd(C, b, dec(0.9, 1.0)) == DEVICE
    plain = GroupBatch([0, 10, 25], [0, 0, 0], [0], 4, 2, 64)
    none = {n: None for n in ("q_r", "k_r", "v_r", "o_r")}
    assert fwd(C, plain, dec(1, 1), **none) == DEVICE
    assert fwd(C, plain, dec(1, 1), state=at(25), state_p=at(25), **none) == DEVICE


@pytest.mark.parametrize("args,code", [
    (([0, 10, 10], [0, 2, 3], [0, 5, 12, 20], 4, 2, 64), INVALID),    # empty prompt
    (([0, 10, 25], [0, 2, 2], [0, 5, 12, 20], 4, 2, 64), INVALID),    # group without branch
    (([0, 10, 25], [0, 2, 3], [0, 5, 5, 20], 4, 2, 64), INVALID),     # empty branch
    (([1, 10, 25], [0, 2, 3], [0, 5, 12, 20], 4, 2, 64), INVALID),    # offsets not from 0
    (([0, 10, 25], [0, 1, 2], [0, 5, 12, 20], 4, 2, 64), INVALID),    # branches that no group has
    (([0, 10, 25], [0, 2, 3], [0, 5, 12, 20], 4, 3, 64), UNSUPPORTED),
    (([0, 10, 25], [0, 2, 3], [0, 5, 12, 20], 4, 2, 96), UNSUPPORTED),
    (([0, 10, 25], [0, 2, 3], [0, 5, 12, 20], 514, 257, 64), UNSUPPORTED),
])
def test_bad_batches(C, args, code):
    b = GroupBatch(*args)
    d = np.ones(b.hkv, np.float32)
    assert fwd(C, b, d) == code and bwd(C, b, d) == code
    assert C.augtree_linear_workspace_size(b.ref, 0) == 0 and C.augtree_last_error() != b""
    with pytest.raises(_lib.AugtreeError):
        api.linear_workspace_size(b)


@pytest.mark.parametrize("bad", [0.0, -0.5, 1.0001, float("nan"), float("inf")])
def test_bad_decays(C, bad):
    b = GroupBatch(*GOOD, 4, 2, 64)
    assert fwd(C, b, dec(0.9, bad)) == INVALID and bwd(C, b, dec(bad, 0.9)) == INVALID
    assert C.augtree_linear_step(2, 4, 2, 64, 0.1, dec(0.9, bad).ctypes.data_as(ctypes.c_void_p), at(0), at(1), at(2), 2,
                                 at(3), None, at(4), at(5), None) == INVALID


def test_bad_pointers_and_workspaces(C):
    b, d = GroupBatch(*GOOD, 4, 2, 64), dec(0.9, 0.9)
    assert C.augtree_linear_fwd(None, None, *[None] * 11, None, 0, None) == INVALID
    assert C.augtree_linear_fwd(b.ref, None, *tensors(FWD, {}), at(30), BIG, None) == INVALID
    for n in FWD:
        assert fwd(C, b, d, **{n: ODD}) == MISALIGNED, n
        if n[:5] != "state":
            assert fwd(C, b, d, **{n: None}) == INVALID, n
    for n in BWD:
        assert bwd(C, b, d, **{n: ODD}) == MISALIGNED, n
        if n != "state":
            assert bwd(C, b, d, **{n: None}) == INVALID, n
    need = [C.augtree_linear_workspace_size(b.ref, k) for k in (0, 1)]
    assert 0 < need[0] < need[1] and need[0] % 256 == 0
    off = ctypes.c_void_p(at(30).value + 16)
    assert fwd(C, b, d, n=need[0] - 1) == WORKSPACE and fwd(C, b, d, ws=None) == WORKSPACE
    assert fwd(C, b, d, ws=off) == MISALIGNED
    assert bwd(C, b, d, n=need[1] - 1) == WORKSPACE and bwd(C, b, d, ws=None) == WORKSPACE
    assert bwd(C, b, d, fwd_ws=at(31), fwd_n=need[0] - 1) == WORKSPACE
    assert bwd(C, b, d, fwd_ws=off, fwd_n=need[0], ws=at(31)) == MISALIGNED
    plain = GroupBatch([0, 10], [0, 0], [0], 4, 2, 64)
    assert fwd(C, plain, d, state_r=at(29)) == INVALID
    scale = GroupBatch(*GOOD, 4, 2, 64, softmax_scale=float("inf"))
    assert fwd(C, scale, d) == INVALID


def test_outputs_lie_apart(C):
    b, d = GroupBatch(*GOOD, 4, 2, 64), dec(0.9, 0.9)
    last = ctypes.c_void_p(at(0).value + 25 * 4 * 64 * 2 - 16)  # inside q_p
    for n in ("o_p", "o_r", "state_p", "state_r"):
        assert fwd(C, b, d, **{n: at(0)}) == INVALID and fwd(C, b, d, **{n: last}) == INVALID, n
        assert b"overlaps" in C.augtree_last_error()
    assert fwd(C, b, d, o_r=at(7)) == INVALID and fwd(C, b, d, ws=at(7)) == INVALID
    assert fwd(C, b, d, state=at(25), state_r=at(25)) == INVALID
    for n in BWD[9:]:
        assert bwd(C, b, d, **{n: at(3)}) == INVALID, n
    assert bwd(C, b, d, dk_p=at(11)) == INVALID and bwd(C, b, d, ws=at(4)) == INVALID
    assert bwd(C, b, d, fwd_ws=at(30), fwd_n=1 << 30) == INVALID  # the same memory as ws


def test_step_refusals(C):
    p, far = at(0), at(1)

    def step(rows=4, hq=4, hkv=2, d=64, scale=0.1, n=4, s_in=p, src=None, s_out=far, q=at(2), o=at(5)):
        return C.augtree_linear_step(rows, hq, hkv, d, scale, np.ones(300, np.float32).ctypes.data_as(ctypes.c_void_p), q,
                                     at(3), at(4), n, s_in, src, s_out, o, None)
    assert step(rows=0) == OK and step(rows=-1) == INVALID and step(n=-1) == INVALID
    assert step(n=3) == INVALID and step(d=32) == UNSUPPORTED and step(hq=3) == UNSUPPORTED
    assert step(hq=257, hkv=257) == UNSUPPORTED and step(scale=0.0) == INVALID
    assert step(q=None) == INVALID and step(q=ODD) == MISALIGNED and step(src=ODD.value + 1) == MISALIGNED
    # overlaps: in place needs the same address and no src
    assert step(src=at(6), s_out=p) == INVALID and step(o=at(2)) == INVALID and step(s_out=at(5)) == INVALID
    assert step(s_out=ctypes.c_void_p(p.value + 2 * 64 * 64 * 4)) == INVALID
    assert step(rows=2 ** 31 - 1, n=2 ** 31 - 1, hq=256, hkv=256, s_in=ctypes.c_void_p(1 << 60), s_out=ctypes.c_void_p(1 << 61)) == UNSUPPORTED
    if not torch.cuda.is_available():
        assert step() == DEVICE and step(s_out=p) == DEVICE and step(src=at(6), n=1) == DEVICE


def test_norm_refusals(C):
    p = fake()

    def fwd_(rows=4, heads=2, d=64, act=1, eps=1e-5, x=p, y=p):
        return C.augtree_head_norm_fwd(rows, heads, d, act, eps, x, None, None, None, y, None)
    assert fwd_(rows=0, x=None) == OK and fwd_(rows=-1) == INVALID
    for d in (0, 4, 12, 1032):
        assert fwd_(d=d) == UNSUPPORTED and C.augtree_head_norm_workspace_size(4, 2, d) == 0
    assert fwd_(heads=0) == UNSUPPORTED and fwd_(heads=65536) == UNSUPPORTED and fwd_(act=2) == INVALID
    assert fwd_(eps=0.0) == INVALID and fwd_(eps=float("nan")) == INVALID and fwd_(x=None) == INVALID
    assert fwd_(y=ODD) == MISALIGNED and fwd_(rows=2 ** 47) == UNSUPPORTED

    def bwd_(rows=4, gate=None, dgate=None, dw=None, ws=None, n=0):
        return C.augtree_head_norm_bwd(rows, 2, 64, 1, 1e-5, p, gate, None, None, p, p, dgate, dw, None, ws, n, None)
    assert bwd_(gate=p) == INVALID and bwd_(dgate=p) == INVALID
    need = C.augtree_head_norm_workspace_size(4, 2, 64)
    assert need > 0 and bwd_(dw=p) == WORKSPACE and bwd_(dw=p, ws=p, n=need - 1) == WORKSPACE
    assert bwd_(dw=p, ws=ctypes.c_void_p((1 << 28) + 16), n=need) == MISALIGNED
    assert bwd_(rows=0) == OK


def test_norm_outputs_lie_apart(C):
    n = 4 * 2 * 64 * 2

    def inside(i):
        return ctypes.c_void_p(at(i).value + n - 16)

    def fwd_(y, x=at(0), gate=at(1), weight=at(2), bias=at(3)):
        return C.augtree_head_norm_fwd(4, 2, 64, 1, 1e-5, x, gate, weight, bias, y, None)

    def bwd_(dx=at(5), dgate=at(6), dw=at(7), db=at(8), ws=at(9)):
        return C.augtree_head_norm_bwd(4, 2, 64, 1, 1e-5, at(0), at(1), at(2), at(3), at(4), dx, dgate, dw, db, ws, 1 << 30,
                                       None)
    for i in range(4):
        assert fwd_(inside(i) if i < 2 else at(i)) == INVALID, i
        assert b"overlaps" in C.augtree_last_error()
    for kw in ("dx", "dgate", "dw", "db", "ws"):
        for i in (0, 1, 4):
            bad = ctypes.c_void_p(at(i).value + 256) if kw == "ws" else inside(i)
            assert bwd_(**{kw: bad}) == INVALID, (kw, i)
        assert bwd_(**{kw: at(2)}) == INVALID, kw
    assert bwd_(dx=at(6)) == INVALID and bwd_(dx=at(0), dgate=at(0)) == INVALID and bwd_(db=at(7)) == INVALID
    if not torch.cuda.is_available():
        assert fwd_(at(0)) == DEVICE and fwd_(at(1)) == DEVICE and bwd_() == DEVICE
        for i in (0, 1, 4):
            assert bwd_(dx=at(i)) == DEVICE and bwd_(dgate=at(i)) == DEVICE


def test_batches_beyond_a_launch(C):
    """2^32 threads: the scan has 256 for every 1024 state elements of a segment, a step 256 for 64 columns."""
    def size(trees, hkv, d):
        b = GroupBatch(np.arange(trees + 1), np.zeros(trees + 1), [0], hkv, hkv, d)
        return C.augtree_linear_workspace_size(b.ref, 0)
    assert size(65535, 16, 128) > 0 and size(65536, 16, 128) == 0
    assert size(65536 * 4 - 1, 16, 64) > 0 and size(65536 * 4, 16, 64) == 0

    def step(rows):
        return C.augtree_linear_step(rows, 128, 128, 128, 0.1, np.ones(128, np.float32).ctypes.data_as(ctypes.c_void_p),
                                     None, at(3), at(4), rows, at(0), None, at(0), at(5), None)
    assert step(65535) == INVALID and step(65536) == UNSUPPORTED


def test_empty_responses_overlap_nothing(C):
    """A batch without branches may come with response pointers, of no bytes, into other tensors."""
    plain, d = GroupBatch([0, 10], [0, 0], [0], 4, 2, 64), dec(0.9, 0.9)
    inner = ctypes.c_void_p(at(0).value + 64)
    if not torch.cuda.is_available():
        assert fwd(C, plain, d, o_r=inner) == DEVICE


def test_python_refusals():
    b = GroupBatch(*GOOD, 4, 2, 64)
    z = lambda t, h: torch.zeros(t, h, 64, dtype=torch.bfloat16)
    x = (z(25, 4), z(25, 2), z(25, 2), z(20, 4), z(20, 2), z(20, 2))
    with pytest.raises(ValueError, match="no CPU path"):
        group_linear_attention(*x, b, [0.9, 0.9])
    with pytest.raises(ValueError, match="no CPU path"):
        api.linear_fwd(b, [0.9, 0.9], *x)
    with pytest.raises(ValueError, match="no CPU path"):
        api.linear_step(*x[:3], [0.9, 0.9], torch.zeros(25, 2, 64, 64))
    with pytest.raises(ValueError, match="no CPU path"):
        head_norm(x[0])
    with pytest.raises(ValueError, match="shape"):
        group_linear_attention(*x, b, [0.9])
    with pytest.raises(ValueError, match="constant"):
        group_linear_attention(*x, b, torch.tensor([0.9, 0.9], requires_grad=True))
    with pytest.raises(ValueError, match="constant"):
        group_linear_attention(*x, b, 0.9, state=torch.zeros(2, 2, 64, 64, requires_grad=True))
    with pytest.raises(ValueError, match="activation"):
        head_norm(x[0], activation="relu")
    with pytest.raises(ValueError, match="cu_branch"):
        api.linear_workspace_size(GroupBatch([0, 10, 25], [0, 3], [0, 5, 12, 20], 4, 2, 64))
    for ws in (torch.zeros(64), torch.zeros(64, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError, match="uint8"):
            api._want_ws(ws, "ws")


def test_block_cuts_follow_from_the_tree():
    """Workspaces grow with the batch, and a batch of two trees needs what its trees need on their own (its states are
    the sum of theirs)."""
    def states(trees, backward):
        cu = lambda v: np.concatenate([[0], np.cumsum(v)])
        b = GroupBatch(cu([p for p, _ in trees]), cu([len(r) for _, r in trees]), cu([x for _, r in trees for x in r]), 8,
                       8, 128)
        return api.linear_workspace_size(b, backward)
    a, c = [(5000, [700, 3])], [(40, [9000])]
    state = 8 * 128 * 128 * 4
    for backward in (False, True):
        both, one, two = states(a + c, backward), states(a, backward), states(c, backward)
        assert both > max(one, two) and abs(both - one - two) < state  # the tables differ by alignment only
