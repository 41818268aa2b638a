"""Refusals of the paged KV cache's entry points (no GPU: every call fails before anything is enqueued)."""
import ctypes

import pytest
import torch

from paper_2609_33133_amd import _lib, api

OK, INVALID, UNSUPPORTED, MISALIGNED, WORKSPACE, DEVICE = range(6)
BIG = 1 << 40


@pytest.fixture(scope="module")
def C():
    return _lib.load()


def at(i, off=0):
    """Address i of tensors that lie apart."""
    return ctypes.c_void_p((1 << 50) + (i << 44) + off)


def pages(**kw):
    f = dict(num_seqs=5, max_pages=7, num_pages=40, page_size=64, table=at(0), length=at(1), parent=at(2), free_pages=at(3),
             free_state=at(4))
    f.update(kw)
    return _lib.Pages(*(f[n] for n, _ in _lib.Pages._fields_))


def plan(C, p=None, rows=9, hq=8, hkv=2, new=at(5), length=at(6), state=at(7), plan=at(8), n=BIG):
    p = pages() if p is None else p
    return C.augtree_page_plan(ctypes.byref(p), new, rows, hq, hkv, length, state, plan, n, None)


PAGE = 2 * 64 * 128 * 2


def write(C, p=None, rows=9, hq=8, hkv=2, d=128, plan=at(8), k=at(9), v=at(10), kind=0, kc=at(11), ks=PAGE, vc=at(12),
          vs=PAGE, k_scale=None, v_scale=None):
    p = pages() if p is None else p
    return C.augtree_cache_write(ctypes.byref(p), plan, rows, hq, hkv, d, k, v, kind, kc, ks, vc, vs, k_scale, v_scale, None)


def attend(C, p=None, rows=9, hq=8, hkv=2, d=128, scale=0.1, plan=at(8), q=at(9), kind=0, kc=at(11), ks=PAGE, vc=at(12),
           vs=PAGE, k_scale=None, v_scale=None, o=at(13), lse=at(14), ws=at(15), n=BIG):
    p = pages() if p is None else p
    return C.augtree_paged_fwd(ctypes.byref(p), plan, rows, hq, hkv, d, scale, q, kind, kc, ks, vc, vs, k_scale, v_scale, o,
                               lse, ws, n, None)


CALLS = (plan, write, attend)


def test_valid_calls_reach_the_device_check(C):
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    for call in CALLS:
        assert call(C) == DEVICE
    assert plan(C, length=at(1), state=at(4)) == DEVICE                # in place
    assert plan(C, pages(parent=None)) == DEVICE
    both = dict(kc=at(11), vc=at(11, PAGE), ks=2 * PAGE, vs=2 * PAGE)  # two halves of one tensor
    assert write(C, **both) == DEVICE and attend(C, **both) == DEVICE
    both.update(kc=both["vc"], vc=both["kc"])
    assert write(C, **both) == DEVICE and attend(C, **both) == DEVICE
    assert write(C, kind=1, k_scale=at(16), v_scale=at(17)) == DEVICE
    assert attend(C, lse=None) == DEVICE


def test_no_rows_are_no_work(C):
    assert write(C, rows=0, k=None, v=None) == OK
    assert attend(C, rows=0, q=None, o=None, ws=None, n=0) == OK


@pytest.mark.parametrize("kw,code", [
    (dict(num_seqs=0), INVALID), (dict(num_seqs=-3), INVALID), (dict(max_pages=0), INVALID), (dict(num_pages=0), INVALID),
    (dict(page_size=8), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED), (dict(page_size=512), UNSUPPORTED),
    (dict(page_size=0), UNSUPPORTED), (dict(page_size=-64), UNSUPPORTED),
    (dict(max_pages=1 << 25), UNSUPPORTED), (dict(num_pages=1 << 25), UNSUPPORTED), (dict(num_seqs=(1 << 20) + 1), UNSUPPORTED),
    (dict(table=None), INVALID), (dict(table=at(0, 4)), MISALIGNED),
])
def test_descriptors(C, kw, code):
    assert plan(C, pages(**kw)) == code, C.augtree_last_error()
    if "table" not in kw:
        assert write(C, pages(**kw)) == code
        assert C.augtree_page_plan_size(ctypes.byref(pages(**kw)), 9, 8, 2) == 0
        assert C.augtree_page_plan_offset(ctypes.byref(pages(**kw)), 9, 8, 2, 0) == -1
        assert C.augtree_paged_workspace_size(ctypes.byref(pages(**kw)), 9, 8, 2, 128) == 0
    assert attend(C, pages(**kw)) == code
    assert C.augtree_last_error().decode() != ""


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), INVALID), (dict(hq=0), INVALID), (dict(hkv=0), INVALID), (dict(hq=9), UNSUPPORTED),
    (dict(hq=65538), UNSUPPORTED), (dict(rows=1 << 28), UNSUPPORTED),
])
def test_sizes(C, kw, code):
    for call in CALLS:
        assert call(C, **kw) == code, C.augtree_last_error()


@pytest.mark.parametrize("kw,code", [
    (dict(new=None), INVALID), (dict(length=None), INVALID), (dict(state=None), INVALID), (dict(plan=None), WORKSPACE),
    (dict(n=100), WORKSPACE), (dict(new=at(5, 4)), MISALIGNED), (dict(plan=at(8, 8)), MISALIGNED),
    (dict(length=at(2)), INVALID), (dict(length=at(1, 16)), INVALID), (dict(plan=at(5)), INVALID), (dict(plan=at(0)), INVALID),
    (dict(state=at(5)), INVALID), (dict(length=at(4)), INVALID),
    (dict(p=dict(length=None)), INVALID), (dict(p=dict(free_pages=None)), INVALID), (dict(p=dict(free_state=None)), INVALID),
    (dict(p=dict(parent=at(2, 4))), MISALIGNED), (dict(p=dict(free_pages=at(0))), INVALID),
])
def test_plan_arguments(C, kw, code):
    kw = dict(kw, p=pages(**kw["p"])) if "p" in kw else kw
    assert plan(C, **kw) == code, C.augtree_last_error()


CACHES = [
    (dict(d=96), UNSUPPORTED), (dict(kind=2), INVALID), (dict(kind=-1), INVALID), (dict(kc=None), INVALID),
    (dict(vc=None), INVALID), (dict(kc=at(11, 8)), MISALIGNED), (dict(ks=PAGE - 16), INVALID), (dict(vs=0), INVALID),
    (dict(vs=-PAGE), INVALID), (dict(ks=PAGE + 8), MISALIGNED), (dict(ks=1 << 41), INVALID),
    (dict(vc=at(11)), INVALID), (dict(vc=at(11, PAGE)), INVALID),                        # one after the other, or one inside
    (dict(vc=at(11, PAGE - 16), ks=2 * PAGE, vs=2 * PAGE), INVALID), (dict(vc=at(11, PAGE), ks=2 * PAGE, vs=3 * PAGE), INVALID),
    (dict(kind=1), INVALID), (dict(kind=1, k_scale=at(16)), INVALID), (dict(plan=None), INVALID), (dict(plan=at(8, 4)), MISALIGNED),
]


@pytest.mark.parametrize("kw,code", CACHES)
def test_caches(C, kw, code):
    assert write(C, **kw) == code, C.augtree_last_error()
    assert attend(C, **kw) == code, C.augtree_last_error()


@pytest.mark.parametrize("call,kw,code", [
    (write, dict(k=None), INVALID), (write, dict(v=at(10, 2)), MISALIGNED), (write, dict(k=at(11)), INVALID),
    (write, dict(v=at(12, PAGE)), INVALID), (write, dict(plan=at(12)), INVALID),
    (attend, dict(q=None), INVALID), (attend, dict(o=None), INVALID), (attend, dict(o=at(9)), INVALID),
    (attend, dict(o=at(11)), INVALID), (attend, dict(lse=at(13)), INVALID), (attend, dict(ws=at(13)), INVALID),
    (attend, dict(o=at(8)), INVALID), (attend, dict(o=at(0)), INVALID), (attend, dict(lse=at(14, 4)), MISALIGNED),
    (attend, dict(ws=None), WORKSPACE), (attend, dict(n=1000), WORKSPACE), (attend, dict(ws=at(15, 16)), MISALIGNED),
    (attend, dict(scale=0.0), INVALID), (attend, dict(scale=float("nan")), INVALID), (attend, dict(scale=float("inf")), INVALID),
])
def test_tensors(C, call, kw, code):
    assert call(C, **kw) == code, C.augtree_last_error()


def test_null_descriptor_and_fields(C):
    assert C.augtree_page_plan(None, at(5), 9, 8, 2, at(6), at(7), at(8), BIG, None) == INVALID
    assert C.augtree_page_plan_size(None, 9, 8, 2) == 0
    p = ctypes.byref(pages())
    fields = [C.augtree_page_plan_offset(p, 9, 8, 2, f) for f in range(4)]
    assert len(set(fields)) == 4 and min(fields) >= 0 and C.augtree_page_plan_offset(p, 9, 8, 2, 4) == -1
    assert max(fields) + 9 <= C.augtree_page_plan_size(p, 9, 8, 2) // 4
    assert C.augtree_page_plan_size(p, 0, 8, 2) > 0
    assert C.augtree_paged_workspace_size(p, 9, 8, 2, 80) == 0


def test_launches_have_room(C):
    """Items of many KV heads exceed a launch."""
    p = pages(num_seqs=1 << 20, max_pages=16, page_size=16)
    assert attend(C, p, rows=1 << 20, hq=1024, hkv=1024, d=64, ks=1 << 24, vs=1 << 24) == UNSUPPORTED


def test_python_refuses_host_tensors():
    t = lambda *s: torch.zeros(*s, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU tensor"):
        api.PageTable(t(2, 3), t(2), t(2), t(8), t(2), 64)
    with pytest.raises(ValueError, match="GPU tensor"):
        api.PageTable.empty(2, 3, 8, 64, device="cpu")
