"""The paged KV cache forms no gradients and takes no tangents, and says so for every tensor that could ask for one (the
checks run before anything is enqueued: no GPU needed)."""
from types import SimpleNamespace

import pytest
import torch
from torch.autograd import forward_ad

from paper_2609_33133_amd import api

ROWS, HQ, HKV, PAGES, PAGE, D = 3, 4, 2, 5, 16, 64


class Reached(Exception):
    """A call went past the checks of its arguments."""


class FakeOn:
    """api._On for host tensors: the library is not reached."""

    def __init__(self, tensors, stream=None):
        pass

    def __enter__(self):
        raise Reached

    def __exit__(self, *exc):
        pass


@pytest.fixture(autouse=True)
def _host_tensors(monkeypatch):
    monkeypatch.setattr(api, "_On", FakeOn)
    monkeypatch.setattr(api, "_need", lambda *a: None)  # (it asks for device tensors)


def args(fp8):
    z = lambda h: torch.zeros(ROWS, h, D, dtype=torch.bfloat16)
    cache = lambda: torch.zeros(PAGES, HKV, PAGE, D).to(torch.float8_e4m3fn if fp8 else torch.bfloat16)
    a = dict(q=z(HQ), k=z(HKV), v=z(HKV), o=z(HQ), lse=torch.zeros(HQ, ROWS), k_cache=cache(), v_cache=cache())
    if fp8:
        a.update(k_scale=torch.ones(HKV), v_scale=torch.ones(HKV))
    return a


def call(name, a):
    pages = SimpleNamespace(num_pages=PAGES, page_size=PAGE)
    plan = SimpleNamespace(data=None, rows=ROWS, hq=HQ, hkv=HKV, pages=pages)
    scales = dict(k_scale=a.get("k_scale"), v_scale=a.get("v_scale"))
    if name == "cache_write":
        return api.cache_write(a["k"], a["v"], a["k_cache"], a["v_cache"], plan, **scales)
    return api.paged_fwd(a["q"], a["k_cache"], a["v_cache"], plan, o=a["o"], lse=a["lse"], **scales)


CASES = ([("cache_write", n) for n in ("k", "v", "k_cache", "v_cache", "k_scale", "v_scale")]
         + [("paged_fwd", n) for n in ("q", "k_cache", "v_cache", "k_scale", "v_scale", "o", "lse")])


@pytest.mark.parametrize("name,which", CASES)
def test_tensors_that_ask_for_a_gradient_are_refused(name, which):
    fp8 = which.endswith("scale")
    a = args(fp8)
    with pytest.raises(Reached):
        call(name, a)
    a[which].requires_grad_(True)
    with pytest.raises(ValueError, match=name + " forms no gradient.*no_grad"):
        call(name, a)
    with torch.no_grad(), pytest.raises(Reached):
        call(name, a)
    with torch.inference_mode(), pytest.raises(Reached):
        call(name, a)


@pytest.mark.parametrize("grad", [True, False])
@pytest.mark.parametrize("name,which", CASES)
def test_dual_tensors_are_refused(name, which, grad):
    fp8 = which.endswith("scale")
    a = args(fp8)
    with forward_ad.dual_level(), torch.set_grad_enabled(grad):
        a[which] = forward_ad.make_dual(a[which], torch.ones_like(a[which]))
        with pytest.raises(ValueError, match=name + ".*tangent"):
            call(name, a)
