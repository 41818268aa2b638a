"""More of the paged KV cache on the GPU."""
import pytest
import torch

from paper_2609_33133_amd import _lib, api

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("seqs", [40, 1025, 2500, 4096])
def test_new_tokens_past_32_bits_are_refused(seqs):
    """Each sequence asks for more tokens than the plan has rows; of 2500 and more their sum passes 2^31."""
    rows = 1 << 20
    pages = api.PageTable.empty(seqs, rows // 256, 30, 256)
    new = torch.full((seqs,), rows if seqs > 2048 else 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    keep = [t.clone() for t in (pages.table, pages.length, pages.free_pages, pages.free_state)]
    plan = api.page_plan(pages, new, rows, 2, 1)
    assert int(plan.status) & (_lib.PAGES_ROWS | _lib.PAGES_SHORT) == _lib.PAGES_ROWS | _lib.PAGES_SHORT
    for a, b in zip(keep, (pages.table, pages.length, pages.free_pages, pages.free_state)):
        assert torch.equal(a, b)
    assert (plan.slots == -1).all() and (plan.cu_rows == 0).all()
