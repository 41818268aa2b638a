"""A batch keeps its own offsets: kernels of a later call (a backward) index tensors by them (CPU only)."""
import numpy as np
import pytest

from paper_2609_33133_amd import api
from paper_2609_33133_amd.api import GroupBatch

CU = ([0, 10, 25], [0, 2, 3], [0, 5, 12, 20])


def test_a_batch_does_not_follow_the_callers_arrays():
    cu = [np.array(c, np.int32) for c in CU]
    b = GroupBatch(*cu, 4, 2, 64)
    size = api.linear_workspace_size(b)
    for c in cu:
        c[1:] *= 1000  # the caller's next batch
    for kept, field, want in zip((b.cu_prompt, b.cu_branch, b.cu_resp),
                                 (b.struct.cu_prompt, b.struct.cu_branch, b.struct.cu_resp), CU):
        assert kept.tolist() == want and [field[i] for i in range(len(want))] == want
    assert (b.tp, b.tr) == (25, 20) and api.linear_workspace_size(b) == size


@pytest.mark.parametrize("name", ["cu_prompt", "cu_branch", "cu_resp"])
def test_a_batch_is_not_refilled_in_place(name):
    """Its row counts are taken once, so other offsets are another batch."""
    b = GroupBatch(*CU, 4, 2, 64)
    with pytest.raises(ValueError, match="read-only"):
        getattr(b, name)[1] = 7
    assert api.linear_workspace_size(b) > 0
