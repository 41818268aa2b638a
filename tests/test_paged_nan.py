"""What NaN and infinities reach in the paged KV cache. On the CPU: its sources are compiled with NaN honoured (a compiler
that may assume there is none leaves results that are NaN undefined)."""
import os

import pytest

from paper_2609_33133_amd import build


@pytest.mark.parametrize("src", ["paged.hip", "attn_paged.hip"])
def test_the_caches_kernels_honour_nan(src):
    assert os.path.exists(os.path.join(build.CSRC, src))
    flags = build.hip_flags(os.path.join(build.CSRC, src))
    assert not [f for f in flags if f in ("-fno-honor-nans", "-fno-honor-infinities", "-ffinite-math-only", "-ffast-math",
                                          "-Ofast")]
