"""Ends of the ranges that the paged operators take, and the definitions there (no GPU)."""
import numpy as np
import pytest

from paper_2505_21070_amd import binding as B
from test_paged_refusals import attend, attn, cache, refused


@pytest.mark.parametrize("scale", [2.4e38, 3.0e38, float(np.finfo(np.float32).max)])
def test_scales_that_softmax_in_powers_of_two_does_not_hold(scale):
    """scale * log2(e) beyond fp32: every score would be infinite or, times 0, no number."""
    refused(attend(a=attn(scale=scale)), "dp_attn_paged")
    assert B._lib.dp_attn_paged_workspace_bytes(cache(), attn(scale=scale), 7) == 0
    assert attend(a=attn(scale=2.3e38, max_q=0)) == B.DP_OK

