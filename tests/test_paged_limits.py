"""Ends of the ranges that the paged operators take, and the definitions there (no GPU)."""
import numpy as np
import pytest

from oracle import paged as O
from paper_2505_21070_amd import binding as B
from test_paged_refusals import attend, attn, cache, refused


@pytest.mark.parametrize("scale", [2.4e38, 3.0e38, float(np.finfo(np.float32).max)])
def test_scales_that_softmax_in_powers_of_two_does_not_hold(scale):
    """scale * log2(e) beyond fp32: every score would be infinite or, times 0, no number."""
    refused(attend(a=attn(scale=scale)), "dp_attn_paged")
    assert B._lib.dp_attn_paged_workspace_bytes(cache(), attn(scale=scale), 7) == 0
    assert attend(a=attn(scale=2.3e38, max_q=0)) == B.DP_OK


def test_codes_of_the_largest_values_stand_for_finite_ones():
    for top in (np.finfo(np.float32).max, 1.9375 * 2.0 ** 127, 1.75 * 2.0 ** 127 * (1 + 2.0 ** -20)):
        x = np.zeros((1, 64))
        x[0, :3] = top, -top, np.inf
        back, e = O.fp8_rows(x)
        assert e[0] == 120 and np.isfinite(np.float32(back[0, :2])).all() and np.isnan(back[0, 2])
        assert (np.abs(back[0, :2] - x[0, :2]) <= 2.0 ** -4 * top).all()


def test_infinite_values_and_their_weights():
    """exp(-2000) is 0 in 64 bits, but no weight is: the value reaches the result unless the score is -inf."""
    k = np.zeros((3, 1, 64))
    k[:, 0, 0] = 0.0, -2000.0, -np.inf
    v = np.ones((3, 1, 64))
    v[1, 0, 4], v[2, 0, 5] = np.inf, np.inf
    q = np.zeros((1, 1, 64))
    q[0, 0, 0] = 1.0
    for last, want in ((2, np.inf), (3, np.inf)):
        out, mean, _ = O.attend(q, [k[:last]], [v[:last]], [0, 1], [last], [np.ones(last, bool)], 0, 1.0, np.zeros_like(q))
        assert out[0, 0, 4] == want and out[0, 0, 5] == 1.0 and np.isfinite(mean).all()
