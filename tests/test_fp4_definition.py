"""What include/dualparal.h says of 4-bit codes in so many words, by the oracle; and how large the products' workspaces get (no GPU)."""
import numpy as np
import pytest

import test_paged_refusals as P
from oracle import fp4 as F
from paper_2505_21070_amd import binding as B


@pytest.mark.parametrize("power", [-100, 0, 37, 124])
def test_ties_and_the_last_code(power):
    x = np.zeros((2, 32))
    x[:, 0] = 7.0                                            # the factor is 1
    x[0, 1:9], x[1, 1:9] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.0 + 2.0 ** -40], [-6.0, -5.0, 6.5, 7.0, -3.5, 4.999, 2.4999, 0.2501]
    code, byte = F.encode(x * 2.0 ** power)
    assert (byte == power + 127).all()
    want = [[6, 0, 1, 1, 2, 2, 4, 4, 6], [6, -6, -4, 6, 6, -4, 4, 2, 0.5]]
    assert (F.decode(code, byte)[:, :9] == np.array(want) * 2.0 ** power).all()


def test_the_ends_of_the_range():
    assert (F.encode(np.zeros((1, 32)))[1] == 27).all()
    for top, byte, reads in ((7 * 2.0 ** 125, 252, 6 * 2.0 ** 125), (7.96875 * 2.0 ** 125, 252, 6 * 2.0 ** 125), (7.03125 * 2.0 ** 124, 252, 4 * 2.0 ** 125), (2.0 ** -130, 27, 0.0)):
        code, got = F.encode(np.full((1, 32), top))
        assert (got == byte).all() and (F.decode(code, got) == reads).all()


def test_workspaces_of_products():
    """Ranges are of tiles of 128 rows and 80 tokens at most, and of 768 blocks at most: so many sums."""
    worst = 0
    for out in (1, 100, 1001, 5120, 8801, 13824, 98304, 1 << 20, 1 << 24):
        for in_ in (32, 992, 5120, 8992, 13824, 1 << 20):
            for n in (1, 16, 17, 33, 49, 64, 65, 80, 81, 100, 333, 1000, 1 << 16):
                if out * in_ <= 1 << 36 and n * out <= 1 << 35:
                    for dtype in (B.DP_BF16, B.DP_F32):
                        worst = max(worst, P.L.dp_linear_fp4_workspace_bytes(bytes(B.Fp4Matrix(out, in_, dtype, P.AT, None)), n))
    assert 0 < worst <= 768 * 128 * 80 * 4
