"""The largest values of the types into codes of 8 bits and back: finite ones stay finite."""
import numpy as np
import pytest
import torch

from oracle import paged as O
from paged import TD, np64

pytestmark = pytest.mark.gpu
# where the codes of the highest power begin, end, and go over: 1.75, 1.875, 1.9375 and 2 times 2^127
VALUES = [1.75, 1.7578125, 1.8125, 1.875, 1.8984375, 1.9296875, 1.9375, 1.9453125, 1.984375]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_largest_values(dtype, d):
    from paper_2505_21070_amd import binding as B
    top = torch.finfo(TD[dtype]).max
    x = torch.zeros((len(VALUES) + 2, 1, d), dtype=TD[dtype])
    for i, m in enumerate(VALUES):
        x[i, 0, i], x[i, 0, 30], x[i, 0, 31] = m * 2.0 ** 127, -m * 2.0 ** 126, 2.0 ** 112
    x[-2, 0, 5], x[-2, 0, 6], x[-2, 0, 7] = top, -top, float("inf")
    x[-1] = -top
    cache = B.KVCache.empty(2, 1, 16, d, dtype, True)
    slot = torch.arange(x.shape[0], dtype=torch.int32, device="cuda")
    cache.write(x.cuda(), -x.cuda(), slot)
    ref, e = O.fp8_rows(np64(x))
    assert e.max() == 120
    k, v = cache.read(slot)
    for got, want in ((k, ref), (v, -ref)):
        assert np.array_equal(np64(got), want, equal_nan=True)
        assert (torch.isfinite(got.float().cpu()) | ~torch.isfinite(x.float())).all()
    # and to a query that sees the one key alone
    one = torch.ones((1, 1, d), dtype=TD[dtype], device="cuda")
    cache.write(one * 0, x[-1:].cuda(), slot[:1])
    out = cache.attend(one, *(torch.tensor(t, dtype=torch.int32, device="cuda") for t in ([0, 1], [1], [[0]])), 1, 1)
    assert (out == -240.0 * 2.0 ** 120).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_normalised_keys_as_large(dtype):
    """Keys that gains bring there, written in one pass with the norm."""
    from paper_2505_21070_amd import binding as B
    top = torch.finfo(TD[dtype]).max
    cache = B.KVCache.empty(1, 1, 16, 64, dtype, True)
    x = torch.ones((1, 1, 64), dtype=TD[dtype], device="cuda")
    gain = torch.full((64,), top, dtype=TD[dtype], device="cuda")
    slot = torch.zeros(1, dtype=torch.int32, device="cuda")
    cache.write_qkv(x, x, x, gain * 0, gain, torch.zeros((1, 3), dtype=torch.int32, device="cuda"), slot, eps=0.0)
    assert (cache.read(slot)[0] == 240.0 * 2.0 ** 120).all()
