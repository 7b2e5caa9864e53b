"""Infinite values that a query sees: whatever their keys' weights, in whatever tile they lie, they reach its result; keys whose score is -inf do not."""
import numpy as np
import pytest
import torch

from paged import Filled, TD, attend_and_check, rows

pytestmark = pytest.mark.gpu
INF, KEYS, LATE = float("inf"), 700, 697
# where the infinite values lie: in the first tile, in whole tiles, among the last keys, which are no whole tile
PLACES = (0, 40, 333, LATE)


def queries(n, d, dtype):
    return (rows(torch.Generator().manual_seed(1), n, 2, d, dtype, 1.3).abs() + 0.5).to(TD[dtype]).cuda()


def values(v, first=0):
    """+inf, -inf, both, NaN and NaN beside +inf, each in a channel of its own, at the places from the first-th on."""
    for i, p in enumerate(PLACES[first:]):
        v[p, 0, 3 + i], v[p, 1, 20 + i] = INF, -INF
        v[p, 0, 9], v[p, 1, 40] = (INF, -INF)[i % 2], float("nan") if i == 1 else INF


@pytest.mark.parametrize("levels", ["alike", "first the highest", "last the highest", "infinite ones the lowest", "rising", "falling"])
@pytest.mark.parametrize("d,rows_", [(64, 1), (128, 1), (64, 30), (128, 20), (64, 150), (128, 100)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_whatever_the_weights(dtype, d, rows_, levels):
    """Scores whose weights, next to the highest, are far below what fp32 holds (one level is 350 and more), or come to that by and by (60 a tile of 32)."""
    at = torch.arange(KEYS)
    level = {"alike": at * 0.0, "first the highest": (at < 5) * 1.0, "last the highest": (at >= KEYS - 2) * 1.0, "rising": at // 32 / 6.0, "falling": -(at // 32) / 6.0,
             "infinite ones the lowest": -sum(1.0 * (at == p) for p in PLACES)}[levels]

    def change(b, k, v):
        k += (level * (60.0 if d == 64 else 40.0)).to(k.dtype)[:, None, None]
        values(v)
    f = Filled([KEYS], 2, d, 16, dtype, False, change=change)
    q = queries(rows_, d, dtype)
    for group in (0, 1, 200):
        attend_and_check(f, q, [rows_], group=group)


@pytest.mark.parametrize("d,rows_", [(64, 1), (128, 30), (64, 150), (128, 100)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_keys_of_no_weight(dtype, d, rows_):
    """Keys whose score is -inf, with values that are not finite, in whole tiles and among the last keys."""
    def change(b, k, v):
        values(v, 0)
        for p in PLACES:
            k[p, :, 3] = -INF
    f = Filled([KEYS], 2, d, 16, dtype, False, change=change)
    got = attend_and_check(f, queries(rows_, d, dtype), [rows_], group=0)
    assert torch.isfinite(got.float()).all()


@pytest.mark.parametrize("seqs,keys", [(1, 6000), (60, 6000)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_joined_partial_results(dtype, seqs, keys):
    """Ranges and runs of keys whose part of the weight is nothing beside the others'."""
    lens = [keys] * seqs
    lens[1:] = [(700 * i) % keys + 1 for i in range(1, seqs)]

    def change(b, k, v):
        n = k.shape[0]
        k[n // 2:] += 60.0
        v[n // 7, 0, 5], v[n // 3, 1, 7] = INF, -INF
    f = Filled(lens, 2, 64, 16, dtype, False, change=change)
    attend_and_check(f, queries(seqs, 64, dtype), [1] * seqs, group=0)


@pytest.mark.parametrize("rows_", [2, 100])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_codes_that_stand_for_no_number(dtype, rows_):
    """What was not finite reads back as NaN from 8 bits, and reaches the queries that see it as such."""
    def change(b, k, v):
        k[600:] += 60.0
        v[333, 0, 5] = INF
    f = Filled([KEYS], 2, 64, 16, dtype, True, change=change)
    f.v[0][333, 0, 5] = np.nan
    got = attend_and_check(f, queries(rows_, 64, dtype), [rows_], group=0)
    assert torch.isnan(got[:, 0, 5]).all() and torch.isfinite(got[:, 1].float()).all()
