"""Attention of new tokens over the pages of a cache in 4 bits, against the definition in 64 bits at bounds derived in paged.attend_bound."""
import ctypes as C

import numpy as np
import pytest
import torch

from paged import TD, attend_and_check, rows
from paged4 import Filled4
from test_gpu_attn_paged import CASES, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", CASES)
def test_against_the_definition(name, dtype, d):
    q_len, keys, hq, hk, page, group = CASES[name]
    f = Filled4(keys, hk, d, page, dtype, seed=len(name))
    attend_and_check(f, queries(sum(q_len), hq, d, dtype), q_len, group)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_empty_and_padded(dtype):
    f = Filled4([30, 0, 5, 64, 0], 2, 128, 16, dtype)
    got = attend_and_check(f, queries(3 + 4 + 9 + 5, 4, 128, dtype), [3, 4, 9, 0, 0], group=1)
    assert (got[3:7] == 0).all() and (got[7:11] == 0).all()
    attend_and_check(f, queries(3 + 4 + 9 + 5, 4, 128, dtype), [3, 4, 9, 0, 0], group=0)
    attend_and_check(f, queries(6, 4, 128, dtype), [0, 0, 6, 0, 0], group=4)


@pytest.mark.parametrize("n", [1, 20, 90, 400])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_keys_at_all(dtype, n):
    f = Filled4([0, 0], 2, 64, 32, dtype)
    for width in (1, 0):
        f.table = f.table[:, :width].contiguous()
        for group in (0, 1):
            assert (attend_and_check(f, queries(2 * n, 4, 64, dtype), [n, n], group, max_kv=500) == 0).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("most", [1, 3, 12])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_padded_batch_of_long_sequences(dtype, most, d):
    """Places that bring no new token or have no keys, between sequences long enough to be split; then a launch made for 24000 keys (a plan, in bf16)."""
    q_len, keys = [0, 1, 0, 0, most, 1, 1, 0, 2], [2500, 2600, 0, 17, 3001, 0, 4100, 2100, 129]
    f = Filled4(keys, 2, d, 16, dtype)
    for group in (0, 1):
        attend_and_check(f, queries(sum(q_len) + 2, 4, d, dtype), q_len, group)
    f.table = torch.cat([f.table, torch.full((9, 1500 - f.table.shape[1]), -1, dtype=torch.int32, device="cuda")], dim=1).contiguous()
    for group in (0, 1):
        attend_and_check(f, queries(sum(q_len) + 2, 4, d, dtype), q_len, group, max_kv=24000)


@pytest.mark.parametrize("q_each", [1, 5])
def test_captured_and_replayed_for_other_lengths(q_each):
    keys = [21000, 5, 0, 16000, 129, 9000, 1, 300, 21000, 4000]
    f = Filled4(keys, 2, 64, 64, "bf16")
    q = queries(10 * q_each, 4, 64, "bf16")
    attend_and_check(f, q, [q_each] * 10, group=1)
    start = torch.arange(11, dtype=torch.int32, device="cuda") * q_each
    first = torch.tensor(keys, dtype=torch.int32, device="cuda")
    lens, out = first.clone(), torch.zeros_like(q)
    f.cache.attend(q, start, lens, f.table, q_each, 21000, causal_group=1, out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f.cache.attend(q, start, lens, f.table, q_each, 21000, causal_group=1, out=out)
    for now in (first, first // 2, torch.clamp(first, max=40), first * 0, first):
        lens.copy_(now)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, f.cache.attend(q, start, now.contiguous(), f.table, q_each, 21000, causal_group=1))


# new tokens, keys, query heads, key heads, head_dim, dtype, group -> rows of a block, whether the keys are cut into ranges
KINDS = {
    "few rows": ([1], [300], 4, 4, 128, "bf16", 0, 16, False),
    "few rows in ranges": ([1], [4000], 8, 2, 64, "bf16", 0, 16, True),
    "32 rows": ([4, 4], [900, 500], 16, 2, 128, "bf16", 1, 32, True),
    "32 rows of 64 in runs": ([20] * 6, [9000, 8000, 9000, 500, 9000, 8999], 9, 9, 64, "bf16", 1, 32, True),
    "128 rows": ([300], [700], 3, 3, 64, "bf16", 0, 128, None),
    "128 rows of 128": ([130], [700], 2, 2, 128, "bf16", 1, 128, None),
    "256 rows": ([512], [4000], 128, 128, 128, "bf16", 0, 256, None),
    "fp32, 64 rows": ([90], [700], 2, 2, 128, "f32", 1, 64, None),
    "fp32, few rows": ([1], [700], 2, 2, 64, "f32", 1, 16, None),
}


@pytest.mark.parametrize("name", KINDS)
def test_every_kind_of_block_with_every_key(name):
    """The kind of block is the one meant; every key counts once: with equal scores and values that say which key they are of, the sum is the mean."""
    from paper_2505_21070_amd import binding as B
    q_len, keys, hq, hk, d, dtype, group, qb, cut = KINDS[name]
    page = 64
    need = [-(-n // page) for n in keys]
    cache = B.KVCache.empty(sum(need) + 1, hk, page, d, dtype, fp4=True)
    table = torch.zeros((len(keys), max(need)), dtype=torch.int32)
    at = 1
    for b, n in enumerate(keys):
        table[b, : need[b]] = torch.arange(at, at + need[b]).to(torch.int32)
        slot = torch.arange(at * page, at * page + n, dtype=torch.int32)
        at += need[b]
        # channel c of key i is 1 where i % d == c, and all keys are zero
        v = torch.zeros((n, hk, d))
        v[torch.arange(n), :, torch.arange(n) % d] = 1.0
        cache.write(torch.zeros((n, hk, d), dtype=TD[dtype], device="cuda"), v.to(TD[dtype]).cuda(), slot.cuda())
    kind = (C.c_int32 * 4)()
    cfg = B._PACK_ATTN(hq, len(keys), max(q_len), max(keys), table.shape[1], group, d ** -0.5)
    B._lib.dp_attn_paged_route(cache._desc, cfg, C.c_int64(sum(q_len)), kind)
    assert kind[0] == qb and (cut is None or (kind[1] > 1 or kind[3] > 0) == cut), list(kind)
    start = np.concatenate([[0], np.cumsum(q_len)])
    i32 = lambda x: torch.tensor(list(map(int, x)), dtype=torch.int32, device="cuda")   # noqa: E731
    out = cache.attend(queries(sum(q_len), hq, d, dtype), i32(start), i32(keys), table.cuda(), max(q_len), max(keys), causal_group=group).float().cpu()
    for b, n in enumerate(keys):
        seen = torch.full((q_len[b],), n) if group == 0 else n - q_len[b] + 1 + torch.arange(q_len[b])
        count = ((seen[:, None] - torch.arange(d)[None, :] + d - 1) // d).clamp(min=0).double()
        want = (count / seen[:, None]).float()[:, None, :]
        got = out[start[b]: start[b + 1]]
        # weights are equal and exact, sums of ones exact; one division and its rounding, one of the result's.  One key lost or twice is 1/count off, 1/141 at least
        assert ((got - want).abs() <= want * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -22) * 1.01).all()


@pytest.mark.parametrize("rows_", [1, 20, 200])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_is_not_seen_does_not_count(dtype, rows_):
    """Groups that are NaN (a value of them was not finite) in keys and values that a query does not see; the pages' free places are NaN (Filled4)."""
    keys = 210

    def change(b, k, v):
        big = torch.finfo(TD[dtype]).max
        for at, kv, vv in ((keys - 1, big, float("inf")), (keys - 2, float("nan"), -float("inf")), (keys - 3, -big, float("nan"))):
            if at >= keys - rows_ + 1:
                k[at, :, 3], v[at, :, 40] = kv, vv
        if rows_ > 5:
            v[keys - 5, :, 7] = -float("inf")
    f = Filled4([keys, keys], 2, 64, 16, dtype, change=change)
    q = queries(2 * rows_, 2, 64, dtype)
    attend_and_check(f, q, [rows_] * 2, group=1)


@pytest.mark.parametrize("n", [1, 30, 300])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_nan_group_reaches_who_sees_it(dtype, n):
    """A value's group of NaN reaches its 32 channels of every query that sees it, in a whole tile as at a border; a key's reaches all channels."""
    def change(b, k, v):
        v[10, :, 33] = float("nan")
        if b == 1:
            k[200, :, 5] = float("inf")
    keys = [n + 500, n + 300]
    f = Filled4(keys, 2, 128, 32, dtype, change=change)
    got = attend_and_check(f, queries(2 * n, 4, 128, dtype), [n] * 2, group=1)
    assert torch.isnan(got[:n, :, 32:64]).all() and torch.isfinite(got[:n, :, :32]).all() and torch.isnan(got[n:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bad_pages(dtype):
    """Pages outside the pool do not exist; numbers that are far off are not followed."""
    keys, page = 330, 16
    f = Filled4([keys] * 2, 2, 64, page, dtype)
    exists = [np.ones(keys, bool), np.ones(keys, bool)]
    for b, p, bad in ((0, 3, -1), (0, 20, 2 ** 31 - 1), (1, 0, -2 ** 31), (1, 7, f.cache.n_pages)):
        f.table[b, p] = bad
        exists[b][p * page: (p + 1) * page] = False
    for n in (1, 40, 200):
        attend_and_check(f, queries(2 * n, 4, 64, dtype), [n, n], group=1, exists=exists)
        attend_and_check(f, queries(2 * n, 4, 64, dtype), [n, n], group=0, exists=exists)


def test_strides_and_in_place():
    f = Filled4([100, 40], 2, 128, 16, "bf16")
    wide = rows(torch.Generator().manual_seed(3), 12, 9, 128, "bf16", 1.3).cuda()
    q = wide[:, 1:7]
    start = torch.tensor([0, 9, 12], dtype=torch.int32, device="cuda")
    lens = torch.tensor([100, 40], dtype=torch.int32, device="cuda")
    apart = f.cache.attend(q.contiguous(), start, lens, f.table, 9, 100, causal_group=1)
    assert torch.equal(f.cache.attend(q, start, lens, f.table, 9, 100, causal_group=1), apart)
    assert f.cache.attend(q, start, lens, f.table, 9, 100, causal_group=1, out=q) is q and torch.equal(q, apart)
