"""Attention of new tokens over the pages of a cache, against the definition in 64 bits at bounds derived in paged.attend_bound."""
import numpy as np
import pytest
import torch

from paged import Filled, TD, attend_and_check, rows

pytestmark = pytest.mark.gpu


def queries(n, heads, d, dtype, seed=1):
    return rows(torch.Generator().manual_seed(seed), n, heads, d, dtype, 1.3).cuda()


# new tokens, keys, query heads, key heads, page, group
CASES = {
    "one token, one key": ([1], [1], 1, 1, 16, 0),
    "one token": ([1], [517], 12, 12, 16, 1),
    "tokens of several lengths": ([1, 1, 1, 1, 1], [1, 16, 17, 64, 301], 8, 2, 16, 1),
    "shared heads, a few tokens": ([3, 1, 2], [40, 129, 65], 24, 3, 32, 1),
    "one token of many shared heads": ([1, 1], [130, 700], 64, 1, 64, 0),
    "a chunk, everything seen": ([37], [101], 3, 3, 16, 0),
    "a chunk of tokens, causal": ([70, 5, 64], [70, 133, 64], 4, 2, 32, 1),
    "a chunk by frames": ([60, 45], [150, 45], 4, 4, 16, 15),
    "frames longer than a tile": ([200, 100], [300, 100], 2, 1, 64, 100),
    "a chunk that fills tiles": ([256], [512], 2, 2, 128, 0),
    "more than a tile of rows": ([300, 1, 140], [420, 33, 140], 2, 2, 64, 0),
    "more than a tile of rows, causal": ([300, 17], [420, 333], 6, 2, 64, 1),
    "odd shared heads": ([50], [90], 15, 5, 16, 7),
    "one page larger than the sequence": ([9], [20], 2, 2, 4096, 1),
    "many keys": ([2], [5000], 4, 4, 256, 0),
}


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("store", ["bf16", "bf16 in 8 bits", "f32", "f32 in 8 bits"])
@pytest.mark.parametrize("name", CASES)
def test_against_the_definition(name, store, d):
    q_len, keys, hq, hk, page, group = CASES[name]
    dtype = store.split()[0]
    f = Filled(keys, hk, d, page, dtype, "8" in store, seed=len(name))
    attend_and_check(f, queries(sum(q_len), hq, d, dtype), q_len, group)


STORES = [("bf16", False), ("bf16", True), ("f32", False), ("f32", True)]


@pytest.mark.parametrize("dtype,fp8", STORES)
def test_empty_and_padded(dtype, fp8):
    """Sequences without new tokens, without keys, with fewer keys than new tokens (their first queries see nothing), and rows of no sequence."""
    f = Filled([30, 0, 5, 64, 0], 2, 128, 16, dtype, fp8)
    got = attend_and_check(f, queries(3 + 4 + 9 + 5, 4, 128, dtype), [3, 4, 9, 0, 0], group=1)
    assert (got[3:7] == 0).all() and (got[7:11] == 0).all()
    attend_and_check(f, queries(3 + 4 + 9 + 5, 4, 128, dtype), [3, 4, 9, 0, 0], group=0)
    attend_and_check(f, queries(6, 4, 128, dtype), [0, 0, 6, 0, 0], group=4)


@pytest.mark.parametrize("n", [1, 20, 90, 400])
@pytest.mark.parametrize("dtype,fp8", STORES)
def test_no_keys_at_all(dtype, fp8, n):
    """Whole calls without a key: with a table that is not looked at, and without one."""
    f = Filled([0, 0], 2, 64, 32, dtype, fp8)
    for width in (1, 0):
        f.table = f.table[:, :width].contiguous()
        for group in (0, 1):
            got = attend_and_check(f, queries(2 * n, 4, 64, dtype), [n, n], group, max_kv=500)
            assert (got == 0).all()


@pytest.mark.parametrize("most", [1, 3, 12])
@pytest.mark.parametrize("dtype,fp8", STORES)
def test_padded_batch_of_long_sequences(dtype, fp8, most):
    """A batch some of whose places bring no new token, or have no keys, between sequences long enough to be split."""
    q_len, keys = [0, 1, 0, 0, most, 1, 1, 0, 2], [2500, 2600, 0, 17, 3001, 0, 4100, 2100, 129]
    f = Filled(keys, 2, 128, 16, dtype, fp8)
    for group in (0, 1):
        attend_and_check(f, queries(sum(q_len) + 2, 4, 128, dtype), q_len, group)
    # the same in a launch made for sequences of 24000 keys
    f.table = torch.cat([f.table, torch.full((9, 1500 - f.table.shape[1]), -1, dtype=torch.int32, device="cuda")], dim=1).contiguous()
    for group in (0, 1):
        attend_and_check(f, queries(sum(q_len) + 2, 4, 128, dtype), q_len, group, max_kv=24000)


@pytest.mark.parametrize("q_each", [1, 5])
@pytest.mark.parametrize("fp8", [False, True])
def test_sequences_of_very_different_lengths(fp8, q_each, dtype="bf16"):
    """Tokens of ten sequences of 0 to 21000 keys; then the call captured, and replayed for other lengths, which have to leave the results of eager calls."""
    keys = [21000, 5, 0, 16000, 129, 9000, 1, 300, 21000, 4000]
    f = Filled(keys, 2, 64, 64, dtype, fp8)
    q = queries(10 * q_each, 4, 64, dtype)
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


@pytest.mark.parametrize("dtype,fp8", STORES)
def test_bounds_larger_than_the_sequences(dtype, fp8):
    """A launch made for far more new tokens and keys than there are, as one captured for all sizes is."""
    q_len = [1, 0, 3, 40]
    f = Filled([5, 70, 300, 140], 2, 64, 32, dtype, fp8)
    f.table = torch.cat([f.table, torch.full((4, 500), -1, dtype=torch.int32, device="cuda")], dim=1).contiguous()
    for max_q in (40, 1000, 1 << 24):
        attend_and_check(f, queries(44, 4, 64, dtype), q_len, 1, max_q=max_q, max_kv=2 ** 31 - 1 - 65536)
    attend_and_check(f, queries(4, 4, 64, dtype), [1, 0, 1, 2], 1, max_q=8, max_kv=2 ** 31 - 1 - 65536)


@pytest.mark.parametrize("dtype,fp8", STORES)
def test_sequences_that_share_pages(dtype, fp8):
    """Pages in several tables, and one page twice in a table: reading does not mind."""
    f = Filled([192], 2, 128, 64, dtype, fp8)
    k, v = f.k[0], f.v[0]
    own = f.table[0].tolist()
    f.table = torch.tensor([own, [own[1], own[1], own[0]], own], dtype=torch.int32, device="cuda")
    twice = np.concatenate([np.arange(64, 128), np.arange(64, 128), np.arange(64)])
    f.keys = [192, 170, 100]
    f.k, f.v = [k, k[twice[:170]], k[:100]], [v, v[twice[:170]], v[:100]]
    for n in (1, 90):
        attend_and_check(f, queries(3 * n, 4, 128, dtype), [n] * 3, group=1)


@pytest.mark.parametrize("rows_", [1, 20, 200])
@pytest.mark.parametrize("dtype,fp8", STORES)
def test_what_is_not_seen_does_not_count(dtype, fp8, rows_):
    """Keys and values that a query does not see hold NaN, infinities and the type's largest values; the pages' free places hold NaN (Filled)."""
    keys = 210

    def change(b, k, v):
        big = torch.finfo(TD[dtype]).max
        for at, kv, vv in ((keys - 1, big, float("inf")), (keys - 2, float("nan"), -float("inf")), (keys - 3, -big, float("nan")),
                           (keys - 5, float("inf"), big)):
            if at >= keys - rows_ + 1:
                k[at], v[at] = kv, vv
            if b == 1 and at == keys - 5 and rows_ > 5:
                v[at, :, 7] = -float("inf")
    if rows_ == 1:
        f = Filled([keys], 2, 64, 16, dtype, fp8)
        attend_and_check(f, queries(1, 2, 64, dtype), [1], group=1)
        return
    f = Filled([keys, keys], 2, 64, 16, dtype, fp8, change=change)
    q = queries(2 * rows_, 2, 64, dtype)
    start = [0, rows_, 2 * rows_]
    out = f.cache.attend(q, torch.tensor(start, dtype=torch.int32, device="cuda"), torch.tensor([keys] * 2, dtype=torch.int32, device="cuda"), f.table,
                         rows_, keys, causal_group=1)
    clean = Filled([keys, keys], 2, 64, 16, dtype, fp8)
    ref = clean.cache.attend(q, torch.tensor(start, dtype=torch.int32, device="cuda"), torch.tensor([keys] * 2, dtype=torch.int32, device="cuda"),
                             clean.table, rows_, keys, causal_group=1)
    for b in range(2):
        assert torch.equal(out[start[b]: start[b + 1] - 5], ref[start[b]: start[b + 1] - 5])
        assert not torch.isfinite(out[start[b + 1] - 1]).all()


@pytest.mark.parametrize("rows_", [3, 40, 300])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_values_that_are_seen(dtype, rows_):
    """An infinite value reaches the queries that see it, and its channel alone."""
    def change(b, k, v):
        v[330, 0, 5], v[331, 1, 9], v[332, 0, 5] = float("inf"), float("nan"), -float("inf")
    f = Filled([340], 2, 128, 32, dtype, False, change=change)
    attend_and_check(f, queries(rows_, 2, 128, dtype), [rows_], group=1)


@pytest.mark.parametrize("rows_", [2, 30, 150])
@pytest.mark.parametrize("dtype,fp8", STORES)
def test_scores_far_apart(dtype, fp8, rows_):
    """The largest score comes last, first, and in the middle, by far more than a weight's exponent holds."""
    def change(b, k, v):
        k[(0, 299, 150)[b]] *= 60.0
        k[(0, 299, 150)[b]] += 20.0
    f = Filled([300] * 3, 1, 128, 64, dtype, fp8, change=change)
    q = queries(3 * rows_, 1, 128, dtype).abs()
    attend_and_check(f, q, [rows_] * 3, group=0)
    attend_and_check(f, q, [rows_] * 3, group=0, scale=3.0)


@pytest.mark.parametrize("rows_", [2, 30, 150, 500])
@pytest.mark.parametrize("dtype,fp8", STORES)
def test_large_values_behind_small_scores(dtype, fp8, rows_):
    """Scores rise by about 60 after the first keys, which is 2^86 in weights that still refer to them, and the values lie around 2^50: each fits
    fp32, their product does not."""
    def change(b, k, v):
        k[64:] += 5.0
        v *= 2.0 ** 50
    f = Filled([700], 2, 128, 64, dtype, fp8, change=change)
    attend_and_check(f, queries(rows_, 2, 128, dtype).abs(), [rows_], group=0)


@pytest.mark.parametrize("rows_", [2, 30, 150])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_of_minus_infinity(dtype, rows_):
    """Keys whose score is -inf weigh nothing, a row of nothing but them gives zeros."""
    def change(b, k, v):
        k[: (90, 200)[b], 0, 3] = -float("inf")
    f = Filled([200, 200], 1, 64, 16, dtype, False, change=change)
    q = queries(2 * rows_, 1, 64, dtype).abs() + 0.5
    got = attend_and_check(f, q.to(TD[dtype]), [rows_] * 2, group=0)
    assert (got[rows_:] == 0).all() and (got[:rows_] != 0).any()


@pytest.mark.parametrize("rows_", [1, 40, 150])
@pytest.mark.parametrize("dtype,fp8", STORES)
def test_pages_that_do_not_exist(dtype, fp8, rows_):
    f = Filled([150, 150], 2, 64, 16, dtype, fp8)
    exists = [np.ones(150, bool) for _ in range(2)]
    for b, at, bad in ((0, 2, -1), (0, 9, 10 ** 6), (1, 0, -2 ** 31), (1, 5, f.cache.n_pages), (1, 6, 2 ** 31 - 1)):
        f.table[b, at] = bad
        exists[b][at * 16: at * 16 + 16] = False
    attend_and_check(f, queries(2 * rows_, 4, 64, dtype), [rows_] * 2, group=1, exists=exists)
    # a table that ends before the keys do
    narrow = f.table[:, :7].contiguous()
    f.table = narrow
    for e in exists:
        e[7 * 16:] = False
    attend_and_check(f, queries(2 * rows_, 4, 64, dtype), [rows_] * 2, group=1, exists=exists)


@pytest.mark.parametrize("rows_", [1, 40, 150])
@pytest.mark.parametrize("dtype,fp8", STORES)
def test_bounds_smaller_than_the_sequences(dtype, fp8, rows_):
    f = Filled([150, 90], 1, 128, 16, dtype, fp8)
    q = queries(2 * rows_, 2, 128, dtype)
    exists = [np.arange(n) < 77 for n in f.keys]
    attend_and_check(f, q, [rows_] * 2, group=1, exists=exists, max_kv=77)
    if rows_ == 1:
        return
    start = torch.tensor([0, rows_, 2 * rows_], dtype=torch.int32, device="cuda")
    lens = torch.tensor(f.keys, dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 7.0)
    f.cache.attend(q, start, lens, f.table, rows_ - 9, 150, causal_group=1, out=out)
    whole = f.cache.attend(q, start, lens, f.table, rows_, 150, causal_group=1)
    for b in range(2):
        assert (out[(b + 1) * rows_ - 9: (b + 1) * rows_] == 7.0).all()
        d = (out[b * rows_: (b + 1) * rows_ - 9].float() - whole[b * rows_: (b + 1) * rows_ - 9].float()).abs().max()
        assert d <= 2.0 ** -5                                  # one softmax, cut differently at most


@pytest.mark.parametrize("dtype,fp8", STORES)
def test_arrays_that_make_no_sense(dtype, fp8):
    """Starts and lengths outside what there is are cut to it."""
    f = Filled([40, 50, 60], 1, 64, 16, dtype, fp8)
    q = queries(20, 1, 64, dtype)
    out = torch.full_like(q, 7.0)
    f.cache.attend(q, torch.tensor([-5, 4, 2, 99], dtype=torch.int32, device="cuda"), torch.tensor([-3, 50, 2 ** 31 - 1], dtype=torch.int32, device="cuda"),
                   f.table, 30, 64, out=out)
    assert torch.isfinite(out[:2].float()).all() and (out[:2] == 0).all()          # rows 0 .. 3 see no key (sequence 0) until sequence 2 takes 2 .. 19
    f.cache.data.view(torch.uint8).fill_(0)
    f.cache.attend(q, torch.tensor([0, 20, 10, -1], dtype=torch.int32, device="cuda"), torch.tensor([40, -1, 7], dtype=torch.int32, device="cuda"),
                   f.table, 20, 64, out=out)
    assert (out == 0).all()


@pytest.mark.parametrize("rows_", [1, 33, 270])
@pytest.mark.parametrize("dtype,fp8", STORES)
def test_strides_and_in_place(dtype, fp8, rows_):
    f = Filled([280], 2, 64, 32, dtype, fp8)
    plain = queries(rows_, 6, 64, dtype)
    ref = attend_and_check(f, plain, [rows_], group=1)
    start = torch.tensor([0, rows_], dtype=torch.int32, device="cuda")
    lens = torch.tensor([280], dtype=torch.int32, device="cuda")
    for make in (lambda: torch.zeros((rows_, 10, 64), dtype=TD[dtype], device="cuda")[:, 2:8],
                 lambda: torch.zeros((6, rows_, 64), dtype=TD[dtype], device="cuda").transpose(0, 1)):
        q, out = make(), make()
        q.copy_(plain)
        assert torch.equal(f.cache.attend(q, start, lens, f.table, rows_, 280, causal_group=1, out=out), ref)
        assert torch.equal(out, ref)
        assert torch.equal(f.cache.attend(q, start, lens, f.table, rows_, 280, causal_group=1, out=q), ref) and torch.equal(q, ref)
    one = plain[:1].expand(rows_, 6, 64)                           # the same query for every new token
    attend_and_check(f, one, [rows_], group=1)


@pytest.mark.parametrize("dtype,fp8", STORES)
def test_a_pool_beyond_32_bits(dtype, fp8):
    """A sequence whose pages lie before and behind the 2^32nd byte of the pool."""
    from paper_2505_21070_amd import binding as B
    hk, d, page = 4, 128, 256
    per_page = 2 * hk * page * d * (1 if fp8 else 2 if dtype == "bf16" else 4)
    n_pages = (1 << 32) // per_page + 9
    f = Filled([700], hk, d, page, dtype, fp8)
    big = B.KVCache.empty(n_pages, hk, page, d, dtype, fp8)
    to = torch.tensor([n_pages - 1, 3, n_pages - 4], device="cuda")
    src = f.table[0].long()
    big.data.view(torch.uint8)[to] = f.cache.data.view(torch.uint8)[src]
    if fp8:
        big.scales[to] = f.cache.scales[src]
    f.cache, f.table = big, to.to(torch.int32)[None].contiguous()
    for n in (1, 70):
        attend_and_check(f, queries(n, 4, d, dtype), [n], group=1)


def test_many_sequences():
    keys = [(37 * i) % 90 + 1 for i in range(300)]
    f = Filled(keys, 1, 64, 16, "bf16", True)
    attend_and_check(f, queries(300, 2, 64, "bf16"), [1] * 300, group=1)


@pytest.mark.parametrize("dtype,fp8", STORES)
def test_results_are_the_same_each_time(dtype, fp8):
    f = Filled([3000, 2000], 2, 128, 64, dtype, fp8)
    for n in (1, 130):
        q = queries(2 * n, 4, 128, dtype)
        args = (q, torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda"), torch.tensor(f.keys, dtype=torch.int32, device="cuda"), f.table, n, 3000)
        first = f.cache.attend(*args)
        for _ in range(3):
            assert torch.equal(f.cache.attend(*args), first)
