"""The attention of blocks of 256 rows (halves half a round apart, stages of whole tiles, one range of keys or several) and of 128 rows in several ranges, against
64 bits; the kind of block of each call is stated and looked up.  Lengths are below the bounds that size the launch, so that one shape meets no, one, two and
more whole tiles, with all remainders that change the way through the kernel."""
import numpy as np
import pytest
import torch

from paged import Filled, TD, attend_and_check
from paged_exact import Pages, check, route

pytestmark = pytest.mark.gpu
D = 128
# key heads, shared, new tokens, bound of the keys, group -> rows of a block, ranges, keys of a range
ONE = (64, 8, 65, 2400, 0), (256, 1, 2432)
CAUSAL = (64, 8, 1024, 9600, 1), (256, 1, 9600)
FRAMES = (64, 8, 1024, 9600, 390), (256, 1, 9600)
RANGES = (8, 8, 254, 9000, 0), (256, 4, 2304)
SMALL = (2, 4, 100, 6000, 0), (128, 12, 512)
SMALL_CAUSAL = (4, 1, 130, 5000, 1), (128, 10, 512)


def made(shape, fp8, keys, **kw):
    (hk, shared, n, bound, group), kind = shape
    assert route("bf16", D, hk * shared, hk, 1, n, n, bound, group)[:3] == kind
    f = Pages([keys], hk, D, 16 if fp8 else 64, "bf16", fp8, **kw)
    assert f.table.shape[1] <= -(-bound // f.cache.page_tokens)
    # the launch is sized by the bound alone if the table is as wide
    wide = torch.full((1, -(-bound // f.cache.page_tokens)), -1, dtype=torch.int32, device="cuda")
    wide[:, : f.table.shape[1]] = f.table
    f.table = wide
    q = torch.randn((n, hk * shared, D), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") * 1.3
    return f, q.to(torch.bfloat16), n, bound, group


def heads_of(q, k):
    """k query heads, the first and last of a key head among them."""
    return sorted({0, q.shape[1] - 1} | {(i * q.shape[1]) // k for i in range(k)} | {(i * q.shape[1]) // k + 7 for i in range(k) if q.shape[1] > 8 * k})


def test_the_exact_form_is_the_definition():
    """paged_exact against the definition, by one call that both check."""
    f = Pages([301], 2, 64, 16, "f32", False)
    q = torch.randn((70, 4, 64), device="cuda")
    got = f.attend(q, [70], group=7)
    check(f, q, got, [70], group=7)
    g = Filled([301], 2, 64, 16, "f32", False)
    g.cache, g.table, g.k, g.v = f.cache, f.table, [t.double().cpu().numpy() for t in f.k], [t.double().cpu().numpy() for t in f.v]
    assert torch.equal(attend_and_check(g, q, [70], group=7), got)


@pytest.mark.parametrize("fp8", [False, True])
def test_one_range(fp8):
    f, q, n, bound, group = made(ONE, fp8, 2400)
    for keys in (0, 1, 40, 63, 64, 65, 127, 128, 129, 191, 192, 193, 255, 256, 257, 320, 333, 384, 2399, 2400):
        got = f.attend(q, [n], [keys], group, max_kv=bound)
        check(f, q, got, [n], [keys], group, None if keys in (129, 2399) else heads_of(q, 6))


@pytest.mark.parametrize("fp8", [False, True])
def test_several_ranges(fp8):
    f, q, n, bound, group = made(RANGES, fp8, 9000)
    for keys in (1, 64, 2303, 2304, 2305, 2367, 2368, 2400, 2432, 2433, 4607, 4608, 4609, 4700, 6911, 6912, 6913, 7042, 9000):
        got = f.attend(q, [n], [keys], group, max_kv=bound)
        check(f, q, got, [n], [keys], group, heads_of(q, 4))


@pytest.mark.parametrize("shape", [CAUSAL, FRAMES], ids=["tokens", "frames"])
@pytest.mark.parametrize("fp8", [False, True])
def test_borders(fp8, shape):
    f, q, n, bound, group = made(shape, fp8, 1500)
    for keys in (300, 1024, 1100, 1500):
        got = f.attend(q, [n], [keys], group, max_kv=bound)
        check(f, q, got, [n], [keys], group, heads_of(q, 5))


@pytest.mark.parametrize("group", [0, 1])
@pytest.mark.parametrize("fp8", [False, True])
def test_several_sequences_in_ranges(fp8, group):
    """Chunks of unequal length over sequences that end in the first, second and third range, beside one without keys and one without new tokens."""
    hk, shared, bound, part = 32, 4, 121571, 12160
    q_len, keys = [62, 40, 0, 33, 26], [12161, 300, 5000, 24400, 0]
    assert route("bf16", D, hk * shared, hk, 5, 161, 62, bound, 1) == (256, 10, part, 0)
    assert route("bf16", D, hk * shared, hk, 5, 161, 62, bound, 0)[0] == 256
    f = Pages(keys, hk, D, 64, "bf16", fp8)
    f.table = torch.cat([f.table, torch.full((5, -(-bound // 64) - f.table.shape[1]), -1, dtype=torch.int32, device="cuda")], dim=1).contiguous()
    q = (torch.randn((161 + 3, hk * shared, D), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)) * 1.3).to(torch.bfloat16)
    out = torch.full_like(q, 7.0)
    f.attend(q, q_len, group=group, max_kv=bound, out=out)
    check(f, q, out, q_len, group=group, heads=heads_of(q, 4))
    assert (out[161:] == 7.0).all() and (out[135: 161] == 0).all()


@pytest.mark.parametrize("shape", [ONE, RANGES, SMALL], ids=["256", "256 ranges", "128 ranges"])
@pytest.mark.parametrize("fp8", [False, True])
def test_pages_that_do_not_exist(fp8, shape):
    keys = 2400
    f, q, n, bound, group = made(shape, fp8, keys)
    exists, page = torch.ones(keys, dtype=torch.bool, device="cuda"), f.cache.page_tokens
    for at, bad in ((0, -1), (3, 10 ** 6), (keys // page - 1, f.cache.n_pages)):
        f.table[0, at] = bad
        exists[at * page: (at + 1) * page] = False
        got = f.attend(q, [n], [keys], group, max_kv=bound)
        check(f, q, got, [n], [keys], group, heads_of(q, 3), [exists])


@pytest.mark.parametrize("shape", [ONE, RANGES, SMALL, SMALL_CAUSAL], ids=["256", "256 ranges", "128 ranges", "128 ranges, causal"])
@pytest.mark.parametrize("fp8", [False, True])
def test_references_that_are_raised(fp8, shape):
    """Scores that rise by far more than 2^100 after a range's first keys, in some heads alone, and values whose weighted sums leave fp32."""
    def change(b, k, v):
        k[70:, ::2] += 5.0
        k[1000:, 1] += 9.0
        v[:, -1] *= 2.0 ** 50
    f, q, n, bound, group = made(shape, fp8, 2400, change=change)
    q = q.abs()
    for keys in (200, 1100, 2390):
        got = f.attend(q, [n], [keys], group, max_kv=bound)
        check(f, q, got, [n], [keys], group, heads_of(q, 4))


@pytest.mark.parametrize("shape", [ONE, RANGES, SMALL], ids=["256", "256 ranges", "128 ranges"])
def test_values_that_are_not_finite(shape):
    """In whole tiles and at the end, at keys of ordinary and of vanishing weight."""
    def change(b, k, v):
        k[100] -= 30.0
        v[100, 0, 5], v[333, 1, 7], v[333, 0, 9], v[2389, 0, 11], v[2389, -1, 11] = float("inf"), -float("inf"), float("nan"), float("inf"), -float("inf")
    f, q, n, bound, group = made(shape, False, 2400, change=change)
    q = q.abs()
    for keys in (101, 400, 2390):
        got = f.attend(q, [n], [keys], group, max_kv=bound)
        shared = q.shape[1] // f.hk
        check(f, q, got, [n], [keys], group, [0, shared, q.shape[1] - 1])


@pytest.mark.parametrize("keys", [511, 512, 513, 575, 576, 700, 1023, 1024, 1025, 1153, 4999])
@pytest.mark.parametrize("shape", [SMALL, SMALL_CAUSAL], ids=["everything seen", "causal"])
@pytest.mark.parametrize("fp8", [False, True])
def test_blocks_of_128_rows_in_ranges(fp8, shape, keys):
    f, q, n, bound, group = made(shape, fp8, keys)
    check(f, q, f.attend(q, [n], group=group, max_kv=bound), [n], group=group)


@pytest.mark.parametrize("shape", [ONE, RANGES], ids=["256", "256 ranges"])
@pytest.mark.parametrize("fp8", [False, True])
def test_the_same_bits_each_time_and_replayed(fp8, shape):
    f, q, n, bound, group = made(shape, fp8, 2400)
    start = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    lens = torch.tensor([2400], dtype=torch.int32, device="cuda")
    want = {keys: f.attend(q, [n], [keys], group, max_kv=bound) for keys in (2400, 2305, 130)}
    for _ in range(5):
        assert torch.equal(f.attend(q, [n], [2400], group, max_kv=bound), want[2400])
    out = torch.zeros_like(q)
    f.cache.attend(q, start, lens, f.table, n, bound, causal_group=group, out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f.cache.attend(q, start, lens, f.table, n, bound, causal_group=group, out=out)
    for keys in (2400, 130, 2305, 2400):
        lens.fill_(keys)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[keys])
        assert torch.equal(f.attend(q, [n], [130], group, max_kv=bound), want[130])
