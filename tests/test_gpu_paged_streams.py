"""Results and workspaces of calls on a named stream: whose memory they are, and that calls of the same sizes on the current stream and on the named one
do not meet in it."""
import pytest
import torch

from paged import TD, positions, rows

pytestmark = pytest.mark.gpu
HQ, HK, D, PAGE = 4, 2, 128, 32


def pool_of(address):
    """The stream whose pool the memory at an address belongs to."""
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= address < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("no memory of the allocator")


def inputs(n, dtype, seed=5):
    gen = torch.Generator().manual_seed(seed)
    x = rows(gen, n, HQ + 2 * HK, D, dtype).cuda()
    return x[:, :HQ], x[:, HQ: HQ + HK], x[:, HQ + HK:], positions(n, gen).cuda()


def filled(keys, dtype="bf16", seqs=1):
    """A cache with `seqs` sequences of so many keys, and what an attend of one token each takes behind the queries."""
    from paper_2505_21070_amd import binding as B
    each = -(-keys // PAGE)
    cache = B.KVCache.empty(seqs * each, HK, PAGE, D, dtype)
    slot = torch.arange(seqs * each * PAGE, dtype=torch.int32, device="cuda")
    _, k, v, _ = inputs(slot.shape[0], dtype, 9)
    cache.write(k, v, slot)
    table = torch.arange(seqs * each, dtype=torch.int32, device="cuda").view(seqs, each)
    lens = torch.arange(seqs, dtype=torch.int32, device="cuda") * 700 % keys + 1
    lens[0] = keys
    return cache, (torch.arange(seqs + 1, dtype=torch.int32, device="cuda"), lens, table, 1, keys)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_memory_is_of_the_stream_that_writes_it(dtype, monkeypatch):
    """Each result and the workspace of a call on a named stream come from that stream's pool, those of a plain call from the current stream's, whatever blocks
    of their sizes are free there."""
    from paper_2505_21070_amd import binding as B
    n = 40
    q, k, v, pos = inputs(n, dtype)
    g = torch.ones(D, dtype=TD[dtype], device="cuda")
    cache, args = filled(4000, dtype, 6)
    slot = torch.arange(n, dtype=torch.int32, device="cuda")
    q1 = q[:6].contiguous()
    works = []
    original = B._lib.dp_attn_paged

    def spy(*a):
        works.append(a[8])
        return original(*a)
    monkeypatch.setattr(B._lib, "dp_attn_paged", spy)

    def results(stream):
        return [*B.qk_norm_rope(q, k, g, g, pos, stream=stream), cache.write_qkv(q, k, v, g, g, pos, slot, stream=stream), *cache.read(slot, stream=stream),
                cache.attend(q1, *args, stream=stream)]
    side = torch.cuda.Stream()
    here = torch.cuda.current_stream().cuda_stream
    side.wait_stream(torch.cuda.current_stream())
    for stream, pool in ((None, here), (side, side.cuda_stream), (None, here), (side, side.cuda_stream)):
        out = results(stream)
        torch.cuda.synchronize()
        assert [pool_of(t.data_ptr()) for t in out] == [pool] * len(out)
        assert works[-1] is not None and pool_of(works[-1]) == pool
        del out                                                      # free blocks of every size, in this pool
    # a stream that is the current one besides
    with torch.cuda.stream(side):
        assert pool_of(cache.read(slot, stream=side)[0].data_ptr()) == side.cuda_stream


@pytest.mark.parametrize("seqs,keys", [(1, 6000), (48, 6000)])
def test_the_same_call_on_two_streams_in_turn(seqs, keys):
    """Calls of one size on the current stream and on a named one, nobody waiting in between, each dropping its workspace (and half of them their result) while
    its kernels run: all as alone."""
    cache, args = filled(keys, "bf16", seqs)
    qs = [rows(torch.Generator().manual_seed(i), seqs, HQ, D, "bf16").cuda() for i in range(2)]
    want = [cache.attend(q, *args) for q in qs]
    assert not torch.equal(*want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = []
    for i in range(30):
        got.append((0, cache.attend(qs[0], *args)))
        got.append((1, cache.attend(qs[1], *args, stream=side)))
        if i % 2:
            del got[-2:]
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[s]) for s, y in got)


def test_a_result_read_here_is_not_handed_out_before(n=3000):
    """A result of a named stream, read on the current one behind a long queue and dropped at once: the named stream's next results take other memory until then."""
    cache, _ = filled(n)
    slot = torch.arange(n, dtype=torch.int32, device="cuda")
    want = cache.read(slot)[0]
    slow = torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    copies = []
    for i in range(4):
        k, v = cache.read(slot, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        for _ in range(20):
            slow = slow @ slow * 1e-4
        copies.append(k.clone())
        del k, v
        cache.read(torch.full_like(slot, -1), stream=side)              # zeros into whatever memory is free
    torch.cuda.synchronize()
    assert all(torch.equal(c, want) for c in copies)


@pytest.mark.parametrize("dtype,seqs", [("bf16", 1), ("bf16", 48), ("f32", 2)])
def test_a_named_stream_inside_a_capture(dtype, seqs):
    """A call on a stream that a capture has branched to: its result and workspace are the graph's, and every replay gives the eager bits."""
    cache, args = filled(6000, dtype, seqs)
    q, other = [rows(torch.Generator().manual_seed(i), seqs, HQ, D, dtype).cuda() for i in range(2)]
    want = cache.attend(q, *args), cache.attend(other, *args)
    now = q.clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        out = cache.attend(now, *args, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        kept = out.clone()
        del out
    for i in (0, 1, 1, 0):
        now.copy_((q, other)[i])
        graph.replay()
        between = cache.attend(other, *args)                         # eager work behind the replay
        torch.cuda.synchronize()
        assert torch.equal(kept, want[i]) and torch.equal(between, want[1])
