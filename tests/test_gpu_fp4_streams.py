"""The operators on 4 bits and the gated norm on named streams, on two at once, in graphs, and where offsets pass 32 bits."""
import pytest
import torch

from paged import TD, positions, rows
from test_gpu_paged_streams import pool_of

pytestmark = pytest.mark.gpu
HQ, HK, D, PAGE = 4, 2, 128, 32
RANGES = {"bf16": (2, 1001, 13824), "f32": (2, 1000, 13824)}        # tokens, outputs, inputs of products whose inputs are cut into ranges


def matrix(out, in_, dtype, seed=3):
    from paper_2505_21070_amd import binding as B
    gen = torch.Generator().manual_seed(seed)
    w = torch.randn((out, in_), generator=gen).to(TD[dtype]).cuda()
    return B.Linear4.pack(w, torch.randn(out, generator=gen).to(TD[dtype]).cuda())


def tokens(n, in_, dtype, seed):
    return torch.randn((n, in_), generator=torch.Generator().manual_seed(seed)).to(TD[dtype]).cuda()


def filled(keys, dtype, seqs):
    """A cache in 4 bits with `seqs` sequences of up to so many keys, and what an attend of one token each takes behind the queries."""
    from paper_2505_21070_amd import binding as B
    each = -(-keys // PAGE)
    cache = B.KVCache.empty(seqs * each, HK, PAGE, D, dtype, fp4=True)
    slot = torch.arange(seqs * each * PAGE, dtype=torch.int32, device="cuda")
    gen = torch.Generator().manual_seed(9)
    cache.write(*[rows(gen, slot.shape[0], HK, D, dtype).cuda() for _ in range(2)], slot)
    lens = torch.arange(seqs, dtype=torch.int32, device="cuda") * 700 % keys + 1
    lens[0] = keys
    table = torch.arange(seqs * each, dtype=torch.int32, device="cuda").view(seqs, each)
    return cache, (torch.arange(seqs + 1, dtype=torch.int32, device="cuda"), lens, table, 1, keys)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_memory_is_of_the_stream_that_writes_it(dtype, monkeypatch):
    from paper_2505_21070_amd import binding as B
    n, out, in_ = RANGES[dtype]
    m, x = matrix(out, in_, dtype), tokens(n, in_, dtype, 1)
    cache, args = filled(4000, dtype, 6)
    gen = torch.Generator().manual_seed(2)
    q, k, v = [rows(gen, 40, h, D, dtype).cuda() for h in (HQ, HK, HK)]
    pos, g = positions(40, gen).cuda(), torch.ones(D, dtype=TD[dtype], device="cuda")
    slot, q1, r = torch.arange(40, dtype=torch.int32, device="cuda"), q[:6].contiguous(), tokens(5, 512, dtype, 4)
    works = []
    for name, at in (("dp_linear_fp4", 7), ("dp_attn_paged", 8)):
        def spy(*a, original=getattr(B._lib, name), at=at):
            works.append(a[at])
            return original(*a)
        monkeypatch.setattr(B._lib, name, spy)

    def results(stream):
        codes, scales = B.pack_fp4(r, stream=stream)
        return [m.forward(x, stream=stream), cache.attend(q1, *args, stream=stream), cache.write_qkv(q, k, v, g, g, pos, slot, stream=stream),
                *cache.read(slot, stream=stream), *B.gated_norm(r.float(), r, stream=stream), codes, scales, B.Linear4(codes, scales, dtype=dtype, stream=stream).laid]
    side, here = torch.cuda.Stream(), torch.cuda.current_stream().cuda_stream
    torch.cuda.synchronize()
    for stream, pool in ((None, here), (side, side.cuda_stream), (None, here), (side, side.cuda_stream)):
        del works[:]
        got = results(stream)
        torch.cuda.synchronize()
        assert [pool_of(t.data_ptr()) for t in got] == [pool] * len(got)
        assert len(works) == 2 and None not in works and [pool_of(w) for w in works] == [pool] * 2
        del got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_products_on_two_streams_in_turn(dtype):
    """Calls of one size, the current stream's and a named one's, nobody waiting, workspaces (and half of the results) dropped while kernels run: all as alone."""
    n, out, in_ = RANGES[dtype]
    m, xs = matrix(out, in_, dtype), [tokens(n, in_, dtype, i) for i in range(2)]
    want = [m.forward(x, act="silu") for x in xs]
    assert not torch.equal(*want)
    torch.cuda.synchronize()
    side, got = torch.cuda.Stream(), []
    for i in range(40):
        got.append((0, m.forward(xs[0], act="silu")))
        got.append((1, m.forward(xs[1], act="silu", stream=side)))
        if i % 2:
            del got[-2:]
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[s]) for s, y in got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 200])
def test_two_graphs_of_one_matrix(n, dtype):
    """Two graphs with workspaces of their own, replayed at the same time on two streams, and eager calls of another number of tokens between."""
    _, out, in_ = RANGES[dtype]
    m, xs, other = matrix(out, in_, dtype), [tokens(n, in_, dtype, i) for i in range(4)], tokens(3, in_, dtype, 8)
    want, beside = [m.forward(x, act="gelu") for x in xs], m.forward(other)
    now, streams, graphs, ys = [xs[0].clone(), xs[1].clone()], [torch.cuda.Stream(), torch.cuda.Stream()], [], []
    torch.cuda.synchronize()
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            ys.append(m.forward(now[i], act="gelu"))
    for turn in range(6):
        for i in range(2):
            now[i].copy_(xs[(turn + i) % 4])
        torch.cuda.synchronize()
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
        eager = m.forward(other)
        torch.cuda.synchronize()
        assert torch.equal(eager, beside) and all(torch.equal(ys[i], want[(turn + i) % 4]) for i in range(2)), turn


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_named_streams_inside_a_capture(dtype):
    """Write, attend, product and norm on a stream that a capture has branched to: every replay gives the eager bits."""
    from paper_2505_21070_amd import binding as B
    cache, args = filled(6000, dtype, 1)
    m = matrix(1024, HQ * D, dtype)
    gen = torch.Generator().manual_seed(1)
    steps = [[rows(gen, 1, h, D, dtype).cuda() for h in (HQ, HK, HK)] for _ in range(2)]
    slot = torch.tensor([5999], dtype=torch.int32, device="cuda")
    x, g = tokens(1, 1024, dtype, 5), torch.ones((1, 1024), device="cuda") * 0.25

    def step(q, k, v, stream=None):
        cache.write(k, v, slot, stream=stream)
        y = m.forward(cache.attend(q, *args, stream=stream).view(1, HQ * D), stream=stream)
        return B.gated_norm(x, y, gate=g, norm="rms", stream=stream)
    want = [step(*s) for s in steps]
    assert not torch.equal(want[0][1], want[1][1])
    now = [t.clone() for t in steps[0]]
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        res = step(*now, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        kept = [t.clone() for t in res]
        del res
    for i in (0, 1, 1, 0):
        for t, s in zip(now, steps[i]):
            t.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(kept[0], want[i][0]) and torch.equal(kept[1], want[i][1])
        again = step(*steps[1])
        torch.cuda.synchronize()
        assert torch.equal(again[1], want[1][1])


@pytest.mark.parametrize("dtype,n", [("bf16", 1100), ("f32", 600)])
def test_rows_of_tokens_beyond_32_bits(n, dtype):
    """Inputs 2^21 elements apart and outputs 2^22: the last ones lie beyond 2^32 bytes from the first."""
    in_, out = 256, 72
    m = matrix(out, in_, dtype)
    x = tokens(n, in_, dtype, 6)
    want = m.forward(x)
    wide = torch.empty(((n - 1) << 21) + in_, dtype=TD[dtype], device="cuda").as_strided((n, in_), (1 << 21, 1))
    wide.copy_(x)
    y = torch.empty(((n - 1) << 22) + out, dtype=TD[dtype], device="cuda").as_strided((n, out), (1 << 22, 1))
    m.forward(wide, out=y)
    assert torch.equal(y, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norms_of_rows_beyond_32_bits(dtype):
    from paper_2505_21070_amd import binding as B
    n, d, far = 1300, 264, 1 << 21
    x, y = tokens(n, d, "f32", 6), tokens(n, d, dtype, 7)
    group = torch.arange(n, dtype=torch.int32, device="cuda") % 3
    gate = torch.randn((3, d), generator=torch.Generator().manual_seed(1)).cuda()
    want = B.gated_norm(x, y, gate=gate, group=group)
    spread = lambda t: torch.empty(((n - 1) * far) + d, dtype=t.dtype, device="cuda").as_strided((n, d), (far, 1)).copy_(t)   # noqa: E731
    xs, ys = spread(x), spread(y)
    got = B.gated_norm(xs, ys, gate=gate, group=group, x_out=xs, out=ys)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
