"""The operators around the paged cache as they are used together: the self-attention of several videos, block after block, out of one pool of pages;
with the call captured and replayed, and on streams other than the current one."""
import numpy as np
import pytest
import torch

from oracle import paged as O
from paged import HALF, NORM_UNITS, TD, U, attend_bound, np64, pair_length, positions, rows

pytestmark = pytest.mark.gpu
HQ, HK, D, PAGE, FRAME = 4, 2, 64, 32, 30


class Video:
    """What a serving program keeps of one video: its pages, how many tokens they hold, and (here) their keys and values."""

    def __init__(self):
        self.pages, self.tokens, self.k, self.v = [], 0, np.zeros((0, HK, D)), np.zeros((0, HK, D))


@pytest.mark.parametrize("dtype,fp8", [("bf16", False), ("bf16", True), ("f32", True)])
def test_blocks_of_several_videos(dtype, fp8):
    from paper_2505_21070_amd import binding as B
    gen = torch.Generator().manual_seed(11)
    cache = B.KVCache.empty(64, HK, PAGE, D, dtype, fp8)
    free = torch.randperm(64, generator=gen).tolist()
    videos = [Video() for _ in range(3)]
    gq, gk = [(torch.randn(D, generator=gen) * 0.2 + 1.2).to(TD[dtype]).cuda() for _ in range(2)]
    # frames that each video brings to a pass: blocks, a video that pauses, one token's worth of nothing
    for step, frames in enumerate([(2, 1, 0), (1, 3, 2), (2, 0, 1)]):
        n_new = [f * FRAME for f in frames]
        total = sum(n_new) + 3                                      # three rows of padding
        x = rows(gen, total, HQ + 2 * HK, D, dtype).cuda()
        q, k, v = x[:, :HQ], x[:, HQ: HQ + HK], x[:, HQ + HK:]
        pos = positions(total, gen).cuda()
        slots = []
        for vid, n in zip(videos, n_new):
            for i in range(vid.tokens, vid.tokens + n):
                if i // PAGE == len(vid.pages):
                    vid.pages.append(free.pop())
                slots.append(vid.pages[i // PAGE] * PAGE + i % PAGE)
        slots += [-1] * 3
        qn = cache.write_qkv(q, k, v, gq, gk, pos, torch.tensor(slots, dtype=torch.int32, device="cuda"))
        rk, rv = O.norm_rope(np64(k), np64(gk), pos.cpu().numpy(), 1e4, float(np.float32(1e-6))), np64(v)
        at = 0
        for vid, n in zip(videos, n_new):
            vid.k, vid.v, vid.tokens = np.concatenate([vid.k, rk[at: at + n]]), np.concatenate([vid.v, rv[at: at + n]]), vid.tokens + n
            at += n
        start = np.concatenate([[0], np.cumsum(n_new)]).astype(int)
        keys = [vid.tokens for vid in videos]
        table = torch.zeros((3, max(len(vid.pages) for vid in videos)), dtype=torch.int32)
        for b, vid in enumerate(videos):
            table[b, : len(vid.pages)] = torch.tensor(vid.pages, dtype=torch.int32)
        args = (torch.tensor(start, dtype=torch.int32, device="cuda"), torch.tensor(keys, dtype=torch.int32, device="cuda"), table.cuda(), max(n_new), max(keys))
        out = torch.full((total, HQ, D), 7.0, dtype=TD[dtype], device="cuda")
        cache.attend(qn, *args, causal_group=FRAME, out=out)
        assert (out[start[-1]:] == 7.0).all()
        # against the whole chain in 64 bits: what attention sees is what the pages hold and the queries as they were rounded
        slot_of = lambda vid: torch.tensor([vid.pages[i // PAGE] * PAGE + i % PAGE for i in range(vid.tokens)], dtype=torch.int32, device="cuda")
        kr, vr = zip(*[map(np64, cache.read(slot_of(vid))) for vid in videos])
        for b, vid in enumerate(videos):
            e = 2.0 ** -4 if fp8 else HALF[dtype]
            least = 2.0 ** -9 * 2.0 ** O.fp8_power(vid.k).astype(float)[..., None] if fp8 and vid.tokens else 0.0
            assert (np.abs(kr[b] - vid.k) <= np.maximum(e * np.abs(vid.k), least) * (1 + 2.0 ** -7) + NORM_UNITS * U * pair_length(vid.k)).all()
            assert np.array_equal(vr[b], O.fp8_rows(vid.v)[0] if fp8 and vid.tokens else vid.v)
        ref, mean_abs, score_abs = O.attend(np64(qn), kr, vr, start, keys, [np.ones(n, bool) for n in keys], FRAME, D ** -0.5, np.full(out.shape, 7.0))
        err = np.abs(np64(out) - ref)
        assert (err <= attend_bound(ref, mean_abs, score_abs, D, max(keys), dtype)).all(), step


def block(n, seed, dtype="bf16"):
    gen = torch.Generator().manual_seed(seed)
    return rows(gen, n, HQ + 2 * HK, D, dtype).cuda(), positions(n, gen).cuda()


@pytest.mark.parametrize("n,keys", [(1, 3000), (40, 700), (300, 2500)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_and_replayed(n, keys, dtype):
    """A layer's chain captured once; lengths, slots, tables and rows change between the replays, and eager calls of other sizes run in between.  Two graphs
    replayed in turn keep their results apart."""
    from paper_2505_21070_amd import binding as B
    width = keys // PAGE + 2
    cache = B.KVCache.empty(2 * width, HK, PAGE, D, dtype, True)
    fill, fpos = block(keys + 64, 3, dtype)
    table = torch.arange(width, dtype=torch.int32, device="cuda")[None].contiguous()
    every = torch.arange(keys + 64, dtype=torch.int32, device="cuda")[: width * PAGE]
    cache.write(fill[: every.shape[0], :HK], fill[: every.shape[0], HK: 2 * HK], every)
    g = torch.ones(D, dtype=TD[dtype], device="cuda")
    start = torch.tensor([0, n], dtype=torch.int32, device="cuda")

    def chain(x, pos, slot, lens, tab, out):
        q = cache.write_qkv(x[:, :HQ], x[:, HQ: HQ + HK], x[:, HQ + HK:], g, g, pos, slot)
        return cache.attend(q, start, lens, tab, n, keys, causal_group=1, out=out)

    sets = []
    for s in range(3):
        x, pos = block(n, 20 + s, dtype)
        length = keys - 40 * s
        sets.append((x, pos, every[length - n: length].clone(), torch.tensor([length], dtype=torch.int32, device="cuda"), table + width * (s == 2)))
    cache.data.view(torch.uint8)[width:] = cache.data.view(torch.uint8)[:width]
    cache.scales[width:] = cache.scales[:width]
    held = cache.data.view(torch.uint8).clone(), cache.scales.clone()

    def fresh():                                                     # a chain writes into the pages that the others see
        cache.data.view(torch.uint8).copy_(held[0])
        cache.scales.copy_(held[1])

    want = []
    for s in sets:
        fresh()
        want.append(chain(*s, torch.empty((n, HQ, D), dtype=TD[dtype], device="cuda")))
    graphs = []
    side = torch.cuda.Stream()
    for first in (0, 1):
        bufs = [t.clone() for t in sets[first]]
        out = torch.zeros((n, HQ, D), dtype=TD[dtype], device="cuda")
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            chain(*bufs, out)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            chain(*bufs, out)
        graphs.append((graph, bufs, out))
    for rep in range(4):
        for gi, (graph, bufs, out) in enumerate(graphs):
            pick = (rep + gi) % 3
            for b, t in zip(bufs, sets[pick]):
                b.copy_(t)
            fresh()
            graph.replay()
            cache.read(every[:5])                                    # eager work in between
            torch.cuda.synchronize()
            assert torch.equal(out, want[pick]), (rep, gi)
            fresh()
            eager = chain(*sets[(pick + 1) % 3], torch.empty_like(out))
            torch.cuda.synchronize()
            assert torch.equal(eager, want[(pick + 1) % 3])
    for (graph, bufs, out), pick in zip(graphs, (0, 2)):               # both under way, one behind the other, in pages of their own
        for b, t in zip(bufs, sets[pick]):
            b.copy_(t)
    fresh()
    for graph, _, _ in graphs:
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(graphs[0][2], want[0]) and torch.equal(graphs[1][2], want[2])


def test_two_streams_at_once():
    """Calls on two streams, named as an argument, at the same time: each as alone."""
    from paper_2505_21070_amd import binding as B
    keys, n = 4000, 3
    caches, want, data = [], [], []
    g = torch.ones(D, dtype=torch.bfloat16, device="cuda")
    table = torch.arange(keys // PAGE, dtype=torch.int32, device="cuda")[None].contiguous()
    start, lens = torch.tensor([0, n], dtype=torch.int32, device="cuda"), torch.tensor([keys], dtype=torch.int32, device="cuda")
    for s in range(2):
        c = B.KVCache.empty(keys // PAGE, HK, PAGE, D, "bf16", s == 1)
        x, pos = block(keys, 30 + s)
        q = c.write_qkv(x[:, :HQ], x[:, HQ: HQ + HK], x[:, HQ + HK:], g, g, pos, torch.arange(keys, dtype=torch.int32, device="cuda"))[-n:]
        caches.append(c)
        data.append(q.contiguous())
        want.append(c.attend(data[-1], start, lens, table, n, keys))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(20):
        for s in range(2):
            got[s].append(caches[s].attend(data[s], start, lens, table, n, keys, stream=streams[s]))
    torch.cuda.synchronize()
    for s in range(2):
        assert all(torch.equal(y, want[s]) for y in got[s])


def test_a_stream_of_another_device_is_refused():
    from paper_2505_21070_amd import binding as B
    cache = B.KVCache.empty(2, HK, PAGE, D)

    class Other:
        device, cuda_stream = torch.device("cuda", torch.cuda.current_device() + 1), 0

    with pytest.raises(AssertionError):
        cache.read(torch.zeros(1, dtype=torch.int32, device="cuda"), stream=Other())
