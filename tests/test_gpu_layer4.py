"""A layer's step in 4 bits, the operators one behind the other as a program uses them, for a first chunk and then single tokens of several sequences, against the
same steps in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import fp4 as F
from oracle import paged as O
from paged import TD, np64

pytestmark = pytest.mark.gpu
EPS = float(np.float32(1e-6))


class Layer:
    def __init__(self, dim, heads, kv_heads, d, ffn, dtype, seqs, seed):
        from paper_2505_21070_amd import binding as B
        gen = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=gen)   # noqa: E731
        self.B, self.heads, self.kv, self.d, self.dtype = B, heads, kv_heads, d, dtype
        self.m, self.w = {}, {}
        for name, (o, i) in dict(qkv=((heads + 2 * kv_heads) * d, dim), out=(dim, heads * d), up=(ffn, dim), down=(dim, ffn)).items():
            bias = (r(o) * 0.1).to(TD[dtype])
            codes, scales = B.pack_fp4((r(o, i) * i ** -0.5).to(TD[dtype]).cuda())
            self.m[name] = B.Linear4(codes, scales, bias.cuda(), dtype)
            self.w[name] = (F.decode(F.unpack(codes.view(torch.uint8).cpu().numpy()), scales.cpu().numpy()), np64(bias))
        self.g = {n: (r(s) * 0.1 + 1.1).to(TD[dtype]) for n, s in dict(q=d, k=d, attn=dim, ffn=dim).items()}
        self.v = {n: r(seqs, dim) * 0.3 for n in ("gate1", "scale1", "shift1", "gate2", "scale2", "shift2")}
        self.gd, self.vd = {n: t.cuda() for n, t in self.g.items()}, {n: t.cuda() for n, t in self.v.items()}

    def gpu(self, x, cache, group, pos, slot, q_start, kv_len, table, max_q, max_kv):
        B, n, h, kv, d = self.B, x.shape[0], self.heads, self.kv, self.d
        _, a = B.gated_norm(x, scale=self.vd["scale1"], shift=self.vd["shift1"], group=group, norm="rms", dtype=self.dtype)
        qkv = self.m["qkv"].forward(a).view(n, h + 2 * kv, d)
        q = cache.write_qkv(qkv[:, :h], qkv[:, h: h + kv], qkv[:, h + kv:], self.gd["q"], self.gd["k"], pos, slot)
        o = cache.attend(q, q_start, kv_len, table, max_q, max_kv, causal_group=1)
        y = self.m["out"].forward(o.view(n, h * d))
        x, a = B.gated_norm(x, y, post_gain=self.gd["attn"], gate=self.vd["gate1"], scale=self.vd["scale2"], shift=self.vd["shift2"], group=group, norm="rms")
        y = self.m["down"].forward(self.m["up"].forward(a, act="gelu"))
        x, _ = B.gated_norm(x, y, post_gain=self.gd["ffn"], gate=self.vd["gate2"], group=group, norm="rms", next_norm=False)
        return x, {"qkv": qkv, "q": q, "o": o}

    def steps(self, x, group, got, q, k_all, v_all, q_start, kv_len):
        """The stream behind the layer in 64 bits.  Keys, values and queries are those that the GPU left (read back): codes beside a border fall either way."""
        v = {n: t.numpy() for n, t in self.v.items()}
        rnd = lambda t: np64(torch.from_numpy(np.asarray(t)).to(TD[self.dtype]))   # noqa: E731
        _, a = F.gated_norm(x, None, "rms", EPS, scale=v["scale1"], shift=v["shift1"], group=group)
        qkv = F.linear(a, *self.w["qkv"])[0]
        o = O.attend(q, k_all, v_all, q_start, kv_len, [np.ones(k, bool) for k in kv_len], 1, self.d ** -0.5, q)[0]
        y = F.linear(o.reshape(len(x), -1), *self.w["out"])[0]
        x, a = F.gated_norm(x, y, "rms", EPS, post_gain=np64(self.g["attn"]), gate=v["gate1"], scale=v["scale2"], shift=v["shift2"], group=group)
        y = F.linear(F.linear(a, *self.w["up"], "gelu")[0], *self.w["down"])[0]
        x, _ = F.gated_norm(x, y, "rms", EPS, post_gain=np64(self.g["ffn"]), gate=v["gate2"], group=group)
        return x, qkv, o


def rel(a, b):
    return np.linalg.norm(a - b) / np.linalg.norm(b)


@pytest.mark.parametrize("dtype,heads,kv_heads,d", [("bf16", 4, 2, 128), ("bf16", 6, 6, 64), ("f32", 4, 1, 64)])
def test_a_chunk_then_tokens(dtype, heads, kv_heads, d):
    from paper_2505_21070_amd import binding as B
    seqs, page, dim, ffn = 3, 16, 384, 1056
    layer = Layer(dim, heads, kv_heads, d, ffn, dtype, seqs, seed=heads)
    cache = B.KVCache.empty(40, kv_heads, page, d, dtype, fp4=True)
    gen = torch.Generator().manual_seed(1)
    order = torch.randperm(40, generator=gen).tolist()
    table = torch.tensor([order[:10], order[10:20], order[20:30]], dtype=torch.int32)
    held = [0, 0, 0]
    for new in ([37, 5, 90], [1, 1, 1], [1, 1, 1], [2, 0, 1]):
        n, start = sum(new), np.concatenate([[0], np.cumsum(new)])
        x = torch.randn((n, dim), generator=gen) * 2
        group = np.repeat(np.arange(seqs), new)
        at = np.concatenate([np.arange(h, h + k) for h, k in zip(held, new)]).astype(int)
        pos = torch.stack([torch.from_numpy(at) // 6, torch.from_numpy(at) // 3 % 2, torch.from_numpy(at) % 3], dim=1).to(torch.int32)
        slot = torch.tensor([int(table[b, i // page]) * page + i % page for b, i in zip(group, at)], dtype=torch.int32)
        held = [h + k for h, k in zip(held, new)]
        i32 = lambda v: torch.tensor([int(i) for i in v], dtype=torch.int32, device="cuda")   # noqa: E731
        args = (x.cuda(), cache, i32(group), pos.cuda(), slot.cuda(), i32(start), i32(held), table.cuda(), max(new), max(held))
        got, mid = layer.gpu(*args)
        again, _ = layer.gpu(*args)
        assert torch.equal(got, again)
        k_all, v_all = [], []
        for b, h in enumerate(held):
            k, v = cache.read(i32(int(table[b, i // page]) * page + i % page for i in range(h)))
            k_all.append(np64(k))
            v_all.append(np64(v))
        ref, qkv, o = layer.steps(np64(x), group, mid, np64(mid["q"]), k_all, v_all, start, held)
        # roundings to the rows' type on the way, half a step each (in the 2-norm): the norm and the product's own behind it for qkv; weights, sums of weights and the result
        # for o; for the stream o, y, norm, the up product and the down product, their sum as if all went one way, times the branches' share, below 1
        u = {"bf16": 2.0 ** -8, "f32": 2e-6}[dtype]
        assert rel(np64(mid["qkv"]).reshape(qkv.shape), qkv) < 2 * u
        assert rel(np64(mid["o"]), o) < 3 * u
        assert rel(np64(got), ref) < 6 * u
        # the rows that the step wrote are what its product left, the values to the code
        vals = F.rows(np64(mid["qkv"])[:, heads + kv_heads:])[0]
        for b in range(seqs):
            if new[b]:
                assert np.array_equal(v_all[b][-new[b]:], vals[start[b]: start[b + 1]])


def test_a_captured_step_replayed():
    """The whole step of single tokens as one graph, replayed as the sequences grow, with eager steps on another cache beside it."""
    from paper_2505_21070_amd import binding as B
    seqs, page, dim, heads, kv, d = 4, 16, 256, 4, 2, 64
    layer = Layer(dim, heads, kv, d, 512, "bf16", seqs, seed=7)
    caches = [B.KVCache.empty(16, kv, page, d, "bf16", fp4=True) for _ in range(2)]
    table = torch.arange(16, dtype=torch.int32, device="cuda").view(4, 4)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")   # noqa: E731
    state = dict(x=torch.zeros((seqs, dim), device="cuda"), group=i32(0, 1, 2, 3), pos=torch.zeros((seqs, 3), dtype=torch.int32, device="cuda"), slot=i32(0, 64, 128, 192),
                 q_start=i32(0, 1, 2, 3, 4), kv_len=i32(1, 1, 1, 1))
    call = lambda c: layer.gpu(state["x"], c, state["group"], state["pos"], state["slot"], state["q_start"], state["kv_len"], table, 1, 64)[0]   # noqa: E731
    call(caches[0]), call(caches[1])                          # both hold the same tokens
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = call(caches[0])
    for step in range(40):
        state["x"].copy_(torch.randn((seqs, dim), generator=torch.Generator().manual_seed(step)))
        state["pos"].fill_(step)
        at = torch.tensor([step, step // 2, 39 - step, 0], dtype=torch.int32, device="cuda")
        state["slot"].copy_(table[torch.arange(4, device="cuda"), (at // page).long()] * page + at % page)
        state["kv_len"].copy_(torch.clamp(at + 1, min=1))
        graph.replay()
        torch.cuda.synchronize()
        eager = call(caches[1])
        assert torch.equal(y, eager), step
        assert torch.equal(caches[0].data.view(torch.uint8), caches[1].data.view(torch.uint8))
