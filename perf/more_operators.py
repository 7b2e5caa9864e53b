"""Passes through the operators of a layer's step whose weights, keys and values are held in 4 bits, as a list of measurable cases.

Four operators:

  cache    keys and values written into the pages of a cache in 4 bits, and read back (KVCache.write, KVCache.read)
  attend   new tokens of several sequences attend to the cached keys and values of their own sequence, held in 4 bits (KVCache.attend)
  linear   tokens times a matrix of 4-bit weights, with a bias and an activation: y = act(x W^T + b) (Linear4.forward)
  norm     a branch's output added to the residual stream, and the next branch's input, in one pass (gated_norm):
           x' = x + r * gate * N(y) * post_gain,  h = N(x') * gain * (1 + scale) + shift, with N a LayerNorm or an RMSNorm

Each has its plain form here, in elementary torch operations, and its definition once more in 64 bits (exact).

4 bits: values are held in groups of 32, as codes of e2m1 (sign, 0 0.5 1 1.5 2 3 4 6), two to a byte with the first one in the low half, and a byte b that stands
for the factor 2^(b - 127) of the group: the least factor 2^e, -100 <= e <= 125, by which no finite value of the group is over 7 (6 and 7 have the same
code).  A group with a value that is not finite has the byte 255.  A cache is two tensors: data [pages, 2 (keys, values), heads, page tokens, head_dim / 2] and
scales [pages, 2, heads, page tokens, head_dim / 32]; a matrix is codes [out, in / 2] and scales [out, in / 32].

Inputs are what the path meets: rows of unit variance, some channels of which are larger than the others, gains around 1.2, pages handed out in no order,
weights as they come out of the rounding of normal ones.
"""
import math
import random

import torch

own = False
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


def _cache(name, **kw):
    return dict(dict(name=name, kind="cache", dtype="bf16", tokens=6240, kv_heads=40, head_dim=128, page=64, run=64), **kw)


def _attend(name, **kw):
    return dict(dict(name=name, kind="attend", dtype="bf16", seqs=1, q_lo=1, q_hi=1, old_lo=0, old_hi=0, heads=12, kv_heads=12, head_dim=128, page=64, group=0), **kw)


def _linear(name, **kw):
    return dict(dict(name=name, kind="linear", dtype="bf16", tokens=1, rows=1536, cols=1536, act="", bias=True), **kw)


def _norm(name, **kw):
    return dict(dict(name=name, kind="norm", dtype="bf16", stream="f32", tokens=6240, dim=5120, groups=4, form="layer", post=False, modulated=True), **kw)


def listed():
    return [
        # a block of 4 frames of 30 x 52 tokens, 40 heads: its keys and values go into the pages and come back
        _cache("cache4_block"),
        # one new token each of 48 sequences, every one in a page of its own, shared key heads of 64, fp32 rows, some rows of padding
        _cache("cache4_tokens_f32", dtype="f32", tokens=48, kv_heads=8, head_dim=64, page=16, run=1),
        # a block over a long history: every query sees every key
        _attend("attend4_history", q_lo=1560, q_hi=1560, old_lo=18720, old_hi=18720),
        # one token each of 64 sequences of 100 to 16000 keys: what serving does between chunks
        _attend("attend4_tokens", seqs=64, old_lo=99, old_hi=15999, heads=32, kv_heads=8, page=16, group=1),
        # one token, one short sequence, heads of 64: latency
        _attend("attend4_one", old_lo=516, old_hi=516, head_dim=64, page=16, group=1),
        # the fused q | k | v product of one token at 1536 channels: latency
        _linear("linear4_token", rows=4608),
        # the widest feed-forward product, one token: how fast the weights are read
        _linear("linear4_wide", rows=13824, cols=5120, act="gelu"),
        # and its way back, for the next tokens of 48 sequences
        _linear("linear4_seqs", tokens=48, rows=5120, cols=13824),
        # a frame of 1560 tokens through a feed-forward product: arithmetic
        _linear("linear4_frame", tokens=1560, rows=8960, act="gelu"),
        # fp32, sizes that divide nothing, an activation as in the timestep's vector
        _linear("linear4_odd_f32", dtype="f32", tokens=37, rows=1001, cols=1504, act="silu", bias=False),
        # a block of four videos at the widest model: fp32 stream, LayerNorm, modulated per video
        _norm("norm_gated_block"),
        # next tokens of 48 sequences, bf16 stream, RMSNorm before and after the branch
        _norm("norm_both_tokens", stream="bf16", tokens=48, dim=1536, groups=1, form="rms", post=True, modulated=False),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def _cost(case):
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / (1e15 if case["dtype"] == "bf16" else 1e14)


def draw(rng):
    most = {k: max(_cost(c) for c in listed() if c["kind"] == k) for k in ("cache", "attend", "linear", "norm")}
    while True:
        kind = rng.choice(("cache", "attend", "attend", "linear", "linear", "linear", "norm", "norm"))
        c = dict(kind=kind, dtype=rng.choice(("bf16", "bf16", "bf16", "f32")))
        if kind in ("cache", "attend"):
            kv = rng.choice((1, 2, 3, 4, 5, 8, 12, 16, 20, 32, 40))
            c.update(kv_heads=kv, head_dim=rng.choice((64, 128)), page=rng.choice((16, 32, 64, 128, 256)))
        if kind == "cache":
            c["tokens"] = _spread(rng, 1, 15000)
            c["run"] = rng.choice((1, c["page"], c["page"]))
            if -(-c["tokens"] // c["run"]) * c["page"] * kv * c["head_dim"] > 1e9:          # of pages
                continue
        if kind == "attend":
            chunk = rng.random() < 0.4
            hi = _spread(rng, 2, 3000) if chunk else rng.choice((1, 1, 1, 2, 5))
            old = _spread(rng, 1, 20000 if chunk else 60000) - 1
            c.update(heads=kv * rng.choice((1, 1, 2, 3, 4, 8)), seqs=_spread(rng, 1, 6 if chunk else 64), q_lo=max(1, hi // rng.choice((1, 1, 3))), q_hi=hi,
                     old_lo=old // rng.choice((1, 2, 50)), old_hi=old, group=rng.choice((0, 0, 1, 60, 390)))
            # the plain form holds all its scores at once
            if c["heads"] > 64 or c["seqs"] * c["heads"] * hi * (hi + old) > 2.5e9 or c["seqs"] * kv * c["head_dim"] * (hi + old) > 1.5e9:
                continue
        if kind == "linear":
            c.update(tokens=_spread(rng, 1, 4000) if rng.random() < 0.7 else _spread(rng, 1, 64), rows=_spread(rng, 8, 20000), cols=32 * _spread(rng, 1, 500),
                     act=rng.choice(("", "gelu", "silu")), bias=rng.random() < 0.5)
        if kind == "norm":
            c.update(stream=rng.choice(("f32", c["dtype"])), tokens=_spread(rng, 1, 15000), dim=8 * _spread(rng, 8, 1024), groups=_spread(rng, 1, 64),
                     form=rng.choice(("layer", "rms")), post=rng.random() < 0.5, modulated=rng.random() < 0.6)
        if _cost(c) <= most[kind]:
            return c


def _spaced(lo, hi, n, step):
    """n whole numbers from lo to hi, in an order that is neither rising nor falling."""
    return [lo + (hi - lo) * ((i * step + n - 1) % n) // max(1, n - 1) if n > 1 else hi for i in range(n)]


def _lengths(case):
    """New tokens and keys (the new ones among them) of each sequence."""
    q = _spaced(case["q_lo"], case["q_hi"], case["seqs"], 1)
    old = _spaced(case["old_lo"], case["old_hi"], case["seqs"], 1)[::-1]
    return q, [a + b for a, b in zip(q, old)]


def _seen(i, n, keys, group):
    """Keys that the i-th of n new tokens sees."""
    return keys if group == 0 else min(keys, ((keys - n + i) // group + 1) * group)


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    n = case.get("tokens", 0)
    if case["kind"] == "linear":
        rows, cols = case["rows"], case["cols"]
        return {"bytes": rows * cols // 2 + rows * cols // 32 + n * (rows + cols) * e + rows * e * case["bias"], "flops": 2 * n * rows * cols}
    if case["kind"] == "norm":
        s = 2 if case["stream"] == "bf16" else 4
        vectors = 4 * case["groups"] * case["dim"] * (3 if case["modulated"] else 1) + case["dim"] * e * (1 + case["post"])
        return {"bytes": 2 * n * case["dim"] * (s + e) + vectors + 4 * n, "flops": n * case["dim"] * (16 if case["post"] else 12)}
    hk, d = case["kv_heads"], case["head_dim"]
    held = hk * (d // 2 + d // 32)                                    # bytes of a token's keys (or values) in the pages
    if case["kind"] == "cache":
        # written: rows in, pages out; read back: pages in, rows out
        return {"bytes": n * (2 * 2 * hk * d * e + 2 * 2 * held + 8), "flops": 4 * n * 2 * hk * d}
    q, kv = _lengths(case)
    pairs = sum(n * keys if case["group"] == 0 else sum(_seen(i, n, keys, case["group"]) for i in range(n)) for n, keys in zip(q, kv))
    table = 4 * sum(-(-keys // case["page"]) for keys in kv)
    return {"bytes": 2 * sum(q) * case["heads"] * d * e + 2 * sum(kv) * held + table, "flops": 4 * d * case["heads"] * pairs}


def _rows(gen, shape, dtype):
    """Rows of unit variance in which one channel of 16 is three times as large as the others."""
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    x[..., ::16] *= 3.0
    return (x * (16 / 24) ** 0.5).to(DT[dtype])


def _pages(case, n_pages):
    shape = (n_pages, 2, case["kv_heads"], case["page"])
    return (torch.zeros(shape + (case["head_dim"] // 2,), device="cuda", dtype=torch.uint8),
            torch.full(shape + (case["head_dim"] // 32,), 127, device="cuda", dtype=torch.uint8))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    host = random.Random(seed)
    s = dict(case=case)
    if case["kind"] == "linear":
        rows, cols, dt = case["rows"], case["cols"], DT[case["dtype"]]
        codes, scales = torch.empty((rows, cols // 2), device="cuda", dtype=torch.uint8), torch.empty((rows, cols // 32), device="cuda", dtype=torch.uint8)
        for first in range(0, rows, 4096):
            w = torch.randn((min(4096, rows - first), cols), generator=gen, device="cuda") * cols ** -0.5
            codes[first: first + 4096], scales[first: first + 4096] = _to_4_bits(w)
        s.update(codes=codes, scales=scales, x=_rows(gen, (case["tokens"], cols), case["dtype"]))
        s["bias"] = (torch.randn(rows, generator=gen, device="cuda") * 0.1).to(dt) if case["bias"] else None
        if own:
            from paper_2505_21070_amd import binding
            s["linear"] = binding.Linear4(codes.view(torch.float4_e2m1fn_x2), scales, s["bias"], dtype=case["dtype"])
        return s
    if case["kind"] == "norm":
        n, dim, dt = case["tokens"], case["dim"], DT[case["dtype"]]
        s.update(x=_rows(gen, (n, dim), "f32").mul_(3.0).to(DT[case["stream"]]), y=_rows(gen, (n, dim), case["dtype"]),
                 gate=torch.randn((case["groups"], dim), generator=gen, device="cuda") * 0.5)
        gains = (torch.randn((2, dim), generator=gen, device="cuda") * 0.1 + 1.2).to(dt)
        s.update(gain=None if case["modulated"] else gains[0], post=gains[1] if case["post"] else None)
        mod = torch.randn((2, case["groups"], dim), generator=gen, device="cuda") * 0.3
        s.update(scale=mod[0] if case["modulated"] else None, shift=mod[1] if case["modulated"] else None)
        # rows of a group (a video) lie one behind the other
        s["group"] = (torch.arange(n, device="cuda") * case["groups"] // n).to(torch.int32)
        return s
    d, hk, page = case["head_dim"], case["kv_heads"], case["page"]
    if case["kind"] == "attend":
        q, kv = _lengths(case)
        pages = [-(-keys // page) for keys in kv]
        n_pages = sum(pages) + 3
        order = list(range(n_pages))
        host.shuffle(order)
        table = torch.zeros((case["seqs"], max(pages)), dtype=torch.int32)
        for b, n in enumerate(pages):
            table[b, :n] = torch.tensor(order[:n], dtype=torch.int32)
            order = order[n:]
        s["q"] = _rows(gen, (sum(q), case["heads"], d), case["dtype"]) * 1.3
        data, scales = _pages(case, n_pages)
        for first in range(0, n_pages, 512):                          # what earlier writes left in the pages
            n = min(512, n_pages - first)
            data[first: first + n], scales[first: first + n] = _to_4_bits(_rows(gen, (n, 2, hk, page, d), case["dtype"]).float())
        starts = [0]
        for n in q:
            starts.append(starts[-1] + n)
        s.update(data=data, scales=scales, table=table.cuda(), q_start=torch.tensor(starts, dtype=torch.int32).cuda(),
                 kv_len=torch.tensor(kv, dtype=torch.int32).cuda(), max_q=max(q), max_kv=max(kv))
        # which sequence a row of queries is of, and which of its new tokens: the plain form's way back from padded chunks
        s["row_seq"] = torch.tensor([b for b, n in enumerate(q) for _ in range(n)]).cuda()
        s["row_in"] = torch.tensor([i for n in q for i in range(n)]).cuda()
    else:
        n, run_ = case["tokens"], case["run"]                          # run: tokens that lie one behind the other in a page
        x = _rows(gen, (n, 3 * hk, d), case["dtype"])                  # one q | k | v product's output
        s.update(k=x[:, hk: 2 * hk], v=x[:, 2 * hk:])
        n_pages = -(-n // run_) + 2
        order = list(range(n_pages))
        host.shuffle(order)
        slot = [order[t // run_] * page + (t % run_ if run_ > 1 else (t * 7) % page) for t in range(n)]
        for t in range(5, n, 61):                                      # rows of padding, which go nowhere
            slot[t] = -1
        data, scales = _pages(case, n_pages)
        s.update(data=data, scales=scales, slot=torch.tensor(slot, dtype=torch.int32).cuda(), kept=torch.tensor([t for t in range(n) if slot[t] >= 0]).cuda())
    if own:
        from paper_2505_21070_amd import binding
        s["cache"] = binding.KVCache(data.view(torch.float4_e2m1fn_x2), scales, dtype=case["dtype"])
    return s


# ---- plain forms

def _to_4_bits(x):
    """Codes, two to a byte, and scale bytes of fp32 rows, in groups of 32 of the last axis."""
    x = x.unflatten(-1, (-1, 32))
    a = x.abs()
    m, e = torch.frexp(torch.where(a < math.inf, a, 0.0).amax(-1))
    e = (e - 3 + (m > 0.875)).clamp(min=-100, max=125)
    a = torch.ldexp(a, -e.unsqueeze(-1))
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)) | (torch.signbit(x).to(torch.uint8) << 3)
    fine = (a < math.inf).all(-1)
    code = torch.where(fine.unsqueeze(-1), code, 0)
    return (code[..., 0::2] | code[..., 1::2] << 4).flatten(-2), torch.where(fine, e + 127, 255).to(torch.uint8)


def _from_4_bits(data, scales):
    code = torch.stack((data & 15, data >> 4), dim=-1).flatten(-2).to(torch.int32)
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=data.device)
    x = torch.where(code > 7, -table[code & 7], table[code & 7]).unflatten(-1, (-1, 32))
    b = scales.to(torch.int32).unsqueeze(-1)
    return torch.where(b < 255, torch.ldexp(x, b - 127), math.nan).flatten(-2)


def _plain_cache(s):
    page, kept = s["case"]["page"], s["kept"]
    slot = s["slot"][kept].long()
    at = (slot // page, slice(None), slice(None), slot % page)
    s["data"][at], s["scales"][at] = _to_4_bits(torch.stack((s["k"][kept], s["v"][kept]), dim=1).float())      # [tokens, 2, heads, head_dim]
    slot = s["slot"].clamp(min=0).long()
    at = (slot // page, slice(None), slice(None), slot % page)
    rows = torch.where((s["slot"] >= 0).view(-1, 1, 1, 1), _from_4_bits(s["data"][at], s["scales"][at]), 0.0).to(DT[s["case"]["dtype"]])
    return {"k": rows[:, 0], "v": rows[:, 1]}


def _plain_attend(s):
    c = s["case"]
    hk, d, n, keys = c["kv_heads"], c["head_dim"], s["max_q"], s["max_kv"]
    shared = c["heads"] // hk
    table = s["table"].long()
    held = _from_4_bits(s["data"][table], s["scales"][table])
    held = held.permute(2, 0, 3, 1, 4, 5).reshape(2, c["seqs"], hk, -1, d)[..., :keys, :]      # [2, sequences, heads, keys, head_dim]
    new = s["q_start"].diff().long()
    rows = (s["q_start"][:-1, None] + torch.arange(n, device="cuda")).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][rows].float().view(c["seqs"], n, hk, shared, d).permute(0, 2, 3, 1, 4).reshape(c["seqs"], hk, shared * n, d)
    score = torch.matmul(q, held[0].transpose(-1, -2)).div_(math.sqrt(d)).view(c["seqs"], hk, shared, n, keys)
    seen = s["kv_len"].long()[:, None].expand(-1, n)
    if c["group"]:
        at = seen - new[:, None] + torch.arange(n, device="cuda")
        seen = torch.minimum(seen, (torch.div(at, c["group"], rounding_mode="floor") + 1) * c["group"])
    hidden = torch.arange(keys, device="cuda") >= seen[..., None]
    score.masked_fill_(hidden[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    weight = score.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    total = weight.sum(-1, keepdim=True)
    out = torch.matmul(weight.view(c["seqs"], hk, shared * n, keys), held[1]).view(c["seqs"], hk, shared, n, d)
    out = out / torch.where(total > 0, total, 1.0)
    return {"out": out.permute(0, 3, 1, 2, 4).reshape(c["seqs"], n, c["heads"], d)[s["row_seq"], s["row_in"]].to(DT[c["dtype"]])}


def _plain_linear(s):
    c = s["case"]
    y = torch.matmul(s["x"].float(), _from_4_bits(s["codes"], s["scales"]).t())
    if s["bias"] is not None:
        y = y + s["bias"].float()
    if c["act"] == "gelu":
        y = 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y * y * y)))
    if c["act"] == "silu":
        y = y / (1 + torch.exp(-y))
    return {"y": y.to(DT[c["dtype"]])}


def _plain_norm(s):
    c = s["case"]

    def normed(x):
        if c["form"] == "layer":
            x = x - x.mean(-1, keepdim=True)
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    group = s["group"].long()
    t = s["y"].float()
    if s["post"] is not None:
        t = normed(t) * s["post"].float()
    x = s["x"].float() + 0.5 * s["gate"][group] * t
    h = normed(x)
    if s["gain"] is not None:
        h = h * s["gain"].float()
    if s["scale"] is not None:
        h = h * (1 + s["scale"][group]) + s["shift"][group]
    return {"x": x.to(DT[c["stream"]]), "h": h.to(DT[c["dtype"]])}


def run(s):
    c = s["case"]
    if own:
        from paper_2505_21070_amd import binding
        if c["kind"] == "cache":
            s["cache"].write(s["k"], s["v"], s["slot"])
            k, v = s["cache"].read(s["slot"])
            return {"k": k, "v": v}
        if c["kind"] == "attend":
            return {"out": s["cache"].attend(s["q"], s["q_start"], s["kv_len"], s["table"], s["max_q"], s["max_kv"], causal_group=c["group"])}
        if c["kind"] == "linear":
            return {"y": s["linear"].forward(s["x"], act=c["act"] or None)}
        x, h = binding.gated_norm(s["x"], s["y"], gain=s["gain"], post_gain=s["post"], gate=s["gate"], scale=s["scale"], shift=s["shift"], group=s["group"],
                                  norm=c["form"], res_scale=0.5, eps=EPS)
        return {"x": x, "h": h}
    return {"cache": _plain_cache, "attend": _plain_attend, "linear": _plain_linear, "norm": _plain_norm}[c["kind"]](s)


# ---- the same from the definitions, in 64 bits

def _exact_4_bits(x):
    """Nearest values of 2 exponent bits and 1 fraction bit (ties to even) times the group's power of two.  The inputs of a case are finite and far from the range's ends."""
    x = x.double().unflatten(-1, (-1, 32))
    top = x.abs().amax(-1, keepdim=True)
    power = torch.where(top > 0, torch.ceil(torch.log2(top.clamp(min=1e-300) / 7)), torch.full_like(top, -100.0))
    power = torch.where(top * torch.exp2(1 - power) <= 7, power - 1, power)
    power = torch.where(top * torch.exp2(-power) > 7, power + 1, power).clamp(min=-100)
    y = x * torch.exp2(-power)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=1.0, max=6.0))) - 1)
    return ((torch.round(y / step) * step).clamp(min=-6, max=6) * torch.exp2(power)).flatten(-2)


def _exact_held(data, scales):
    """What codes and scale bytes stand for."""
    bits = data.to(torch.int64).unsqueeze(-1) >> torch.tensor([0, 4], device=data.device) & 15
    sign, power, fraction = bits >> 3, bits >> 1 & 3, bits & 1
    size = torch.where(power > 0, (2 + fraction).double() * torch.exp2(power.double() - 2), fraction.double() / 2)
    x = torch.where(sign > 0, -size, size).flatten(-2).unflatten(-1, (-1, 32))
    return (x * torch.exp2(scales.double() - 127).unsqueeze(-1)).flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "cache":
        live = (s["slot"] >= 0).double().view(-1, 1, 1)
        return {name: _exact_4_bits(s[name]) * live for name in ("k", "v")}
    if case["kind"] == "linear":
        if case["tokens"] * case["rows"] * case["cols"] > 4e11:
            return None
        y = torch.cat([s["x"].double() @ _exact_held(s["codes"][i: i + 2048], s["scales"][i: i + 2048]).T for i in range(0, case["rows"], 2048)], dim=1)
        if s["bias"] is not None:
            y = y + s["bias"].double()
        if case["act"] == "gelu":
            y = y * torch.sigmoid(math.sqrt(8 / math.pi) * (y + 0.044715 * y ** 3))
        if case["act"] == "silu":
            y = y * torch.sigmoid(y)
        return {"y": y}
    if case["kind"] == "norm":
        def normed(x):
            mean = x.sum(-1, keepdim=True) / x.shape[-1] if case["form"] == "layer" else torch.zeros_like(x[..., :1])
            return (x - mean) / ((x - mean).pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt()
        group = s["group"].long()
        t = s["y"].double() if s["post"] is None else normed(s["y"].double()) * s["post"].double()
        x = s["x"].double() + s["gate"].double()[group] * t / 2
        h = normed(x) if s["gain"] is None else normed(x) * s["gain"].double()
        if case["modulated"]:
            h = h + h * s["scale"].double()[group] + s["shift"].double()[group]
        return {"x": x, "h": h}
    d, hk, shared = case["head_dim"], case["kv_heads"], case["heads"] // case["kv_heads"]
    q_len, kv_len = _lengths(case)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    row = 0
    for b, (n, keys) in enumerate(zip(q_len, kv_len)):
        table = s["table"][b].long()
        held = _exact_held(s["data"][table], s["scales"][table]).permute(1, 2, 0, 3, 4).reshape(2, hk, -1, d)[:, :, :keys]
        ends = torch.tensor([_seen(i, n, keys, case["group"]) for i in range(n)], device="cuda")
        for h in range(case["heads"]):
            k, v = held[0, h // shared], held[1, h // shared]
            score = (s["q"][row: row + n, h].double() @ k.T) / d ** 0.5
            score = torch.where(torch.arange(keys, device="cuda")[None, :] < ends[:, None], score, torch.full((), -math.inf, dtype=torch.float64, device="cuda"))
            out[row: row + n, h] = torch.softmax(score, dim=-1) @ v
        row += n
    return {"out": out}
