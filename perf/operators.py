"""Passes through the operators around a paged key/value cache, as a list of measurable cases.

Three operators, four kinds of case:

  norm     RMSNorm of queries and keys for each head and their 3D rotation, in one pass (binding.qk_norm_rope)
  cache    keys and values written into the pages of a cache, in 8 bits or as they are, and read back (KVCache.write, KVCache.read)
  project  the two in one: queries normalised and rotated, keys normalised, rotated and written, values written (KVCache.write_qkv),
           and what the pages then hold read back
  attend   a chunk of new tokens of several sequences attends to the cached keys and values of its own sequence (KVCache.attend)

Each has its plain form here, in elementary torch operations, and its definition once more in 64 bits (exact).  A cache is two
tensors: data [pages, 2 (keys, values), heads, page tokens, head_dim] and, for 8-bit data (float8_e4m3fn), scales of the same shape
without the last axis: bytes b that stand for the factor 2^(b - 127) of a token's head.

Inputs are what the path meets: rows of unit variance, some channels of which are larger than the others, gains around 1.2,
positions at absolute frames, pages handed out in no order.
"""
import math
import random

import torch

own = False
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
THETA, EPS = 1e4, 1e-6


def _norm(name, **kw):
    return dict(dict(name=name, kind="norm", dtype="bf16", frames=4, tok_h=30, tok_w=52, heads=12, kv_heads=12, head_dim=128, frame0=500), **kw)


def _cache(name, **kw):
    return dict(dict(name=name, kind="cache", dtype="bf16", fp8=True, tokens=6240, kv_heads=12, head_dim=128, page=64, run=64), **kw)


def _project(name, **kw):
    return dict(dict(name=name, kind="project", dtype="bf16", fp8=True, frames=4, tok_h=30, tok_w=52, heads=12, kv_heads=12, head_dim=128,
                     frame0=64, page=64, run=64), **kw)


def _attend(name, **kw):
    return dict(dict(name=name, kind="attend", dtype="bf16", fp8=True, seqs=1, q_lo=1, q_hi=1, old_lo=0, old_hi=0, heads=12, kv_heads=12,
                     head_dim=128, page=64, group=0), **kw)


def listed():
    return [
        # a block of 4 frames of 30 x 52 tokens at the widest model in use: 40 heads of queries and of keys out of one q | k | v product
        _norm("norm_block", heads=40, kv_heads=40),
        # shared key heads of 64 in fp32, a token count that divides nothing
        _norm("norm_shared_f32", dtype="f32", frames=27, tok_h=7, tok_w=9, heads=16, kv_heads=4, head_dim=64),
        # one token: what counts is latency
        _norm("norm_token", frames=1, tok_h=1, tok_w=1),
        # a block's keys and values go into the pages in 8 bits and come back
        _cache("cache_block", kv_heads=40),
        # one new token each of 48 sequences, every one in a page of its own
        _cache("cache_tokens", tokens=48, kv_heads=8, page=16, run=1),
        # a block on its way from the q | k | v product into the pages
        _project("project_block"),
        # a block of 6240 tokens over itself and 2 cached frames, 8-bit pages, every query sees every key
        _attend("attend_block", q_lo=6240, q_hi=6240, old_lo=3120, old_hi=3120, heads=40, kv_heads=40),
        # a block over a long history held as it is
        _attend("attend_history", fp8=False, q_lo=1560, q_hi=1560, old_lo=18720, old_hi=18720),
        # chunks of four videos of different age, heads of 64 that share keys, each frame of 390 tokens sees the frames up to itself
        _attend("attend_frames", fp8=False, seqs=4, q_lo=390, q_hi=1560, old_lo=0, old_hi=5850, heads=16, kv_heads=8, head_dim=64, page=32, group=390),
        # one token each of 64 sequences of 100 to 16000 keys: what serving does between chunks
        _attend("attend_tokens", seqs=64, old_lo=99, old_hi=15999, heads=32, kv_heads=8, page=16, group=1),
        # one token, one short sequence: latency
        _attend("attend_one", fp8=False, old_lo=516, old_hi=516, page=16, group=1),
        # fp32, two ragged chunks
        _attend("attend_f32", dtype="f32", fp8=False, seqs=2, q_lo=130, q_hi=390, old_lo=390, old_hi=1170, page=32),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def _cost(case):
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / (1e15 if case["dtype"] == "bf16" else 1e14)


def draw(rng):
    most = {k: max(_cost(c) for c in listed() if c["kind"] == k) for k in ("norm", "cache", "project", "attend")}
    while True:
        kind = rng.choice(("norm", "cache", "project", "attend", "attend", "attend"))
        kv = rng.choice((1, 2, 3, 4, 5, 8, 12, 16, 20, 32, 40))
        heads = kv * rng.choice((1, 1, 2, 3, 4, 8))
        c = dict(kind=kind, dtype=rng.choice(("bf16", "bf16", "bf16", "f32")), heads=heads, kv_heads=kv, head_dim=rng.choice((64, 128)))
        if heads > 64:
            continue
        if kind in ("norm", "project"):
            c.update(frames=_spread(rng, 1, 28), tok_h=_spread(rng, 1, 45), tok_w=_spread(rng, 1, 80), frame0=_spread(rng, 1, 4000) - 1)
        if kind != "norm":
            c.update(fp8=rng.random() < 0.6, page=rng.choice((16, 32, 64, 128, 256)))
        if kind == "cache":
            del c["heads"]
            c["tokens"] = _spread(rng, 1, 15000)
        if kind in ("cache", "project"):
            c["run"] = rng.choice((1, c["page"], c["page"]))
        if kind == "attend":
            chunk = rng.random() < 0.5
            hi = _spread(rng, 2, 7000) if chunk else rng.choice((1, 1, 2, 5))
            old = _spread(rng, 1, 16000 if chunk else 60000) - 1
            c.update(seqs=_spread(rng, 1, 6 if chunk else 64), q_lo=max(1, hi // rng.choice((1, 1, 3))), q_hi=hi, old_lo=old // rng.choice((1, 2, 50)),
                     old_hi=old, group=rng.choice((0, 0, 1, 60, 390)))
            # the plain form holds all its scores at once
            if c["seqs"] * heads * hi * (hi + old) > 2.5e9 or c["seqs"] * kv * c["head_dim"] * (hi + old) > 1.5e9:
                continue
        if kind in ("cache", "project") and -(-_tokens(c) // c["run"]) * c["page"] * kv * c["head_dim"] > 1e9:      # of pages
            continue
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


def _tokens(case):
    return case["tokens"] if case["kind"] == "cache" else case["frames"] * case["tok_h"] * case["tok_w"]


def work(case):
    d, hk, e = case["head_dim"], case["kv_heads"], 2 if case["dtype"] == "bf16" else 4
    held = hk * (d + 1) if case.get("fp8") else hk * d * e          # bytes of a token's keys (or values) in the pages
    if case["kind"] == "attend":
        q, kv = _lengths(case)
        pairs = sum(n * keys if case["group"] == 0 else sum(_seen(i, n, keys, case["group"]) for i in range(n)) for n, keys in zip(q, kv))
        table = 4 * sum(-(-keys // case["page"]) for keys in kv)
        return {"bytes": 2 * sum(q) * case["heads"] * d * e + 2 * sum(kv) * held + table, "flops": 4 * d * case["heads"] * pairs}
    n = _tokens(case)
    if case["kind"] == "norm":
        return {"bytes": n * (2 * (case["heads"] + hk) * d * e + 12), "flops": 8 * n * (case["heads"] + hk) * d}
    # written: rows in, pages out; read back: pages in, rows out
    both = n * (2 * 2 * hk * d * e + 2 * 2 * held + 4)
    if case["kind"] == "cache":
        return {"bytes": both, "flops": 4 * n * 2 * hk * d}
    return {"bytes": both + n * (2 * case["heads"] * d * e + 12), "flops": n * (8 * (case["heads"] + hk) + 8 * hk) * d}


def _rows(gen, n, heads, d, dtype):
    """Rows of unit variance in which one channel of 16 is three times as large as the others."""
    x = torch.randn((n, heads, d), generator=gen, device="cuda", dtype=torch.float32)
    x[..., ::16] *= 3.0
    return (x * (16 / 24) ** 0.5).to(DT[dtype])


def _positions(case):
    f = torch.arange(case["frame0"], case["frame0"] + case["frames"], device="cuda", dtype=torch.int32)
    y = torch.arange(case["tok_h"], device="cuda", dtype=torch.int32)
    x = torch.arange(case["tok_w"], device="cuda", dtype=torch.int32)
    return torch.stack(torch.meshgrid(f, y, x, indexing="ij"), dim=-1).reshape(-1, 3).contiguous()


def _pages(case, n_pages):
    shape = (n_pages, 2, case["kv_heads"], case["page"])
    if case["fp8"]:
        return (torch.zeros(shape + (case["head_dim"],), device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn),
                torch.full(shape, 127, device="cuda", dtype=torch.uint8))
    return torch.zeros(shape + (case["head_dim"],), device="cuda", dtype=DT[case["dtype"]]), None


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    host = random.Random(seed)
    d, hk, page = case["head_dim"], case["kv_heads"], case.get("page")
    s = dict(case=case)
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
        s["q"] = _rows(gen, sum(q), case["heads"], d, case["dtype"]) * 1.3
        data, scales = _pages(case, n_pages)
        for first in range(0, n_pages, 512):                          # what earlier writes left in the pages
            n = min(512, n_pages - first) * 2 * page
            x = _rows(gen, n, hk, d, case["dtype"]).view(-1, 2, page, hk, d).transpose(2, 3)
            if case["fp8"]:
                code, scales[first: first + 512] = _to_8_bits(x.float())
                data.view(torch.uint8)[first: first + 512] = code.view(torch.uint8)
            else:
                data[first: first + 512] = x
        starts = [0]
        for n in q:
            starts.append(starts[-1] + n)
        s.update(data=data, scales=scales, table=table.cuda(), q_start=torch.tensor(starts, dtype=torch.int32).cuda(),
                 kv_len=torch.tensor(kv, dtype=torch.int32).cuda(), max_q=max(q), max_kv=max(kv))
        # which sequence a row of queries is of, and which of its new tokens: the plain form's way back from padded chunks
        s["row_seq"] = torch.tensor([b for b, n in enumerate(q) for _ in range(n)]).cuda()
        s["row_in"] = torch.tensor([i for n in q for i in range(n)]).cuda()
    else:
        n, heads = _tokens(case), case.get("heads", 0)
        qkv = _rows(gen, n, heads + 2 * hk, d, case["dtype"])          # one q | k | v product's output
        s.update(q=qkv[:, :heads], k=qkv[:, heads: heads + hk], v=qkv[:, heads + hk:])
        if case["kind"] != "cache":
            gains = torch.randn((2, d), generator=gen, device="cuda") * 0.1 + 1.2
            s.update(gq=gains[0].to(DT[case["dtype"]]), gk=gains[1].to(DT[case["dtype"]]), pos=_positions(case))
        if case["kind"] != "norm":
            run_ = case["run"]                                         # tokens that lie one behind the other in a page
            n_pages = -(-n // run_) + 2
            order = list(range(n_pages))
            host.shuffle(order)
            slot = [order[t // run_] * page + (t % run_ if run_ > 1 else (t * 7) % page) for t in range(n)]
            if case["kind"] == "cache":
                for t in range(5, n, 61):                              # rows of padding, which go nowhere
                    slot[t] = -1
            data, scales = _pages(case, n_pages)
            s.update(data=data, scales=scales, slot=torch.tensor(slot, dtype=torch.int32).cuda(),
                     kept=torch.tensor([t for t in range(n) if slot[t] >= 0]).cuda())
    if own and case["kind"] != "norm":
        from paper_2505_21070_amd import binding
        s["cache"] = binding.KVCache(s["data"], s["scales"], dtype=case["dtype"])
    return s


# ---- plain forms

def _to_8_bits(x):
    """Codes and scale bytes of fp32 rows: the least factor 2^e, e >= -100, by which no finite value of the row is over 448."""
    a = x.abs()
    m, e = torch.frexp(torch.where(a < math.inf, a, 0.0).amax(-1))
    e = (e - 9 + (m > 0.875)).clamp(min=-100)
    y = torch.where(a < math.inf, torch.ldexp(x, -e.unsqueeze(-1)), math.nan)
    return y.to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _from_8_bits(code, scale):
    return torch.ldexp(code.float(), scale.unsqueeze(-1).to(torch.int32) - 127)


def _rotate(x, pos):
    d = x.shape[-1]
    c = d // 6
    n = torch.tensor([d // 2 - 2 * c, c, c], device=x.device)
    axis = torch.repeat_interleave(torch.arange(3, device=x.device), n, output_size=d // 2)
    i = torch.arange(d // 2, device=x.device) - (n.cumsum(0) - n)[axis]
    angle = pos.double()[:, axis] * THETA ** (-i.double() / n[axis])
    cos, sin = angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1).flatten(-2)


def _plain_norm(x, gain, pos):
    f = x.float()
    return _rotate(f * torch.rsqrt(f.square().mean(-1, keepdim=True) + EPS) * gain.float(), pos)


def _plain_write(s, k, v):
    """k, v: fp32 rows.  Those of padding go nowhere."""
    page, kept = s["case"]["page"], s["kept"]
    slot = s["slot"][kept].long()
    rows = torch.stack((k[kept], v[kept]), dim=1)                     # [tokens, 2, heads, head_dim]
    at = (slot // page, slice(None), slice(None), slot % page)
    if s["case"]["fp8"]:
        code, scale = _to_8_bits(rows)
        s["data"].view(torch.uint8)[at] = code.view(torch.uint8)
        s["scales"][at] = scale
    else:
        s["data"][at] = rows.to(s["data"].dtype)


def _plain_read(s):
    page = s["case"]["page"]
    slot = s["slot"].clamp(min=0).long()
    at = (slot // page, slice(None), slice(None), slot % page)
    if s["case"]["fp8"]:
        rows = _from_8_bits(s["data"].view(torch.uint8)[at].view(torch.float8_e4m3fn), s["scales"][at])
    else:
        rows = s["data"][at].float()
    rows = torch.where((s["slot"] >= 0).view(-1, 1, 1, 1), rows, 0.0).to(DT[s["case"]["dtype"]])
    return rows[:, 0], rows[:, 1]


def _plain_attend(s):
    c = s["case"]
    hk, d, n, keys = c["kv_heads"], c["head_dim"], s["max_q"], s["max_kv"]
    shared = c["heads"] // hk
    table = s["table"].long()
    held = s["data"].view(torch.uint8)[table].view(torch.float8_e4m3fn) if c["fp8"] else s["data"][table]
    held = _from_8_bits(held, s["scales"][table]) if c["fp8"] else held.float()
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
    return out.permute(0, 3, 1, 2, 4).reshape(c["seqs"], n, c["heads"], d)[s["row_seq"], s["row_in"]].to(DT[c["dtype"]])


def run(s):
    c = s["case"]
    if own:
        from paper_2505_21070_amd import binding
        if c["kind"] == "norm":
            q, k = binding.qk_norm_rope(s["q"], s["k"], s["gq"], s["gk"], s["pos"], rope_theta=THETA, eps=EPS)
            return {"q": q, "k": k}
        if c["kind"] == "attend":
            return {"out": s["cache"].attend(s["q"], s["q_start"], s["kv_len"], s["table"], s["max_q"], s["max_kv"], causal_group=c["group"])}
        out = {}
        if c["kind"] == "cache":
            s["cache"].write(s["k"], s["v"], s["slot"])
        else:
            out["q"] = s["cache"].write_qkv(s["q"], s["k"], s["v"], s["gq"], s["gk"], s["pos"], s["slot"], rope_theta=THETA, eps=EPS)
        out["k"], out["v"] = s["cache"].read(s["slot"])
        return out
    dt = DT[c["dtype"]]
    if c["kind"] == "norm":
        return {"q": _plain_norm(s["q"], s["gq"], s["pos"]).to(dt), "k": _plain_norm(s["k"], s["gk"], s["pos"]).to(dt)}
    if c["kind"] == "attend":
        return {"out": _plain_attend(s)}
    out = {}
    if c["kind"] == "cache":
        _plain_write(s, s["k"].float(), s["v"].float())
    else:
        out["q"] = _plain_norm(s["q"], s["gq"], s["pos"]).to(dt)
        _plain_write(s, _plain_norm(s["k"], s["gk"], s["pos"]), s["v"].float())
    out["k"], out["v"] = _plain_read(s)
    return out


# ---- the same from the definitions, in 64 bits

def _exact_norm(x, gain, pos):
    x = x.double()
    x = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * gain.double()
    d = x.shape[-1]
    sizes = [d // 2 - 2 * (d // 6), d // 6, d // 6]
    angles = []
    for axis, n in enumerate(sizes):
        per = torch.tensor([THETA ** (-i / n) for i in range(n)], dtype=torch.float64, device="cuda")
        angles.append(torch.outer(pos[:, axis].double(), per))
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), torch.cat(angles, dim=1))
    return torch.view_as_real(torch.view_as_complex(x.reshape(*x.shape[:-1], d // 2, 2)) * turn[:, None, :]).reshape(x.shape)


def _exact_8_bits(x):
    """Nearest values of 4 exponent and 3 fraction bits (ties to even) times the row's power of two."""
    top = x.abs().amax(-1, keepdim=True)
    power = torch.full_like(top, -100.0)
    power = torch.where(top > 0, torch.maximum(torch.ceil(torch.log2(top.clamp(min=1e-300) / 448)), power), power)
    power = torch.where((top > 0) & (top * torch.exp2(1 - power) <= 448) & (power > -100), power - 1, power)
    power = torch.where(top * torch.exp2(-power) > 448, power + 1, power)
    y = x * torch.exp2(-power)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step * torch.exp2(power)


def exact(case, seed):
    s = prepare(case, seed)
    d, hk = case["head_dim"], case["kv_heads"]
    if case["kind"] == "norm":
        return {"q": _exact_norm(s["q"], s["gq"], s["pos"]), "k": _exact_norm(s["k"], s["gk"], s["pos"])}
    if case["kind"] != "attend":
        out = {}
        rows = {"k": s["k"].double(), "v": s["v"].double()}
        if case["kind"] == "project":
            out["q"] = _exact_norm(s["q"], s["gq"], s["pos"])
            rows["k"] = _exact_norm(s["k"], s["gk"], s["pos"])
        live = (s["slot"] >= 0).double().view(-1, 1, 1)
        for name, x in rows.items():
            if case["fp8"] and not (name == "k" and case["kind"] == "project"):
                x = _exact_8_bits(x)
            # normalised keys beside a border of two codes fall on either side of it with the last bits of what came before: no one value
            out[name] = None if case["fp8"] and name == "k" and case["kind"] == "project" else x * live
        return out
    shared = case["heads"] // hk
    q_len, kv_len = _lengths(case)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    row = 0
    for b, (n, keys) in enumerate(zip(q_len, kv_len)):
        held = s["data"][s["table"][b].long()] if not case["fp8"] else s["data"].view(torch.uint8)[s["table"][b].long()].view(torch.float8_e4m3fn)
        held = held.float().double()
        if case["fp8"]:
            held = held * torch.exp2(s["scales"][s["table"][b].long()].double() - 127).unsqueeze(-1)
        held = held.permute(1, 2, 0, 3, 4).reshape(2, hk, -1, d)[:, :, :keys]
        ends = torch.tensor([_seen(i, n, keys, case["group"]) for i in range(n)], device="cuda")
        for h in range(case["heads"]):
            k, v = held[0, h // shared], held[1, h // shared]
            score = (s["q"][row: row + n, h].double() @ k.T) / d ** 0.5
            score = torch.where(torch.arange(keys, device="cuda")[None, :] < ends[:, None], score, torch.full((), -math.inf, dtype=torch.float64, device="cuda"))
            out[row: row + n, h] = torch.softmax(score, dim=-1) @ v
        row += n
    return {"out": out}
