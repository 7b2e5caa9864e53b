"""Every key counts once.  Queries of zeros weigh all keys alike, and each key's value is one at one (key head, channel) alone, so a result times the number of keys
seen is a whole number, of a few dozen at most: how many of that channel's keys were seen.  A key that is lost or taken twice, at the border of a range, of a
unit of a plan, of a tile or of a page, moves one of them by 1, where all roundings together (the quotient's, half a step of the type) move it by less than 0.2."""
import pytest
import torch

from paged import HALF, TD
from paged_exact import Pages, ends_of, route

pytestmark = pytest.mark.gpu
STORES = [("bf16", False), ("bf16", True), ("f32", False), ("f32", True)]
# query heads, key heads, head_dim, sequences, new tokens of each, bound of the keys, group; what a bf16 call and an fp32 call are cut into (None: fp32 has no such blocks)
CASES = {
    "one token in ranges": (4, 4, 128, 1, 1, 15000, 1, "parts", "parts"),
    "one token of heads of 64": (8, 8, 64, 1, 1, 9000, 0, "parts", "parts"),
    "a few tokens of shared heads": (32, 4, 128, 1, 4, 15000, 1, "parts", "parts"),
    "tokens of many sequences": (4, 4, 128, 40, 1, 20000, 1, "runs", "parts"),
    "tokens of many sequences, heads of 64": (32, 8, 64, 30, 1, 20000, 0, "runs", "parts"),
    "a few tokens of many sequences": (16, 4, 128, 33, 5, 9000, 1, "runs", "parts"),
    "many short sequences": (4, 4, 128, 90, 1, 1500, 1, "", ""),
    "a chunk in ranges": (4, 4, 128, 1, 130, 5000, 1, "parts", "parts"),
    "a chunk of heads of 64 in ranges": (8, 8, 64, 1, 70, 5000, 0, "parts", "parts"),
    "chunks by frames in ranges": (4, 2, 128, 3, 150, 6000, 60, "parts", "parts"),
    "a wide block": (512, 64, 128, 1, 65, 2400, 0, "256", None),
    "a wide block in ranges": (64, 8, 128, 1, 254, 9000, 0, "256 parts", None),
    "a wide block, causal": (512, 64, 128, 1, 1024, 9600, 1, "256", None),
}


@pytest.mark.parametrize("name,dtype,fp8", [(name,) + s for name in CASES for s in STORES if s[0] == "bf16" or CASES[name][8] is not None])
def test_every_key_counts_once(name, dtype, fp8):
    hq, hk, d, seqs, n, bound, group, kind, kind32 = CASES[name]
    page, of = 32, hk * d

    def change(b, k, v):
        j = torch.arange(bound, device="cuda")
        v.zero_().view(bound, of)[j, j % of] = 1.0
    f = Pages([bound], hk, d, page, dtype, fp8, change=change)
    f.table = f.table.expand(seqs, -1).contiguous()                      # all sequences read the same pages, each up to its own length
    qb, parts, part, runs = route(dtype, d, hq, hk, seqs, seqs * n, n, bound, group, page)
    kind = kind if dtype == "bf16" else kind32
    assert ("256" not in kind or qb == 256) and ("parts" not in kind or parts > 2) and ("runs" not in kind or runs > 0)
    lens = {1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 95, 127, 128, 129, 255, 256, 257, 511, 512, 513, bound // 2, bound - 1, bound}
    for i in range(1, parts):
        lens |= {i * part + e for e in (-1, 0, 1, 31, 33, 64)}
    lens |= {128 * (i * i % (bound // 128)) + e for i in range(1, seqs) for e in (-1, 0, 1)}
    lens = sorted(x for x in lens if 0 < x <= bound)
    lens = [lens[(i * 17) % len(lens)] for i in range(len(lens))] if len(lens) % 17 else lens       # long ones beside short ones
    if "causal" in name:
        lens = [700, 1024, 1100, 3001, bound]
    q = torch.zeros((seqs * n, hq, d), dtype=TD[dtype], device="cuda")
    start = torch.arange(seqs + 1, dtype=torch.int32, device="cuda") * n
    first = torch.arange(of, device="cuda").view(hk, 1, d).expand(hk, hq // hk, d).reshape(hq, d)   # of each result, the first key that it counts
    for at in range(0, len(lens), seqs):
        now = (lens[at: at + seqs] + lens * seqs)[:seqs]
        out = f.cache.attend(q, start, torch.tensor(now, dtype=torch.int32, device="cuda"), f.table, n, bound, causal_group=group)
        for b, keys in enumerate(now):
            ends = ends_of(n, keys, group)[:, None, None]
            count = torch.clamp((ends - first + of - 1) // of, min=0)
            assert int(count.max()) <= 41
            seen = out[b * n: (b + 1) * n].double() * ends
            bad = (seen - count).abs() > count * (HALF[dtype] + 2.0 ** -22) * 1.01
            assert not bad.any(), (name, keys, torch.nonzero(bad)[:5].tolist(), seen[bad][:5].tolist(), count.expand_as(seen)[bad][:5].tolist())
