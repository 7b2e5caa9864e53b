"""Shared helpers of the tests of the paged cache: inputs, and comparison with the definitions in 64 bits at derived bounds."""
import numpy as np
import torch

from oracle import paged as O

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}          # half a step, relative
U = 2.0 ** -24
TD = {"bf16": torch.bfloat16, "f32": torch.float32}


def np64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def rows(gen, n, heads, d, dtype, scale=1.0):
    return (torch.randn((n, heads, d), generator=gen) * scale).to(TD[dtype])


def positions(n, gen, far=4000):
    return torch.stack([torch.randint(0, far, (n,), generator=gen), torch.randint(0, 45, (n,), generator=gen),
                        torch.randint(0, 80, (n,), generator=gen)], dim=1).to(torch.int32)


# fp32 work of a normalised, rotated value, in units of 2^-24 of its pair's length: sum of squares (12 roundings of positive terms, halved by
# the root) 6, root 2, two products 2, cosine and sine (angle 1.6 and function 4, of two terms) 8, products and sum 3: below 24
NORM_UNITS = 24


def pair_length(y):
    p = np.sqrt(y[..., 0::2] ** 2 + y[..., 1::2] ** 2)
    return np.repeat(p, 2, axis=-1)


def check_norm(got, x, gain, pos, theta, eps, dtype):
    ref = O.norm_rope(np64(x), np64(gain), pos.cpu().numpy(), theta, eps)
    err = np.abs(np64(got) - ref)
    tol = HALF[dtype] * np.abs(ref) * (1 + 2.0 ** -8) + NORM_UNITS * U * pair_length(ref)
    assert (err <= tol).all(), (float((err / np.maximum(tol, 1e-300)).max()), int((err > tol).sum()))


def attend_bound(ref, mean_abs, score_abs, d, keys, dtype):
    """Bound of |kernel - definition| for each output.  Scores: d products and sums in fp32 and the scale, at most (d + 4) * 2^-24 of the sum of
    |q||k|, and half that in the maximum's place: an exponent off by delta moves a weight by delta, relative, in numerator and denominator.  exp2 of an
    argument of size s: 2^-22 and the argument's own rounding, s * 2^-24 * 2.  Sums over the keys: keys * 2^-24 in either.  DP_BF16: every weight rounded to bf16, at most
    2^-8 in the numerator against the rounded denominator: 2 * 2^-8.  The result's own rounding."""
    delta = 2 * ((d + 4) * U * score_abs + 2.0 ** -22 + 4 * U * score_abs)[..., None]
    rel = 2 * delta + 2 * keys * U + (2 * 2.0 ** -8 if dtype == "bf16" else 8 * U)
    return mean_abs * rel * 1.01 + HALF[dtype] * np.abs(ref) * 1.01 + 1e-37


class Filled:
    """A cache on the device with sequences in pages of random order, and the same keys and values on the host."""

    def __init__(self, keys, kv_heads, d, page, dtype, fp8, seed=0, device="cuda", change=None, spare=3):
        from paper_2505_21070_amd import binding as B
        gen = torch.Generator().manual_seed(seed)
        rng = np.random.RandomState(seed)
        need = [-(-n // page) for n in keys]
        n_pages = sum(need) + spare
        order = rng.permutation(n_pages).tolist()
        width = max(need + [1])
        table = torch.full((len(keys), width), -7, dtype=torch.int32)        # what lies behind a sequence's pages is never looked at
        self.cache = B.KVCache.empty(n_pages, kv_heads, page, d, dtype, fp8, device)
        # what other sequences left in the pages: NaN
        self.cache.data.view(torch.uint8).fill_(0x7f if fp8 else 0xff)
        self.k, self.v = [], []
        for b, n in enumerate(keys):
            own, order = order[: need[b]], order[need[b]:]
            table[b, : need[b]] = torch.tensor(own, dtype=torch.int32)
            k, v = rows(gen, n, kv_heads, d, dtype, 1.3), rows(gen, n, kv_heads, d, dtype)
            if change:
                change(b, k, v)
            slot = torch.tensor([own[i // page] * page + i % page for i in range(n)], dtype=torch.int32, device=device)
            self.cache.write(k.to(device), v.to(device), slot)
            kr, vr = np64(k), np64(v)
            if fp8 and n:
                kr, vr = O.fp8_rows(kr)[0], O.fp8_rows(vr)[0]
            self.k.append(kr)
            self.v.append(vr)
        self.table, self.keys, self.d, self.dtype = table.to(device), list(keys), d, dtype


def attend_and_check(f, q, q_len, group=0, scale=None, extra_rows=0, exists=None, max_q=None, max_kv=None, **kw):
    """q: [sum(q_len) + extra_rows, heads, d] on the device."""
    start = np.concatenate([[0], np.cumsum(q_len)]).astype(int)
    scale = f.d ** -0.5 if scale is None else scale
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device=q.device)
    got = f.cache.attend(q, torch.tensor(start, dtype=torch.int32, device=q.device), torch.tensor(f.keys, dtype=torch.int32, device=q.device), f.table,
                         max(list(q_len) + [0]) if max_q is None else max_q, max(f.keys + [0]) if max_kv is None else max_kv, causal_group=group,
                         scale=scale, out=out, **kw)
    exists = [np.ones(n, bool) for n in f.keys] if exists is None else exists
    ref, mean_abs, score_abs = O.attend(np64(q), f.k, f.v, start, f.keys, exists, group, scale, np.full(q.shape, 7.0))
    g = np64(got)
    assert (g[start[-1]:] == 7.0).all(), "rows of no sequence are left alone"
    same = (np.isnan(g) == np.isnan(ref)) & (np.isinf(g) == np.isinf(ref))
    assert same.all(), np.argwhere(~same)[:5].tolist()
    fin = np.isfinite(ref)
    assert (g[~fin & ~np.isnan(ref)] == ref[~fin & ~np.isnan(ref)]).all()
    tol = attend_bound(ref, mean_abs, score_abs, f.d, max(f.keys + [1]), f.dtype)
    with np.errstate(invalid="ignore"):
        err = np.abs(g - ref)
    bad = fin & ~(err <= np.where(np.isfinite(tol), tol, np.inf))
    assert not bad.any(), (np.argwhere(bad)[:5].tolist(), float(err[bad].max()), int(bad.sum()))
    return got
