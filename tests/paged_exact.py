"""Attention over pages in 64 bits on the device, for shapes that are too large for the definition's loops; pinned to the definition in
test_gpu_attn_wide.py.  And which kind of block a call takes."""
import ctypes as C

import numpy as np
import torch

from paged import TD, attend_bound
from paper_2505_21070_amd import binding as B

_route = B._lib.dp_attn_paged_route
_route.argtypes, _route.restype = [C.c_void_p, C.c_void_p, C.c_int64, C.POINTER(C.c_int32)], None


def route(dtype, d, hq, hk, n_seqs, n, max_q, max_kv, group, page=64):
    """(rows of a block, ranges, keys of a range, runs of a plan) of a call with n new tokens in all."""
    out = (C.c_int32 * 4)()
    cache = B.KvCacheDesc(hk, d, page, 1, B.DP_BF16 if dtype == "bf16" else B.DP_F32, 0, 1 << 20, None)
    _route(bytes(cache), bytes(B.AttnConfig(hq, n_seqs, max_q, max_kv, -(-max_kv // page), group, 0.1)), n, out)
    return tuple(out)


def ends_of(n, keys, group, device="cuda"):
    """Keys that each of n new tokens sees."""
    p = keys - n + torch.arange(n, device=device)
    if group == 0:
        return torch.full_like(p, keys)
    return torch.where(p < 0, 0, torch.clamp((torch.div(p, group, rounding_mode="floor") + 1) * group, max=keys))


class Pages:
    """A cache whose sequences lie in pages of random order, made on the device; NaN in all free places.  k and v: what the pages hold, read back."""

    def __init__(self, keys, hk, d, page, dtype, fp8, seed=0, change=None, spare=2):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        need = [-(-n // page) for n in keys]
        n_pages = sum(need) + spare
        order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed))
        self.cache = B.KVCache.empty(n_pages, hk, page, d, dtype, fp8)
        self.cache.data.view(torch.uint8).fill_(0x7f if fp8 else 0xff)
        self.table = torch.full((len(keys), max(need + [1])), -1, dtype=torch.int32)
        self.k, self.v, self.keys, self.d, self.dtype, self.hk = [], [], list(keys), d, dtype, hk
        for b, n in enumerate(keys):
            own, order = order[: need[b]], order[need[b]:]
            self.table[b, : need[b]] = own.to(torch.int32)
            k, v = [(torch.randn((n, hk, d), generator=gen, device="cuda") * s).to(TD[dtype]) for s in (1.3, 1.0)]
            if change:
                change(b, k, v)
            at = torch.arange(n)
            slot = (own[at // page] * page + at % page).to(torch.int32).cuda()
            self.cache.write(k, v, slot)
            k, v = self.cache.read(slot)
            self.k.append(k)
            self.v.append(v)
        self.table = self.table.cuda()

    def attend(self, q, q_len, lens=None, group=0, max_q=None, max_kv=None, out=None):
        lens = self.keys if lens is None else lens
        start = np.concatenate([[0], np.cumsum(q_len)])
        put = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        return self.cache.attend(q, put(start), put(lens), self.table, max(q_len) if max_q is None else max_q, max(lens) if max_kv is None else max_kv,
                                 causal_group=group, out=out)


def exact(q, k, v, ends, scale, exists=None):
    """q [n, d], k and v [keys, d] of one head: (result, mean of |v| under the weights, largest sum of |q||k| * scale), in 64 bits."""
    q, k, v = q.double(), k.double(), v.double()
    hidden = torch.arange(k.shape[0], device="cuda")[None] >= ends[:, None]
    if exists is not None:
        hidden = hidden | ~exists[None]
    s = torch.where(hidden, -torch.inf, q @ k.T.contiguous() * scale)
    top = s.amax(1, keepdim=True) if k.shape[0] else torch.full((q.shape[0], 1), -torch.inf, dtype=torch.float64, device="cuda")
    w = torch.exp(s - torch.where(top == -torch.inf, 0.0, top))
    w = w / torch.where(top == -torch.inf, 1.0, w.sum(1, keepdim=True))
    fin = torch.where(torch.isfinite(v), v, 0.0)
    out, mean = w @ fin, w @ fin.abs()
    for bad in (torch.inf, -torch.inf, torch.nan):                       # a value that is not finite reaches who sees it
        is_bad = torch.isnan(v) if bad != bad else v == bad
        if is_bad.any():
            out = torch.where((s > -torch.inf).double() @ is_bad.double() > 0, out + bad, out)
    size = torch.where(hidden, 0.0, q.abs() @ k.abs().T.contiguous() * scale)
    return out, mean, size.amax(1) if k.shape[0] else torch.zeros(q.shape[0], dtype=torch.float64, device="cuda")


def check(f, q, got, q_len, lens=None, group=0, heads=None, exists=None):
    """The results of all rows of some query heads (all, unless named) at the bounds of paged.attend_bound."""
    lens = f.keys if lens is None else lens
    shared, at = q.shape[1] // f.hk, 0
    for b, n in enumerate(q_len):
        ends = ends_of(n, lens[b], group)
        for h in range(q.shape[1]) if heads is None else heads:
            keys = lens[b]
            ref, mean, size = exact(q[at: at + n, h], f.k[b][:keys, h // shared], f.v[b][:keys, h // shared], ends, f.d ** -0.5,
                                    None if exists is None else exists[b][:keys])
            ref, mean, size, g = (t.cpu().numpy() for t in (ref, mean, size, got[at: at + n, h].double()))
            fin = np.isfinite(ref)
            assert (np.isnan(g) == np.isnan(ref)).all() and (g[np.isinf(ref)] == ref[np.isinf(ref)]).all() and np.isfinite(g[fin]).all(), (b, h, lens[b])
            tol = attend_bound(np.where(fin, ref, 0.0), mean, size, f.d, max(keys, 1), f.dtype)
            bad = np.abs(np.where(fin, g - np.where(fin, ref, 0.0), 0.0)) > tol
            assert not bad.any(), (b, h, lens[b], np.argwhere(bad)[:4].tolist(), int(bad.sum()))
        at += n
