"""Rows into and out of the paged cache in 4 bits, against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import fp4 as F
from oracle import paged as O
from paged import NORM_UNITS, TD, U, check_norm, np64, pair_length, positions, rows
from paged4 import codes_of

pytestmark = pytest.mark.gpu


def fused(gen, n, hq, hk, d, dtype):
    """q, k, v as views of one product's output."""
    x = rows(gen, n, hq + 2 * hk, d, dtype).cuda()
    return x[:, :hq], x[:, hq: hq + hk], x[:, hq + hk:]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,hk,d,page", [(1, 1, 64, 16), (1, 1, 128, 16), (9, 3, 128, 16), (70, 8, 64, 64), (40, 40, 128, 32), (300, 1, 128, 128), (3, 700, 64, 16)])
def test_write_and_read(n, hk, d, page, dtype):
    from paper_2505_21070_amd import binding as B
    gen = torch.Generator().manual_seed(n * hk)
    n_pages = -(-n // page) * 2 + 1
    cache = B.KVCache.empty(n_pages, hk, page, d, dtype, fp4=True)
    cache.data.view(torch.uint8).fill_(0x5a)
    cache.scales.fill_(99)
    _, k, v = fused(gen, n, 1, hk, d, dtype)
    k *= torch.exp2(torch.randint(-20, 20, (n, hk, d // 32), generator=gen).float()).repeat_interleave(32, -1).cuda().to(TD[dtype])
    slot = torch.randperm(n_pages * page, generator=gen)[:n].to(torch.int32)
    gone = [t for t in range(n) if t % 4 == 3]
    for j, t in enumerate(gone):
        slot[t] = [-1, n_pages * page, -2 ** 31, 2 ** 31 - 1][j % 4]
    cache.write(k, v, slot.cuda())
    kr, vr = cache.read(slot.cuda())
    for got, x in ((kr, k), (vr, v)):
        ref = F.rows(np64(x))[0]
        ref[gone] = 0.0
        assert np.array_equal(np64(got), ref)
    # in the layout that the tensors show, nothing else touched
    kept = [t for t in range(n) if t not in gone]
    page_of, at = slot[kept].numpy() // page, slot[kept].numpy() % page
    rest = np.ones((n_pages, 2, hk, page), bool)
    code, byte = codes_of(cache), cache.scales.cpu().numpy()
    for j, x in enumerate((k, v)):
        c, b = F.encode(np64(x)[kept])
        assert np.array_equal(byte[page_of, j, :, at], b) and np.array_equal(code[page_of, j, :, at], c)
        rest[page_of, j, :, at] = False
    assert (cache.data.view(torch.uint8).cpu().numpy()[rest] == 0x5a).all() and (byte[rest] == 99).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_at_the_ends_of_the_codes(dtype):
    from paper_2505_21070_amd import binding as B
    cache = B.KVCache.empty(2, 1, 16, 64, dtype, fp4=True)
    x = torch.zeros((14, 1, 64), dtype=TD[dtype])
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, -7.0])
    x[0, 0, :16] = ties
    x[1, 0, 16:32], x[1, 0, 32:48] = ties * 2.0 ** 20, ties * 2.0 ** -60
    x[2, 0, :3] = torch.tensor([7.03125, 3.515625, -0.25])                 # just beyond 7: the next power
    x[3, 0, 5], x[3, 0, 40] = float("nan"), 3.0                            # one group of two
    x[4, 0, :2] = torch.tensor([float("inf"), 1.0])
    x[5, 0, 31], x[5, 0, 32] = -float("inf"), -1.0
    x[6] = float("nan")
    x[7, 0, :2] = torch.tensor([torch.finfo(TD[dtype]).max, -1e38])
    x[8, 0, :3] = torch.tensor([1.75 * 2.0 ** 127, 2.0 ** 127, -2.0 ** 125])
    x[9, 0, :3] = torch.tensor([1.765625 * 2.0 ** 127, 2.0 ** 127, -2.0 ** 125])
    x[10, 0, :4] = torch.tensor([2.0 ** -100, 2.0 ** -101, 2.0 ** -102, 1.5 * 2.0 ** -102])
    x[11, 0, :2] = torch.tensor([2.0 ** -126, 2.0 ** -133])
    x[12, 0, ::2], x[12, 0, 1::2] = -0.0, 0.0
    x[13, 0, :] = torch.arange(64).float() * 0.0625 + 1
    slot = torch.arange(14, dtype=torch.int32, device="cuda")
    cache.write(x.cuda(), x.flip(0).contiguous().cuda(), slot)
    k, v = cache.read(slot)
    ref = F.rows(np64(x))[0]
    assert np.isfinite(ref[7:10]).all() and np.isnan(ref[3, 0, :32]).all() and np.isfinite(ref[3, 0, 32:]).all()
    assert np.array_equal(np64(k), ref, equal_nan=True)
    assert np.array_equal(np64(v), ref[::-1], equal_nan=True)
    assert np.array_equal(cache.scales.cpu().numpy()[0, 0, 0, :14], F.encode(np64(x))[1][:, 0])
    assert np.array_equal(codes_of(cache)[0, 0, 0, :14], F.encode(np64(x))[0][:, 0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,hq,hk,d", [(1, 12, 12, 128), (5, 3, 1, 128), (7, 16, 4, 64), (33, 40, 8, 128), (257, 5, 5, 64)])
def test_write_qkv(n, hq, hk, d, dtype):
    from paper_2505_21070_amd import binding as B
    gen = torch.Generator().manual_seed(n + 3)
    q, k, v = fused(gen, n, hq, hk, d, dtype)
    gq, gk = [(torch.randn(d, generator=gen) * 0.2 + 1).to(TD[dtype]).cuda() for _ in range(2)]
    pos = positions(n, gen).cuda()
    n_pages = -(-n // 16) + 1
    cache = B.KVCache.empty(n_pages, hk, 16, d, dtype, fp4=True)
    slot = torch.randperm(n_pages * 16, generator=gen)[:n].to(torch.int32)
    if n > 2:
        slot[n // 2] = -1
    qo = cache.write_qkv(q, k, v, gq, gk, pos, slot.cuda())
    kr, vr = cache.read(slot.cuda())
    apart, _ = B.qk_norm_rope(q, k, gq, gk, pos)
    assert torch.equal(qo, apart)
    check_norm(qo, q, gq, pos, 1e4, float(np.float32(1e-6)), dtype)
    kept = slot.numpy() >= 0
    assert (np64(kr)[~kept] == 0).all() and (np64(vr)[~kept] == 0).all()
    assert np.array_equal(np64(vr)[kept], F.rows(np64(v))[0][kept])
    rk = O.norm_rope(np64(k), np64(gk), pos.cpu().numpy(), 1e4, float(np.float32(1e-6)))
    # half the step around the value, in units of the group's power: 0.5 up to 2, 1 up to 4, 2 beyond.  The work's error moves a value by at most `work` before it is
    # rounded, and where the group's largest value lies within it of 7 * 2^e, the power is one lower, with smaller steps but for values in (6, 7] * 2^e (one
    # more unit of the lower power: no more than half of the higher one's last step, which the bound has), or one higher: steps twice as wide
    work = NORM_UNITS * U * pair_length(rk)
    e = F.power(rk)
    top = np.abs(F.groups(rk)).max(-1)
    e = np.where(top + F.groups(work).max(-1) > 7 * 2.0 ** e, e + 1, e).repeat(32, -1).reshape(rk.shape)
    y = (np.abs(rk) + work) / 2.0 ** e
    step = np.where(y <= 2, 0.5, np.where(y <= 4, 1.0, 2.0))
    assert (np.abs(np64(kr) - rk)[kept] <= (step / 2 * 2.0 ** e + work)[kept]).all()


def test_write_qkv_in_place_of_the_queries_and_no_tokens():
    from paper_2505_21070_amd import binding as B
    gen = torch.Generator().manual_seed(8)
    q, k, v = fused(gen, 21, 4, 2, 128, "bf16")
    g = torch.ones(128, dtype=torch.bfloat16, device="cuda")
    pos, slot = positions(21, gen).cuda(), torch.arange(21, dtype=torch.int32, device="cuda")
    a, b = [B.KVCache.empty(2, 2, 16, 128, "bf16", fp4=True) for _ in range(2)]
    qo = a.write_qkv(q, k, v, g, g, pos, slot)
    assert b.write_qkv(q, k, v, g, g, pos, slot, q_out=q) is q
    assert torch.equal(q, qo) and torch.equal(a.data.view(torch.uint8), b.data.view(torch.uint8)) and torch.equal(a.scales, b.scales)
    none, empty = k[:0], slot[:0]
    before = a.data.view(torch.uint8).clone()
    a.write(none, none, empty)
    assert [t.shape for t in a.read(empty)] == [(0, 2, 128)] * 2 and torch.equal(a.data.view(torch.uint8), before)


def test_a_pool_beyond_32_bits():
    """The last pages of a pool of more than 2^32 bytes of codes."""
    from paper_2505_21070_amd import binding as B
    page, hk, d = 64, 8, 128
    n_pages = (1 << 33) // (2 * hk * page * d // 2) + 3
    cache = B.KVCache.empty(n_pages, hk, page, d, "bf16", fp4=True)
    gen = torch.Generator().manual_seed(9)
    k, v = rows(gen, 4, hk, d, "bf16"), rows(gen, 4, hk, d, "bf16")
    slot = torch.tensor([n_pages * page - 1, n_pages * page - page, 0, (n_pages // 2) * page + 3], dtype=torch.int32, device="cuda")
    cache.write(k.cuda(), v.cuda(), slot)
    kr, vr = cache.read(slot)
    assert np.array_equal(np64(kr), F.rows(np64(k))[0]) and np.array_equal(np64(vr), F.rows(np64(v))[0])
    # and read by attention: the last page alone, its last key and the page's first one seen, keys between hold zeros
    q = rows(gen, 1, hk, d, "bf16").cuda()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    out = cache.attend(q, i32(0, 1), i32(page), i32([n_pages - 1]), 1, page)
    kk, vv = np.zeros((page, hk, d)), np.zeros((page, hk, d))
    kk[[-1, 0]], vv[[-1, 0]] = np64(kr)[:2], np64(vr)[:2]
    ref = O.attend(np64(q), [kk], [vv], [0, 1], [page], [np.ones(page, bool)], 0, d ** -0.5, np64(q))[0]
    assert np.abs(np64(out) - ref).max() <= 3 * 2.0 ** -8 * np.abs(vv).max()


def test_refused_by_the_binding():
    from paper_2505_21070_amd import binding as B
    cache = B.KVCache.empty(2, 2, 16, 64, "bf16", fp4=True)
    assert cache.head_dim == 64 and cache.data.dtype == torch.float4_e2m1fn_x2 and cache.scales.shape == (2, 2, 2, 16, 2)
    for data, scales, dtype in ((cache.data, None, "bf16"), (cache.data, cache.scales, None), (cache.data, cache.scales[..., 0].contiguous(), "bf16"),
                                (cache.data, cache.scales.float(), "bf16"), (cache.data.view(torch.uint8), cache.scales, "bf16")):
        with pytest.raises(AssertionError):
            B.KVCache(data, scales, dtype)
    with pytest.raises(AssertionError):
        B.KVCache.empty(2, 2, 16, 64, "bf16", fp8=True, fp4=True)
    x = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    slot = torch.zeros(3, dtype=torch.int32, device="cuda")
    for k, v, s in ((x.float(), x, slot), (x, x[:2], slot), (x, x, slot.long()), (x[..., :32], x, slot)):
        with pytest.raises(AssertionError):
            cache.write(k, v, s)
