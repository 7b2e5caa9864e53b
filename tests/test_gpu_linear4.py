"""Products with 4-bit weights on the GPU, against the definition in 64 bits."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import fp4 as F
from paged import HALF, TD, U, np64

pytestmark = pytest.mark.gpu
# tokens, out, in: each kernel and its tiles' borders, one group, rows that divide nothing, long sums
# (test_every_tile: which)
SIZES = [(1, 1, 32), (1, 16, 64), (1, 17, 96), (1, 4608, 1536), (2, 33, 256), (3, 100, 288), (15, 64, 512), (16, 48, 2080), (17, 31, 160), (32, 130, 4128), (33, 129, 544), (48, 80, 1024), (64, 65, 320),
         (65, 64, 128), (65, 1, 32), (70, 257, 96), (100, 300, 992), (128, 256, 256), (129, 255, 160), (200, 513, 1504), (260, 70, 64), (513, 129, 416), (1000, 24, 2048)]


def matrix(out, in_, seed=0, scale_bits=4):
    """(Linear4's codes and scales, the values they stand for)"""
    gen = torch.Generator().manual_seed(seed)
    codes = torch.randint(0, 256, (out, in_ // 2), generator=gen).to(torch.uint8)
    scales = torch.randint(127 - scale_bits, 128 + scale_bits, (out, in_ // 32), generator=gen).to(torch.uint8)
    return codes.cuda().view(torch.float4_e2m1fn_x2), scales.cuda(), F.decode(F.unpack(codes.numpy()), scales.numpy())


def check(got, x, w, bias, act, dtype):
    """Sums: one rounding (or a truncation, two halves) for each product of each part and for the wavefronts' sums and the bias; sizes of an input's parts
    are its own.  The activation's slope is at most 1.13; its own work: the exponent's argument, 4 roundings, moves the result by its size, function, reciprocal, product 6."""
    ref, y, size = F.linear(np64(x), w, None if bias is None else np64(bias), act)
    adds = w.shape[1] * (3 if dtype == "f32" else 1) + 12
    work = 2 * adds * U * size * (1.13 if act else 1.0)
    if act:
        arg = np.abs(y) * 1.45 if act == "silu" else 2.31 * np.abs(y + 0.044715 * y ** 3)
        work = work + np.abs(ref) * U * (6 + 4 * arg)
    err, tol = np.abs(np64(got) - ref), HALF[dtype] * (np.abs(ref) + work) + work + 1e-37
    assert got.shape == ref.shape and (err <= tol).all(), (np.argwhere(err > tol)[:4].tolist(), float((err / tol).max()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,out,in_", SIZES)
def test_against_the_definition(n, out, in_, dtype):
    from paper_2505_21070_amd import binding as B
    codes, scales, w = matrix(out, in_, seed=n + out)
    gen = torch.Generator().manual_seed(n)
    x = (torch.randn((n, in_), generator=gen) * 0.3).to(TD[dtype])
    x[:, ::16] *= 7
    bias = torch.randn(out, generator=gen).to(TD[dtype]).cuda()
    for b, act in ((None, None), (bias, "gelu"), (bias, "silu")):
        m = B.Linear4(codes, scales, b, dtype)
        check(m.forward(x.cuda(), act=act), x, w, b, act, dtype)


# each tile, and each that a call's inputs may be cut into ranges for: number, ranges -> a call that takes it, with ends that divide nothing
REACH = {
    "bf16": {(0, 1): (1, 500, 1504), (0, 4): (1, 1500, 8992), (0, 8): (1, 500, 8992), (1, 1): (1, 2900, 8992), (2, 1): (1, 8801, 2016), (2, 4): (1, 2900, 13792), (3, 1): (17, 4505, 1504),
             (3, 4): (17, 1500, 8992), (4, 1): (17, 8801, 1504), (4, 2): (17, 4505, 13792), (4, 8): (33, 1001, 13792), (5, 1): (65, 3333, 1504), (6, 1): (33, 8801, 2016), (6, 4): (81, 1500, 13792),
             (7, 1): (50, 8801, 1504), (8, 1): (33, 20001, 1504), (8, 2): (33, 20001, 13792), (8, 8): (33, 2900, 8992), (9, 1): (49, 20001, 992), (9, 2): (49, 8801, 8992),
             (10, 1): (65, 20001, 992), (10, 4): (65, 6601, 13792), (10, 8): (65, 3333, 13792), (11, 1): (450, 11001, 992), (12, 1): (300, 20001, 992), (13, 1): (333, 20001, 992),
             (14, 1): (400, 20001, 992), (15, 1): (500, 20001, 992), (16, 1): (1000, 11001, 992), (17, 1): (700, 20001, 992)},
    "f32": {(0, 1): (1, 500, 1504), (0, 8): (1, 500, 8992), (1, 1): (1, 4505, 1504), (1, 8): (1, 500, 4000), (2, 1): (1, 8801, 1504), (2, 4): (1, 2900, 13792), (3, 1): (17, 8801, 992),
            (3, 8): (17, 1500, 13792), (4, 1): (17, 20001, 1504), (4, 2): (17, 8801, 1504), (4, 8): (33, 1500, 4000), (5, 1): (33, 20001, 992), (5, 4): (65, 3333, 2016), (6, 1): (600, 5003, 992),
            (6, 2): (49, 20001, 4000), (6, 8): (1, 8801, 8992), (7, 4): (33, 20001, 4000), (7, 8): (33, 2900, 5088), (8, 1): (49, 20001, 1504), (9, 1): (161, 11001, 992),
            (10, 1): (257, 11001, 2016), (11, 1): (193, 20001, 992), (12, 1): (300, 20001, 992)},
}
# rows that end with a whole eight: the tiles that go through LDS on their way out
EVEN = [("bf16", (11, 1), (450, 11000, 992)), ("bf16", (12, 1), (300, 20000, 992)), ("bf16", (13, 1), (333, 20000, 992)), ("bf16", (14, 1), (400, 20000, 992)),
        ("bf16", (15, 1), (500, 20000, 992)), ("bf16", (16, 1), (1000, 11000, 992)), ("bf16", (17, 1), (700, 20000, 992)), ("f32", (12, 1), (300, 20000, 992))]


def kind_of(out, in_, dtype, n):
    from paper_2505_21070_amd import binding as B
    got = (C.c_int32 * 2)()
    B._lib.dp_linear_fp4_route(bytes(B.Fp4Matrix(out, in_, int(dtype == "bf16"), None, None)), C.c_int64(n), got)
    return tuple(got)


@pytest.mark.parametrize("dtype,kind,sizes", [(d, k, REACH[d][k]) for d in REACH for k in REACH[d]] + EVEN)
def test_every_tile(dtype, kind, sizes):
    """Whole numbers through each kind of tile, exact; its first and last outputs, tokens and inputs among them."""
    from paper_2505_21070_amd import binding as B
    n, out, in_ = sizes
    assert kind_of(out, in_, dtype, n) == kind
    gen = torch.Generator().manual_seed(n)
    codes = torch.randint(0, 256, (out, in_ // 2), generator=gen).to(torch.uint8)
    scales = torch.randint(126, 128, (out, in_ // 32), generator=gen).to(torch.uint8)
    x = torch.randint(-2, 3, (n, in_), generator=gen).to(TD[dtype])
    bias = torch.randint(-8, 8, (out,), generator=gen).to(TD[dtype])
    y = torch.full((n + 1, out + 8), 99.0, dtype=TD[dtype], device="cuda")
    m = B.Linear4(codes.cuda().view(torch.float4_e2m1fn_x2), scales.cuda(), bias.cuda(), dtype)
    for to in (None, y[:n, :out]):
        got = m.forward(x.cuda(), out=to)
        for rows in (slice(0, 64), slice(out // 2 - 40, out // 2 + 40), slice(max(0, out - 300), out)):
            w = torch.from_numpy(F.decode(F.unpack(codes[rows].numpy()), scales[rows].numpy()))
            want = x.double() @ w.T + bias[rows].double()
            assert want.abs().max() < 2 ** 20 and torch.equal(got[:, rows].cpu(), want.float().to(TD[dtype]))
    assert (y[n] == 99).all() and (y[:, out:] == 99).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,out,in_", SIZES + [(7, 512, 13824), (90, 300, 13824)])
def test_whole_numbers_are_exact(n, out, in_, dtype):
    """Small whole numbers: every sum is exact, so every input is there once, and nothing else."""
    from paper_2505_21070_amd import binding as B
    codes, scales, w = matrix(out, in_, seed=n, scale_bits=1)
    x = torch.randint(-3, 4, (n, in_), generator=torch.Generator().manual_seed(out)).to(TD[dtype])
    got = B.Linear4(codes, scales, None, dtype).forward(x.cuda())
    want = torch.from_numpy(np64(x) @ w.T)
    assert want.abs().max() < 2 ** 20
    assert torch.equal(got.cpu(), want.float().to(TD[dtype]))


@pytest.mark.parametrize("n", [1, 20, 64, 65, 130])
def test_all_bits_of_fp32_inputs(n):
    """One weight of 1 at a time: the output is the input, bit by bit, as far as bf16's exponents reach."""
    from paper_2505_21070_amd import binding as B
    in_ = 160
    code = np.zeros((in_, in_), int)
    code[np.arange(in_), np.arange(in_)] = 2
    codes = torch.from_numpy((code[:, 0::2] | code[:, 1::2] << 4).astype(np.uint8)).cuda().view(torch.float4_e2m1fn_x2)
    m = B.Linear4(codes, torch.full((in_, in_ // 32), 127, dtype=torch.uint8, device="cuda"), dtype="f32")
    bits = torch.randint(-2 ** 31, 2 ** 31, (n, in_), generator=torch.Generator().manual_seed(n)).to(torch.int32)
    bits = bits & ~0x7f800000 | torch.randint(30, 254, (n, in_), generator=torch.Generator().manual_seed(1)).to(torch.int32) << 23
    x = bits.view(torch.float32)
    # other inputs of the row are up to 2^97 times as large, and multiplied by 0
    assert torch.equal(m.forward(x.cuda()).cpu(), x)


@pytest.mark.parametrize("n", [1, 17, 64, 65, 140])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_that_are_not_finite(dtype, n):
    from paper_2505_21070_amd import binding as B
    out, in_ = 40, 224
    codes, scales, w = matrix(out, in_, seed=3)
    scales[5, 6] = 255
    w[5, 192:] = np.nan
    x = torch.randn((n, in_), generator=torch.Generator().manual_seed(2)).to(TD[dtype])
    at = [0] if n == 1 else [0, n // 2, n - 1]
    for j, t in enumerate(at):
        x[t, 200 if j == 0 else 3] = [float("inf"), float("nan"), -float("inf")][j]
    got = np64(B.Linear4(codes, scales, None, dtype).forward(x.cuda()))
    with np.errstate(invalid="ignore"):
        ref = np64(x) @ w.T
        products = np64(x)[:, None, :] * w[None]
        ref = np.where(np.isnan(products).any(-1), np.nan, ref)
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    inf = np.isinf(ref)
    assert np.array_equal(got[inf], ref[inf]) and inf.any() and np.isnan(got[:, 5]).all()
    fine = np.isfinite(ref)
    size = (np.abs(np.where(np.isfinite(np64(x)), np64(x), 0)) @ np.abs(np.nan_to_num(w)).T)[fine]          # see check()
    assert (np.abs(got[fine] - ref[fine]) <= HALF[dtype] * np.abs(ref[fine]) * (1 + 2.0 ** -7) + 2 * (3 * in_ + 12) * U * size).all()


@pytest.mark.parametrize("n", [1, 40, 300])
def test_every_nan_is_one(n):
    """fp32 NaNs that only their lower bits tell from infinity, beside a weight of 1 and one of 0."""
    from paper_2505_21070_amd import binding as B
    codes = torch.zeros((2, 64), dtype=torch.uint8, device="cuda")
    codes[0, 10] = 0x02                                    # output 0 takes input 20, output 1 nothing
    m = B.Linear4(codes.view(torch.float4_e2m1fn_x2), torch.full((2, 4), 127, dtype=torch.uint8, device="cuda"), dtype="f32")
    x = torch.zeros((n, 128))
    x.view(torch.int32)[0, 20], x.view(torch.int32)[n - 1, 21] = 0x7f800001, -0x7fffff
    y = m.forward(x.cuda())
    assert torch.isnan(y[0]).all() and torch.isnan(y[n - 1]).all() and (y[1: n - 1] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 5, 40, 65, 300])
def test_strides_and_what_lies_around(n, dtype):
    from paper_2505_21070_amd import binding as B
    out, in_ = 77, 288
    codes, scales, w = matrix(out, in_, seed=9)
    m = B.Linear4(codes, scales, None, dtype)
    gen = torch.Generator().manual_seed(4)
    wide = torch.full((n + 2, in_ + 64), float("nan"), dtype=TD[dtype], device="cuda")
    x = wide[1: n + 1, 32: 32 + in_]
    x.copy_(torch.randn((n, in_), generator=gen))
    plain = m.forward(x.contiguous())
    assert torch.equal(m.forward(x), plain)
    y = torch.full((n + 2, out + 5), 7.0, dtype=TD[dtype], device="cuda")
    assert m.forward(x, out=y[1: n + 1, 3: 3 + out]) .data_ptr() == y[1:, 3:].data_ptr()
    assert torch.equal(y[1: n + 1, 3: 3 + out], plain)
    y[1: n + 1, 3: 3 + out] = 7.0
    assert (y == 7).all()
    # one row as every token
    assert torch.equal(m.forward(x[:1].expand(n, in_)), plain[:1].expand(n, out)) if n > 1 else True


def test_pack():
    from paper_2505_21070_amd import binding as B
    for dtype in ("bf16", "f32"):
        for out, in_ in ((1, 32), (7, 96), (300, 1504), (33, 64)):
            w = torch.randn((out, in_ + 8), generator=torch.Generator().manual_seed(out)) * 2.0 ** torch.randint(-30, 30, (out, 1), generator=torch.Generator().manual_seed(1)).float()
            w = w.to(TD[dtype])
            w[0, :3] = torch.tensor([1e38, -0.0, 1e-38])
            if out > 1:
                w[1, 31], w[2, 5] = float("nan"), -float("inf")
            codes, scales = B.pack_fp4(w.cuda()[:, :in_])
            code, byte = F.encode(np64(w[:, :in_]))
            assert np.array_equal(F.unpack(codes.view(torch.uint8).cpu().numpy()), code) and np.array_equal(scales.cpu().numpy(), byte)
            m = B.Linear4.pack(w.cuda()[:, :in_])
            assert m.torch_dtype == TD[dtype] and (m.out, m.in_) == (out, in_) and torch.equal(m.laid, B.Linear4(codes, scales, dtype=dtype).laid)


@pytest.mark.parametrize("n", [1, 30, 200])
def test_captured_and_replayed_and_repeated(n):
    from paper_2505_21070_amd import binding as B
    codes, scales, _ = matrix(700, 1024)
    m = B.Linear4(codes, scales, None, "bf16")
    x = torch.randn((n, 1024), device="cuda").bfloat16()
    y = m.forward(x)
    assert torch.equal(m.forward(x), y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.forward(x, act="gelu", out=y)
    for k in range(4):
        x.mul_(1.25)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(m.forward(x, act="gelu"), y)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    z = m.forward(x, act="gelu", stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(z, y)
    assert m.forward(x[:0]).shape == (0, 700)


def test_codes_beyond_32_bits():
    """A matrix of more than 2^32 bytes of codes: its last outputs."""
    from paper_2505_21070_amd import binding as B
    in_, out = 1 << 16, (1 << 17) + 300
    codes = torch.zeros((out, in_ // 2), dtype=torch.uint8, device="cuda")
    scales = torch.full((out, in_ // 32), 127, dtype=torch.uint8, device="cuda")
    codes[-1, -1], codes[-2, 0] = 0x20, 0x02
    m = B.Linear4(codes.view(torch.float4_e2m1fn_x2), scales)
    del codes, scales
    for n in (1, 70):
        x = torch.zeros((n, in_), dtype=torch.bfloat16, device="cuda")
        x[:, -1], x[:, 0] = 3.0, 5.0
        y = m.forward(x)
        assert (y[:, -1] == 3).all() and (y[:, -2] == 5).all() and (y[:, :-2] == 0).all()


def test_refused_by_the_binding():
    from paper_2505_21070_amd import binding as B
    codes, scales, _ = matrix(8, 64)
    m = B.Linear4(codes, scales)
    x = torch.zeros((3, 64), dtype=torch.bfloat16, device="cuda")
    for bad in ((codes.view(torch.uint8), scales), (codes, scales[:, :1].contiguous()), (codes, scales.float()), (codes.cpu(), scales), (codes, scales, torch.zeros(7, device="cuda").bfloat16()),
                (codes, scales, torch.zeros(8, device="cuda"))):
        with pytest.raises(AssertionError):
            B.Linear4(*bad)
    for bad in (x.float(), x[:, :32], x.cpu(), x.t().contiguous().t()):
        with pytest.raises(AssertionError):
            m.forward(bad)
    with pytest.raises(AssertionError):
        m.forward(x, out=torch.zeros((3, 9), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(KeyError):
        m.forward(x, act="relu")
    with pytest.raises(B.DualParalError) as e:
        m.forward(torch.zeros((3, 68), dtype=torch.bfloat16, device="cuda")[:, 4:])
    assert e.value.code == B.DP_EINVAL and "16-byte" in str(e.value)
    for w in (torch.zeros((4, 40), device="cuda"), torch.zeros((64, 4), device="cuda").t(), torch.zeros((4, 64), device="cuda").half()):
        with pytest.raises(AssertionError):
            B.pack_fp4(w)
