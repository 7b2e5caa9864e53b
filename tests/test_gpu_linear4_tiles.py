"""Products with 4-bit weights: every tile, and every tile that a call's inputs may be cut into ranges for, with real inputs, activations, all bits of fp32 and what is not
finite.  The sizes are those of test_every_tile, each of which one tile alone is chosen for."""
import numpy as np
import pytest
import torch

from oracle import fp4 as F
from paged import HALF, TD, U, np64
from test_gpu_linear4 import EVEN, REACH, check, kind_of

pytestmark = pytest.mark.gpu
TILES = [(d, k, REACH[d][k]) for d in REACH for k in REACH[d]] + EVEN


def matrix(out, in_, seed):
    """Codes and scales on the device, outputs of about unit size; some of its rows, first and last ones among them, and what they stand for."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(0, 256, (out, in_ // 2), generator=gen, device="cuda", dtype=torch.uint8)
    middle = 127 - round(np.log2(1.74 * in_ ** 0.5))
    scales = torch.randint(middle - 1, middle + 2, (out, in_ // 32), generator=gen, device="cuda", dtype=torch.uint8)
    rows = torch.cat([torch.arange(0, 64), torch.arange(out // 2 - 40, out // 2 + 40), torch.arange(max(0, out - 300), out)]).unique()

    def weights():
        return F.decode(F.unpack(codes[rows.cuda()].cpu().numpy()), scales[rows.cuda()].cpu().numpy())
    return codes, scales, rows, weights


def inputs(n, in_, dtype):
    x = torch.randn((n, in_), generator=torch.Generator().manual_seed(n)) * 0.3
    x[:, ::16] *= 7
    return x.to(TD[dtype])


@pytest.mark.parametrize("dtype,kind,sizes", TILES)
def test_against_the_definition(dtype, kind, sizes):
    from paper_2505_21070_amd import binding as B
    n, out, in_ = sizes
    assert kind_of(out, in_, dtype, n) == kind
    codes, scales, rows, weights = matrix(out, in_, n)
    w, x = weights(), inputs(n, in_, dtype)
    bias = torch.randn(out, generator=torch.Generator().manual_seed(out)).to(TD[dtype])
    m = B.Linear4(codes.view(torch.float4_e2m1fn_x2), scales, bias.cuda(), dtype)
    for act in (None, "gelu", "silu"):
        check(m.forward(x.cuda(), act=act)[:, rows.cuda()], x, w, bias[rows], act, dtype)


@pytest.mark.parametrize("dtype,kind,sizes", TILES)
def test_values_that_are_not_finite(dtype, kind, sizes):
    """In inputs of the first, the middle and the last token, and in a group of weights; the others as if they were not there."""
    from paper_2505_21070_amd import binding as B
    n, out, in_ = sizes
    assert kind_of(out, in_, dtype, n) == kind
    codes, scales, rows, weights = matrix(out, in_, n + 1)
    scales[out - 2, in_ // 32 - 1] = 255
    w, x = weights(), inputs(n, in_, dtype)
    special = {0: (in_ - 24, float("inf"))} if n == 1 else {0: (in_ - 24, float("inf")), n // 2: (3, float("nan")), n - 1: (130, -float("inf"))}
    for t, (i, v) in special.items():
        x[t, i] = v
    m = B.Linear4(codes.view(torch.float4_e2m1fn_x2), scales, None, dtype)
    x64, bad = np64(x), len(w) - 2
    assert int(rows[bad]) == out - 2 and np.isnan(w[bad]).any()
    with np.errstate(invalid="ignore", over="ignore"):
        y = np.where(np.isfinite(x64), x64, 0.0) @ np.nan_to_num(w).T
        for t, (i, v) in special.items():
            y[t] += v * w[:, i]                              # infinity times 0 is NaN
        y[:, bad] = np.nan
        ref = {None: y, "gelu": F.activation(y, "gelu")}
    # two halves of a rounding for each product of each part, and the groups' and ranges' sums, as in check(); the activation's slope is at most 1.13, its own work as there
    size = np.abs(np.where(np.isfinite(x64), x64, 0.0)) @ np.abs(np.nan_to_num(w)).T
    for act, want in ref.items():
        got = np64(m.forward(x.cuda(), act=act)[:, rows.cuda()])
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.isnan(got[:, bad]).all()
        inf = np.isinf(want)
        assert np.array_equal(got[inf], want[inf]) and inf[0].any()
        fine = np.isfinite(want)
        with np.errstate(invalid="ignore"):
            work = 2 * (in_ * (3 if dtype == "f32" else 1) + 12) * U * size * (1.13 if act else 1.0)
            if act:
                work = work + np.abs(want) * U * (6 + 4 * 2.31 * np.abs(y + 0.044715 * y ** 3))
            tol = HALF[dtype] * (np.abs(want) + work) + work + 1e-37
            assert (np.abs(got - want)[fine] <= tol[fine]).all()


@pytest.mark.parametrize("kind", REACH["f32"])
def test_all_bits_of_fp32_inputs(kind):
    """A weight of 1 for each output: it is its input, bit by bit, as far as bf16's exponents reach; then with NaNs that only their lower bits tell from infinity."""
    from paper_2505_21070_amd import binding as B
    n, out, in_ = REACH["f32"][kind]
    assert kind_of(out, in_, "f32", n) == kind
    at = (torch.arange(out, device="cuda") * 11 + 3) % in_     # 11 divides no number of inputs here: all of them, if there are so many outputs
    codes = torch.zeros((out, in_ // 2), dtype=torch.uint8, device="cuda")
    codes[torch.arange(out, device="cuda"), at // 2] = torch.where(at % 2 == 0, 0x02, 0x20).to(torch.uint8)
    m = B.Linear4(codes.view(torch.float4_e2m1fn_x2), torch.full((out, in_ // 32), 127, dtype=torch.uint8, device="cuda"), dtype="f32")
    gen = torch.Generator(device="cuda").manual_seed(n)
    bits = torch.randint(-2 ** 31, 2 ** 31, (n, in_), generator=gen, device="cuda").to(torch.int32)
    bits = bits & ~0x7f800000 | torch.randint(30, 254, (n, in_), generator=gen, device="cuda").to(torch.int32) << 23
    x = bits.view(torch.float32)
    assert torch.equal(m.forward(x), x[:, at])
    bits[0, 20] = 0x7f800001
    if n > 1:
        bits[n - 1, in_ - 1] = -0x7fffff
    y = m.forward(x)
    assert torch.isnan(y[0]).all() and torch.isnan(y[n - 1]).all() and torch.equal(y[1: n - 1], x[1: n - 1, at])
