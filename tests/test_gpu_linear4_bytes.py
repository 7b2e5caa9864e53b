"""Matrices of 4-bit weights from elsewhere: every byte that a group may have, with every code."""
import numpy as np
import pytest
import torch

from oracle import fp4 as F
from paged import TD, np64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 50, 300])
def test_every_byte_with_every_code(n, dtype):
    """A group for each byte and code, that code in it once, among zeros: weights below 2^-126 keep their bits, groups with one of 2^128 or more are NaN."""
    from paper_2505_21070_amd import binding as B
    of = np.arange(4096)
    code = np.zeros((4096, 32), int)
    code[of, of * 7 % 32] = of % 16
    byte = (of // 16)[:, None]
    w = F.decode(code, byte)[of, of * 7 % 32]
    w = np.where(np.abs(w) >= 2.0 ** 128, np.nan, w)
    codes = torch.from_numpy((code[:, 0::2] | code[:, 1::2] << 4).astype(np.uint8)).cuda().view(torch.float4_e2m1fn_x2)
    m = B.Linear4(codes, torch.from_numpy(byte.astype(np.uint8)).cuda(), dtype=dtype)
    x = torch.ones((n, 32), dtype=TD[dtype], device="cuda")
    x[1::2] = 0.5
    got, want = np64(m.forward(x)), w[None] * np64(x)[:, :1]
    wrong = ~((got == want) | (np.isnan(got) & np.isnan(want)))
    assert not wrong.any(), (np.unique(np.argwhere(wrong)[:, 1] // 16).tolist(), got[wrong][:4], want[wrong][:4])


@pytest.mark.parametrize("byte", [0, 1, 253, 254])
def test_groups_of_zeros(byte):
    """Zeros of either sign, whatever their factor, also beside large inputs."""
    from paper_2505_21070_amd import binding as B
    codes = torch.tensor([0x80, 0x08, 0, 0x88], dtype=torch.uint8).repeat(40 * 48 // 4).view(40, 48).cuda()
    m = B.Linear4(codes.view(torch.float4_e2m1fn_x2), torch.full((40, 3), byte, dtype=torch.uint8, device="cuda"))
    assert (m.forward(torch.full((5, 96), 3e38, device="cuda").bfloat16()) == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_and_groups_beside_one_another(dtype):
    """Groups of all factors beside one another: those that are NaN are so by themselves."""
    from paper_2505_21070_amd import binding as B
    out, in_ = 301, 224
    rng = np.random.RandomState(5)
    code, byte = rng.randint(0, 16, (out, in_)), rng.choice([0, 1, 2, 126, 127, 251, 252], (out, in_ // 32))
    for row in range(0, out, 3):                               # a high factor: for codes that stay finite with it, but in every sixth row
        g, b = rng.randint(in_ // 32), rng.choice([253, 254])
        byte[row, g] = b
        own = code[row, g * 32: g * 32 + 32]
        own[:] = np.where(own & 7 >= (6 if b == 253 else 4), own & 8 | 3, own)
        if row % 2 == 0:
            own[rng.randint(32)] = rng.choice([6, 7, 14, 15] if b == 253 else [4, 5, 6, 7, 12, 15])
    w = F.decode(code, byte)
    w = np.where((np.abs(w) >= 2.0 ** 128).reshape(out, -1, 32).any(-1).repeat(32, 1), np.nan, w)
    codes = torch.from_numpy((code[:, 0::2] | code[:, 1::2] << 4).astype(np.uint8)).cuda().view(torch.float4_e2m1fn_x2)
    m = B.Linear4(codes, torch.from_numpy(byte.astype(np.uint8)).cuda(), dtype=dtype)
    got = np64(m.forward(torch.eye(in_, dtype=TD[dtype], device="cuda")))
    want = np.where(np.isnan(w).any(1)[None], np.nan, w.T)
    assert 0 < np.isnan(want[0]).sum() < out // 3 and np.array_equal(got, want, equal_nan=True)
