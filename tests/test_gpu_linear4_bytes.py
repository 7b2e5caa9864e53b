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
