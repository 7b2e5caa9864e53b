"""Pins of the fp64 definitions around the paged cache against library routines and by hand."""
import numpy as np
import pytest
import torch

from oracle import paged as O


def test_codes_are_torchs_of_8_bits():
    x = torch.cat([torch.linspace(-448, 448, 20001), torch.randn(20000) * 0.01, torch.tensor([0.0, 2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -9])])
    assert np.array_equal(O.fp8_round(x.double().numpy()), x.to(torch.float8_e4m3fn).double().numpy())


@pytest.mark.parametrize("top,e", [(448.0, 0), (449.0, 1), (1.75, -8), (1.7500001, -7), (2.0, -7), (0.0, -100), (1e-38, -100), (3.3e38, 120)])
def test_power_of_a_row(top, e):
    x = np.zeros((1, 64))
    x[0, 5], x[0, 7], x[0, 9] = -top, np.nan, np.inf
    assert O.fp8_power(x)[0] == e
    back = O.fp8_rows(x)[0]
    assert np.isnan(back[0, [7, 9]]).all() and np.isfinite(np.delete(back, [7, 9])).all()


def test_norm_and_rotation_of_a_head():
    rng = np.random.RandomState(1)
    x, g = rng.randn(3, 2, 64), rng.randn(64)
    zero = np.zeros((3, 3), int)
    assert np.allclose(O.norm_rope(x, g, zero, 1e4, 0.0), x / np.sqrt((x ** 2).mean(-1, keepdims=True)) * g)
    pos = np.array([[3, 0, 0], [0, 5, 0], [0, 0, 7]])
    y = O.norm_rope(x, g, pos, 1e4, 1e-6)
    base = O.norm_rope(x, g, zero, 1e4, 1e-6)
    first = {0: 0, 1: 12, 2: 22}                      # each axis' first pair turns by its position: 12 | 10 | 10 pairs of 64 channels
    for axis, p in first.items():
        z = (base[axis, :, 2 * p] + 1j * base[axis, :, 2 * p + 1]) * np.exp(1j * pos[axis, axis])
        assert np.allclose(y[axis, :, 2 * p], z.real) and np.allclose(y[axis, :, 2 * p + 1], z.imag)
        others = [q for a, q in first.items() if a != axis]
        assert np.allclose(y[axis][:, [2 * q for q in others]], base[axis][:, [2 * q for q in others]])


def test_attention_is_torchs_softmax():
    gen = torch.Generator().manual_seed(2)
    q, k, v = torch.randn(5, 4, 64, generator=gen), torch.randn(9, 2, 64, generator=gen), torch.randn(9, 2, 64, generator=gen)
    for group in (0, 1, 4):
        out, _, _ = O.attend(q.numpy(), [k.numpy()], [v.numpy()], [0, 5], [9], [np.ones(9, bool)], group, 0.125, np.zeros(q.shape))
        mask = torch.tensor([[j < O.seen_keys(i, 5, 9, group) for j in range(9)] for i in range(5)])
        ref = torch.nn.functional.scaled_dot_product_attention(q.double().transpose(0, 1), k.double().repeat_interleave(2, 1).transpose(0, 1),
                                                               v.double().repeat_interleave(2, 1).transpose(0, 1), attn_mask=mask, scale=0.125)
        assert np.allclose(out, ref.transpose(0, 1).numpy())


def test_what_a_query_sees():
    assert [O.seen_keys(i, 3, 7, 0) for i in range(3)] == [7, 7, 7]
    assert [O.seen_keys(i, 3, 7, 1) for i in range(3)] == [5, 6, 7]
    assert [O.seen_keys(i, 3, 7, 4) for i in range(3)] == [7, 7, 7]
    assert [O.seen_keys(i, 5, 8, 4) for i in range(5)] == [4, 8, 8, 8, 8]
    assert [O.seen_keys(i, 4, 2, 1) for i in range(4)] == [0, 0, 1, 2]
