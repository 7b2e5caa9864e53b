"""The definitions of the 4-bit operators against other ways to say the same."""
import numpy as np
import torch

from oracle import fp4 as F


def test_nearest_by_thresholds():
    """The middles between codes, a hair beside them, and the ties, which go to the even code."""
    mids = (F.CODES[1:] + F.CODES[:-1]) / 2
    assert np.array_equal(F.nearest(F.CODES), np.arange(8)) and np.array_equal(F.nearest(-F.CODES), np.arange(8))
    assert np.array_equal(F.nearest(mids * (1 + 1e-12)), np.arange(1, 8)) and np.array_equal(F.nearest(mids * (1 - 1e-12)), np.arange(7))
    assert np.array_equal(F.nearest(mids), [0, 2, 2, 4, 4, 6, 6])
    assert np.array_equal(F.nearest(np.array([6.5, 7.0, 1e9])), [7, 7, 7])


def test_powers_and_the_round_trip():
    rng = np.random.RandomState(0)
    x = rng.randn(50, 96) * 2.0 ** rng.randint(-90, 90, (50, 1))
    back, e = F.rows(x)
    top = np.abs(F.groups(x)).max(-1)
    assert (top <= 7 * 2.0 ** e).all() and (top > 7 * 2.0 ** (e - 1.0)).all()
    # off by at most half the step around a value: 1/2 below 2 (steps of 0.5), then 1 and 2 times the power
    y, step = np.abs(F.groups(x)) / 2.0 ** e[..., None], None
    step = np.where(y <= 2, 0.5, np.where(y <= 4, 1.0, 2.0))
    assert (np.abs(F.groups(back) - F.groups(x)) <= step / 2 * 2.0 ** e[..., None]).all()
    # what reads back is held without loss
    again, e2 = F.rows(back)
    assert np.array_equal(again, back)
    code, byte = F.encode(x)
    assert np.array_equal(F.decode(code, byte), back) and byte.shape == (50, 3)
    packed = (code[:, 0::2] | code[:, 1::2] << 4).astype(np.uint8)
    assert np.array_equal(F.unpack(packed), code)


def test_ends():
    x = np.zeros((4, 32))
    x[1, 0], x[2, 3], x[3, 1] = np.nan, np.inf, float(np.finfo(np.float32).max)
    code, byte = F.encode(x)
    assert byte[0, 0] == 27 and byte[1, 0] == byte[2, 0] == 255 and (code[1:3] == 0).all() and byte[3, 0] == 252 and code[3, 1] == 7
    assert np.isnan(F.decode(code, byte)[1:3]).all()


def test_linear_and_norms_against_torch():
    rng = np.random.RandomState(1)
    x, w, b = rng.randn(5, 64), rng.randn(7, 64), rng.randn(7)
    f = torch.nn.functional
    t = f.linear(*map(torch.from_numpy, (x, w, b)))
    for act, of in ((None, lambda v: v), ("gelu", lambda v: f.gelu(v, approximate="tanh")), ("silu", f.silu)):
        assert np.allclose(F.linear(x, w, b, act)[0], of(t).numpy(), rtol=1e-12, atol=1e-12)
    g = rng.randn(64)
    assert np.allclose(F.norm(x, "layer", 1e-6) * g, f.layer_norm(torch.from_numpy(x), (64,), torch.from_numpy(g), None, 1e-6).numpy())
    assert np.allclose(F.norm(x, "rms", 1e-6) * g, f.rms_norm(torch.from_numpy(x), (64,), torch.from_numpy(g), 1e-6).numpy())
    gate, scale, shift, group = rng.randn(2, 64), rng.randn(2, 64), rng.randn(2, 64), np.array([0, 1, 1, 0, 0])
    y = rng.randn(5, 64)
    a, h = F.gated_norm(x, y, "rms", 1e-6, 0.5, None, g, gate, scale, shift, group)
    t = torch.from_numpy(x) + 0.5 * torch.from_numpy(gate)[group] * f.rms_norm(torch.from_numpy(y), (64,), torch.from_numpy(g), 1e-6)
    assert np.allclose(a, t.numpy())
    assert np.allclose(h, (f.rms_norm(t, (64,), None, 1e-6) * (1 + torch.from_numpy(scale)[group]) + torch.from_numpy(shift)[group]).numpy())
    assert np.array_equal(F.gated_norm(x, None, "rms", 1e-6)[0], x)
