"""fp64 definitions of the operators whose operands are held in 4 bits, and of the gated residual with its norms.  Written from the formulas; shares no
code with the library.

4 bits: groups of 32 values as codes of e2m1 (sign, 2 exponent bits, 1 fraction bit) times 2^e, e the least in [-100, 125] by which no finite value of the
group exceeds 7; a group with a value that is not finite is all NaN."""
import numpy as np

GROUP, REACH, MOST, LEAST_POWER, LAST_POWER = 32, 7.0, 6.0, -100, 125
CODES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
EVEN = np.array([0, 2, 4, 6])


def groups(x):
    x = np.asarray(x, np.float64)
    return x.reshape(x.shape[:-1] + (-1, GROUP))


def power(x):
    """Exponent of every group of the last axis."""
    g = np.abs(groups(x))
    top = np.where(np.isfinite(g), g, 0.0).max(-1)
    e = np.full(top.shape, LEAST_POWER)
    while (more := (top > REACH * 2.0 ** e.astype(np.float64)) & (e < LAST_POWER)).any():
        e[more] += 1
    return e


def nearest(y):
    """The code (0 .. 7) nearest to |y|, of two the even one; beyond the last it is the last."""
    far = np.abs(np.abs(y)[..., None] - CODES)
    best = far.min(-1, keepdims=True)
    tied = far == best
    first = tied.argmax(-1)
    even = np.zeros(tied.shape, bool)
    even[..., EVEN] = tied[..., EVEN]
    return np.where(even.any(-1), even.argmax(-1), first)


def encode(x):
    """(codes 0 .. 15 of the shape of x, bytes of its groups)"""
    g, e = groups(x), power(x)
    fine = np.isfinite(g).all(-1)
    y = np.where(fine[..., None], g, 0.0) / 2.0 ** e.astype(np.float64)[..., None]
    code = nearest(y) | (np.signbit(y) & fine[..., None]).astype(int) << 3
    return code.reshape(np.shape(x)), np.where(fine, e + 127, 255)


def decode(code, byte):
    """What codes and bytes stand for."""
    code = np.asarray(code)
    x = np.where(code & 8, -1.0, 1.0) * CODES[code & 7]
    factor = np.where(np.asarray(byte) == 255, np.nan, 2.0 ** (np.asarray(byte, np.float64) - 127))
    return (groups(x) * factor[..., None]).reshape(code.shape)


def rows(x):
    """(x as it reads back, exponents of its groups)"""
    code, byte = encode(x)
    return decode(code, byte), power(x)


def unpack(data):
    """Codes of bytes that hold two each, the first in the low half."""
    data = np.asarray(data)
    return np.stack([data & 15, data >> 4], axis=-1).reshape(data.shape[:-1] + (-1,)).astype(int)


def activation(y, act):
    with np.errstate(over="ignore", invalid="ignore"):
        if act == "gelu":
            return 0.5 * y * (1 + np.tanh(np.sqrt(2 / np.pi) * (y + 0.044715 * y ** 3)))
        if act == "silu":
            return y / (1 + np.exp(-y))
    return y


def linear(x, w, bias=None, act=None):
    """act(x w^T + bias), and for tolerances the sums before it and the sums of sizes."""
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        y = x @ w.T
        size = np.abs(x) @ np.abs(w).T
    if bias is not None:
        y = y + np.asarray(bias, np.float64)
        size = size + np.abs(np.asarray(bias, np.float64))
    return activation(y, act), y, size


def norm(x, kind, eps):
    """LayerNorm (biased variance) or RMSNorm of rows, without gains."""
    x = np.asarray(x, np.float64)
    if kind == "layer":
        x = x - x.mean(-1, keepdims=True)
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)


def gated_norm(x, y, kind, eps, res_scale=1.0, gain=None, post_gain=None, gate=None, scale=None, shift=None, group=None):
    """x' = x + res_scale * gate[group] * (N(y) post_gain, or y), h = N(x') gain (1 + scale[group]) + shift[group].  y None: x' = x."""
    x = np.asarray(x, np.float64)
    of = (lambda v: np.asarray(v, np.float64)[group]) if group is not None else (lambda v: np.asarray(v, np.float64)[0])
    if y is not None:
        t = np.asarray(y, np.float64)
        if post_gain is not None:
            t = norm(t, kind, eps) * np.asarray(post_gain, np.float64)
        x = x + res_scale * (1.0 if gate is None else of(gate)) * t
    h = norm(x, kind, eps)
    if gain is not None:
        h = h * np.asarray(gain, np.float64)
    if scale is not None:
        h = h * (1 + of(scale)) + of(shift)
    return x, h
