"""fp64 definitions of the operators around the paged key/value cache: per-head RMSNorm with 3D rotation, codes of 8 bits with a
power of two per row, attention of new tokens over their sequence's pages.  Written from the formulas; shares no code with the library."""
import numpy as np

FP8_MAX, FP8_MIN_EXP, MIN_POWER = 448.0, -6, -100      # e4m3: largest value, exponent of the least normal value; least power of a row


def norm_rope(x, gain, pos, theta, eps):
    """x [n, heads, d], gain [d], pos [n, 3] -> R(pos) (x / sqrt(mean(x^2) + eps) * gain), pairs (2i, 2i+1) split over frame, row, column."""
    x, gain = np.asarray(x, np.float64), np.asarray(gain, np.float64)
    d = x.shape[-1]
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain
    c = d // 6
    out = np.empty_like(y)
    pair = 0
    for axis, count in enumerate((d // 2 - 2 * c, c, c)):
        for i in range(count):
            ang = np.asarray(pos)[:, axis].astype(np.float64) * theta ** (-i / count)
            a, b = y[..., 2 * pair], y[..., 2 * pair + 1]
            cos, sin = np.cos(ang)[:, None], np.sin(ang)[:, None]
            out[..., 2 * pair], out[..., 2 * pair + 1] = a * cos - b * sin, a * sin + b * cos
            pair += 1
    return out


def fp8_power(x):
    """Least e >= -100 with every finite |x| of a row (last axis) <= 448 * 2^e."""
    x = np.abs(np.asarray(x, np.float64))
    top = np.where(np.isfinite(x), x, 0.0).max(-1)
    e = np.full(top.shape, MIN_POWER)
    while (more := top > FP8_MAX * 2.0 ** e.astype(np.float64)).any():
        e[more] += 1
    return e


def fp8_round(y):
    """Nearest e4m3 value (ties to the even fraction) of |y| <= 448; what is not finite becomes NaN."""
    y = np.asarray(y, np.float64)
    fin = np.isfinite(y)
    z = np.where(fin, y, 0.0)
    ex = np.maximum(np.floor(np.log2(np.maximum(np.abs(z), 2.0 ** FP8_MIN_EXP))), FP8_MIN_EXP)
    step = 2.0 ** (ex - 3)
    return np.where(fin, np.rint(z / step) * step, np.nan)


def fp8_rows(x):
    """(values that the codes stand for, exponents e): the row as it reads back.  At e = 120 the codes end at 240: the next one, 256, would stand for 2^128,
    which fp32 and bf16 do not hold."""
    e = fp8_power(x)
    s = 2.0 ** e.astype(np.float64)[..., None]
    most = np.where(e == 120, 240.0, FP8_MAX)[..., None]
    y = fp8_round(np.asarray(x, np.float64) / s)
    return np.where(np.isnan(y), y, np.clip(y, -most, most)) * s, e


def seen_keys(i, n, keys, group):
    """How many of its keys the i-th of n new tokens sees."""
    if group == 0:
        return keys
    p = keys - n + i
    return 0 if p < 0 else min(keys, (p // group + 1) * group)


def attend(q, k, v, q_start, keys_of, exists, group, scale, out):
    """q [n, hq, d]; k, v: lists of [keys, hk, d] per sequence; exists: lists of bool [keys].  Writes rows of sequences into a copy of out; returns it and, for
    tolerances, per row and head the mean of |v| under the weights and the largest sum of |q||k| * scale."""
    q, out = np.asarray(q, np.float64), np.array(out, np.float64)
    mean_abs, score_abs = np.zeros_like(out), np.zeros(out.shape[:2])
    shared = q.shape[1] // (k[0].shape[1] if k else 1)
    for b in range(len(keys_of)):
        n = q_start[b + 1] - q_start[b]
        for i in range(n):
            t = q_start[b] + i
            vis = np.arange(keys_of[b]) < seen_keys(i, n, keys_of[b], group)
            vis &= exists[b]
            for h in range(q.shape[1]):
                kk, vv = np.asarray(k[b], np.float64)[vis, h // shared], np.asarray(v[b], np.float64)[vis, h // shared]
                out[t, h] = 0.0
                if not len(kk):
                    continue
                with np.errstate(invalid="ignore", over="ignore"):
                    s = kk @ q[t, h] * scale
                    if np.all(s == -np.inf):
                        continue
                    w = np.exp(s - s.max())
                    w = w / w.sum()
                    # a weight is above 0, however small it is in 64 bits, unless the score is -inf: values that are not finite reach the result or do not
                    finite = np.where(np.isfinite(vv), vv, 0.0)
                    out[t, h] = w @ finite + (vv - finite)[s != -np.inf].sum(0)
                    mean_abs[t, h] = w @ np.abs(finite)
                    score_abs[t, h] = (np.abs(kk) @ np.abs(q[t, h])).max() * scale
    return out, mean_abs, score_abs
