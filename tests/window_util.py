"""Plain 64-bit forms of positions and of attention with a window and sinks, for the tests of both."""
import numpy as np
import torch

from rows_util import D


def sees(p, j, window, sinks):
    """Whether the token at position p attends row j (arrays that broadcast)."""
    return (j <= p) & ((j < sinks) | (p - j < window)) if window > 0 else j <= p


def attend(q, parts, scale=None):
    """q [rows, d]; parts: (scores' Keys [m, c], queries [rows, c], bias [rows], Values [m, d], seen [rows, m]), all fp64.  (out, the largest sum |q| |k|
    scale of a score that a row sees, the mean of |v| under the row's weights.)  Rows that see nothing: zeros."""
    scale = 1 / np.sqrt(D) if scale is None else scale
    rows = q.shape[0]
    s, a, seen, vals = [], [], [], []
    for k, qk, bias, v, see in parts:
        with np.errstate(invalid="ignore"):
            s.append(np.where(see, (qk @ k.T + bias[:, None]) * scale, -np.inf))
            a.append(np.where(see, (np.abs(qk) @ np.abs(k).T + np.abs(bias)[:, None]) * scale, 0.0))
        seen.append(see)
        vals.append(v)
    s, a, seen, vals = np.concatenate(s, 1), np.concatenate(a, 1), np.concatenate(seen, 1), np.concatenate(vals)
    out, mean = np.zeros((rows, vals.shape[1])), np.zeros((rows, vals.shape[1]))
    for i in range(rows):
        at = np.nonzero(seen[i])[0]
        if not len(at) or (s[i, at] == -np.inf).all():
            continue
        w = np.exp(s[i, at] - s[i, at].max())
        out[i], mean[i] = (w / w.sum()) @ vals[at], (w / w.sum()) @ np.abs(vals[at])
    return out, a.max(1, initial=0.0), mean


def tolerance(ref, size, mean, n, dt, weights_bf16):
    """A score of fp32 products and sums is off by less than 2^-20 of its absolute sum `size` (128 roundings of 2^-24 unless all go one way; with q R_r
    and R_r in two bf16 parts 2^-16 of it), what the exponential adds by 2^-20; weights that are rounded to bf16 by half a step more, 2^-8, and their n-term sums
    by sqrt(n) 2^-24.  A mean under weights that are off by a relative e is off by 2 e of the mean of |v|.  The output is rounded
    once."""
    part = 2.0 ** -20 if dt == torch.float32 or weights_bf16 else 2.0 ** -16
    e = part * size + part + np.sqrt(n) * 2.0 ** -24
    return torch.finfo(dt).eps / 2 * np.abs(ref) + (2 * e[..., None] + (2.0 ** -8 if weights_bf16 else 0.0)) * mean


def turned(x, pos, inv_freq, axis, adjacent, sign=1.0):
    """Rows x [..., n, d] (fp64) of positions pos [axes, n]; (out, a bound of what fp32 arithmetic may be off by): angles in 80 bits."""
    out, err = x.copy(), np.zeros_like(x)
    p = len(axis)
    for i, a in enumerate(axis):
        one, two = (2 * i, 2 * i + 1) if adjacent else (i, p + i)
        angle = np.asarray(pos[a], np.longdouble) * np.longdouble(inv_freq[i])
        c, s = np.cos(angle).astype(np.float64), sign * np.sin(angle).astype(np.float64)
        u, v = x[..., one], x[..., two]
        out[..., one], out[..., two] = u * c - v * s, u * s + v * c
        # the fraction of a turn is rounded to fp32 (2^-25 turns, 2^-22 radians), the functions and the two products and their sum add 2^-22; the product
        # and division in fp64 are off by 2^-52 of the angle together
        e = 2.0 ** -21 + 2.0 ** -51 * np.abs(angle).astype(np.float64)
        err[..., one] = err[..., two] = e * (np.abs(u) + np.abs(v))
    return out, err
