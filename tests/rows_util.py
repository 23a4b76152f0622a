"""Plain 64-bit forms of the 8-bit cache and of the attention of drafted tokens, for the tests of both."""
import numpy as np
import torch

import paper_2605_19218_amd as rk

D, DEV = 128, "cuda:0"


def up32(n):
    return max(32, (n + 31) // 32 * 32)


def kind(dt):
    return rk.RK_F32 if dt == torch.float32 else rk.RK_BF16


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def rotation(g, B, H, r):
    """[B, H, d, r] fp32 on the device: orthonormal columns."""
    q = np.linalg.qr(g.standard_normal((B, H, D, D)))[0][..., :r]
    return torch.from_numpy(np.ascontiguousarray(q, dtype=np.float32)).to(DEV)


def normal(g, shape, dt, std=1.0):
    return torch.from_numpy((std * g.standard_normal(shape)).astype(np.float32)).to(dt).to(DEV)


def attend(q, K, V, lens, Rr, dmu, text=None, text_lens=None, drafts=None, n_drafts=None, mask=None, scale=None):
    """q [B, T, Hq, d], K [B, H, N, r], V [B, H, N, d] as stored, text / drafts (k, v) [B, H, M, d], mask [B, T] of Python ints, all
    fp64: (out, what bounds its error): for each row the largest sum |q~| |k~| scale of a score that it sees, and the largest |v|.
    A row that nothing is asked of is NaN in both."""
    B, T, Hq, _ = q.shape
    H, scale = K.shape[1], 1 / np.sqrt(D) if scale is None else scale
    out = np.full(q.shape, np.nan)
    size, top = np.full((B, T, Hq), np.nan), np.full((B, T, Hq), np.nan)
    for b in range(B):
        for h in range(Hq):
            hk = h // (Hq // H)
            k, v, n = K[b, hk, :lens[b]], V[b, hk, :lens[b]], int(lens[b])
            for t in range(T if n_drafts is None else int(n_drafts[b])):
                qt = q[b, t, h] @ Rr[b, hk]
                s = [(k @ qt + (q[b, t, h] @ dmu[b, hk] if dmu is not None else 0.0)) * scale]
                a = [(np.abs(k) @ np.abs(qt) + (np.abs(q[b, t, h]) @ np.abs(dmu[b, hk]) if dmu is not None else 0.0)) * scale]
                vs = [v]
                if text is not None:
                    m = int(text_lens[b])
                    s.append(text[0][b, hk, :m] @ q[b, t, h] * scale)
                    a.append(np.abs(text[0][b, hk, :m]) @ np.abs(q[b, t, h]) * scale)
                    vs.append(text[1][b, hk, :m])
                if drafts is not None:
                    word = (2 << t) - 1 if mask is None else mask[b][t]
                    see = [j for j in range(int(n_drafts[b])) if word >> j & 1]
                    s.append(drafts[0][b, hk, see] @ q[b, t, h] * scale)
                    a.append(np.abs(drafts[0][b, hk, see]) @ np.abs(q[b, t, h]) * scale)
                    vs.append(drafts[1][b, hk, see])
                s, a, vs = np.concatenate(s), np.concatenate(a), np.concatenate(vs)
                if not len(s) or (s == -np.inf).all():
                    out[b, t, h], size[b, t, h], top[b, t, h] = 0.0, 0.0, 0.0
                    continue
                w = np.exp(s - s.max())
                out[b, t, h] = (w / w.sum()) @ vs
                size[b, t, h], top[b, t, h] = a.max(), np.abs(vs).max()
    return out, size, top


def tolerance(ref, size, top, n, dt):
    """A score is off by `size` times the parts' 2^-16 (bf16: q R_r from R_r in two parts, then itself in two, 2^-17 each) or 2^-20 (fp32:
    128 + r products and sums of 2^-24 each stay under 2^-20 of the absolute sum unless all round one way), plus what the exponential adds
    (2^-22); the weights by as much, two parts of them by 2^-17 more (bf16), their n-term sums by sqrt(n) 2^-24, and a weighted mean of values
    up to `top` by twice that.  The output is rounded once, by half a step."""
    e = (2.0 ** -16 * size + 2.0 ** -16 if dt == torch.bfloat16 else 2.0 ** -20 * size + 2.0 ** -20) + np.sqrt(n) * 2.0 ** -24
    return torch.finfo(dt).eps / 2 * np.abs(ref) + (2 * e * top)[..., None]
