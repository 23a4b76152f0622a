"""The 8-bit caches against their definition in 64 bits: written for prompts and single tokens, read back, attended."""
import numpy as np
import pytest
import torch

import paper_2605_19218_amd as rk
from rows_util import D, DEV, attend, f64, kind, normal, rotation, tolerance, up32

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    c = rk.rk_create(0)
    yield c
    rk.rk_destroy(c)


class Cache:
    def __init__(self, ctx, B, H, r, cap, dt, fill=0):
        self.ctx, self.B, self.H, self.r, self.cap, self.dt = ctx, B, H, r, cap, dt
        kb, vb = rk.rk_cache_bytes_quant(self.layout(H))
        self.k = torch.full((kb,), fill, dtype=torch.uint8, device=DEV)
        self.v = torch.full((vb,), fill, dtype=torch.uint8, device=DEV)
        self.len = torch.zeros(B, dtype=torch.int32, device=DEV)

    def layout(self, Hq, most=0, seq_len=None):
        return rk.Layout(self.B, Hq, self.H, self.r, kind(self.dt), self.cap, most, seq_len=seq_len)

    def rows(self, seq_len=None, fill=0.0):
        k = torch.full((self.B, self.H, self.cap, self.r), fill, dtype=self.dt, device=DEV)
        v = torch.full((self.B, self.H, self.cap, D), fill, dtype=self.dt, device=DEV)
        rk.rk_unpack_cache_quant(self.ctx, self.layout(self.H, seq_len=seq_len), self.k, self.v, k, v)
        return f64(k), f64(v)

    def compress(self, K, V, Rr, n, **sel):
        rk.rk_compress_quant(self.ctx, self.layout(self.H), rk.Rows(K, n, **sel), Rr, self.k, values=rk.Rows(V, n, **sel), v_cache=self.v,
                          seq_len_out=self.len)


def held(got, x, off, dt):
    """`got` is x in 8 bits: off by half a step (at most max |x| / 127, 2^-7 more by its rounding upwards, and by what max |x| is off) plus
    what x itself is off, and rounded once more as it is read back."""
    top = np.abs(x).max(-1, keepdims=True) + off
    lim = 0.5 * top / 127 * (1 + 2.0 ** -7) * (1 + 2.0 ** -22) + off
    lim = lim + torch.finfo(dt).eps / 2 * (np.abs(x) + lim)
    assert (np.abs(got - x) <= lim).all(), (np.abs(got - x) / lim).max()


def rotated(K, Rr):
    """K R_r, and how far fp32 sums of bf16 products of R_r in two parts (2^-17 of R_r, in fp32 of the Keys too) are from it."""
    k, R = f64(K), f64(Rr)
    return k @ R, (np.abs(k) @ np.abs(R)).max(-1, keepdims=True) * (2.0 ** -15 + 128 * 2.0 ** -24)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("r", [1, 16, 24, 37, 48, 64, 80, 96, 113, 128])
def test_write_and_read_back(ctx, dt, r):
    B, H, N = 3, 2, 517
    g = np.random.default_rng(r)
    Rr = rotation(g, B, H, r)
    K = normal(g, (B, H, N, D), dt) * torch.from_numpy(np.exp(2 * g.standard_normal((B, H, N, 1))).astype(np.float32)).to(dt).to(DEV)
    V = normal(g, (B, H, N, D), dt)
    c = Cache(ctx, B, H, r, up32(N), dt, fill=0x35)
    before = c.rows()
    lens = torch.tensor([517, 0, 34], dtype=torch.int32, device=DEV)
    c.compress(K, V, Rr, N, n_tokens_dev=lens)
    assert c.len.tolist() == lens.tolist()
    got = c.rows()
    want, off = rotated(K, Rr)
    for b, n in enumerate(lens.tolist()):
        held(got[0][b, :, :n], want[b, :, :n], off[b, :, :n], dt)
        held(got[1][b, :, :n], f64(V)[b, :, :n], 0.0, dt)
        assert np.array_equal(got[0][b, :, n:], before[0][b, :, n:]) and np.array_equal(got[1][b, :, n:], before[1][b, :, n:])
    some = c.rows(lens, fill=7.0)
    for b, n in enumerate(lens.tolist()):
        assert np.array_equal(some[0][b, :, :n], got[0][b, :, :n]) and (some[0][b, :, n:] == 7).all() and (some[1][b, :, n:] == 7).all()


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("n", [1, 15, 16, 17, 31, 32, 33, 127, 128, 129, 1000])
def test_exact_rows_come_back(ctx, dt, n):
    """Whole numbers up to 127 by a power of two, taken through columns of the identity: held without an error, at any length, row order and stride."""
    B, H, r = 2, 3, 64
    g = np.random.default_rng(n)

    def coded(w):
        c = np.clip(np.rint(g.standard_normal((B, n, H, w)) * 40), -127, 127)
        c[..., g.integers(w)] = 127
        return torch.from_numpy((c * np.exp2(g.integers(-20, 20, (B, n, H, 1)))).astype(np.float32)).to(dt).to(DEV)

    K = torch.zeros(B, n, H, D, dtype=dt, device=DEV)
    K[..., :r] = coded(r)
    V = coded(D)
    eye = torch.eye(D, device=DEV)[:, :r].expand(B, H, D, r).contiguous()
    c = Cache(ctx, B, H, r, up32(n), dt)
    c.compress(K.transpose(1, 2), V.transpose(1, 2), eye, n)
    k, v = c.rows()
    assert np.array_equal(k[:, :, :n], f64(K.transpose(1, 2))[..., :r]) and np.array_equal(v[:, :, :n], f64(V.transpose(1, 2)))
    keep = torch.from_numpy(np.concatenate([np.sort(g.choice(n, (n + 1) // 2, replace=False)) for _ in range(B)]).astype(np.int32)).to(DEV)
    m = (n + 1) // 2
    off = torch.arange(B + 1, dtype=torch.int64, device=DEV) * m
    c2 = Cache(ctx, B, H, r, up32(m), dt)
    c2.compress(K.transpose(1, 2), V.transpose(1, 2), eye, m, tok_idx=keep, tok_off=off)
    k2, v2 = c2.rows()
    for b in range(B):
        at = keep[b * m:(b + 1) * m].cpu().numpy()
        assert np.array_equal(k2[b, :, :m], k[b][:, at]) and np.array_equal(v2[b, :, :m], v[b][:, at])


@pytest.mark.parametrize("dt", [BF, F32])
def test_rows_that_are_no_numbers(ctx, dt):
    B, H, r, N = 1, 1, 32, 40
    g = np.random.default_rng(5)
    K, V = normal(g, (B, H, N, D), dt), normal(g, (B, H, N, D), dt)
    K[0, 0, 3, 7], K[0, 0, 5, 7], V[0, 0, 6, 127], V[0, 0, 35, 0] = float("nan"), float("inf"), float("-inf"), float("nan")
    K[0, 0, 8], V[0, 0, 8], K[0, 0, 33], V[0, 0, 33] = 0, 0, 2.0 ** -120, 2.0 ** -120
    eye = torch.eye(D, device=DEV)[:, :r].expand(B, H, D, r).contiguous()
    c = Cache(ctx, B, H, r, 64, dt)
    c.compress(K, V, eye, N)
    k, v = c.rows()
    k, v = k[0, 0], v[0, 0]
    for t in range(N):
        assert np.isnan(k[t]).all() == (t in (3, 5)) and np.isnan(k[t]).any() == (t in (3, 5))
        assert np.isnan(v[t]).all() == (t in (6, 35)) and np.isnan(v[t]).any() == (t in (6, 35))
    assert (k[[8, 33]] == 0).all() and (v[[8, 33]] == 0).all()


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("r,Hkv", [(32, 1), (37, 8), (64, 2), (128, 3)])
def test_append(ctx, dt, r, Hkv):
    B, cap = 6, 96
    g = np.random.default_rng(r)
    Rr = rotation(g, B, Hkv, r)
    c = Cache(ctx, B, Hkv, r, cap, dt, fill=0x36)
    lens = [0, 1, 31, 32, 95, 96]                       # the last is full: untouched
    c.len = torch.tensor(lens, dtype=torch.int32, device=DEV)
    before = c.rows()
    kn, vn = normal(g, (B, Hkv, D), dt), normal(g, (B, Hkv, D), dt)
    out = torch.full((B,), -1, dtype=torch.int32, device=DEV)
    for aliased in (False, True):
        rk.rk_append_quant(ctx, c.layout(Hkv, 95, c.len), kn, vn, Rr, c.k, c.v, c.len if aliased else out)
    assert out.tolist() == [1, 2, 32, 33, 96, 96] and c.len.tolist() == out.tolist()
    got = c.rows()
    want, off = rotated(kn[:, :, None], Rr)
    for b, n in enumerate(lens):
        keep = [t for t in range(cap) if t != n]
        assert np.array_equal(got[0][b][:, keep], before[0][b][:, keep]) and np.array_equal(got[1][b][:, keep], before[1][b][:, keep])
        if n < cap:
            held(got[0][b, :, n:n + 1], want[b], off[b], dt)
            held(got[1][b, :, n:n + 1], f64(vn)[b][:, None], 0.0, dt)


def decode(ctx, c, q, Rr, dmu, most, text=None, splits=0, scale=0.0):
    Hq = q.shape[1]
    lay = c.layout(Hq, most, c.len)
    rk.rk_set_option(ctx, rk.RK_OPT_DECODE_SPLITS, splits)
    out = torch.full_like(q, 3.0)
    ws = torch.empty(rk.rk_tree_workspace_size(ctx, lay, 1), dtype=torch.uint8, device=DEV)
    rk.rk_decode_attn_quant(ctx, lay, q, c.k, c.v, Rr, dmu, text, scale, out, ws)
    rk.rk_set_option(ctx, rk.RK_OPT_DECODE_SPLITS, 0)
    return out


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("Hq,Hkv,r,N,M,splits", [(2, 2, 32, 70, 0, 0), (32, 8, 32, 1024, 40, 0), (28, 4, 64, 700, 300, 3), (7, 7, 37, 33, 1, 0),
                                                 (20, 1, 128, 260, 65, 2), (48, 1, 96, 1500, 0, 7), (8, 1, 16, 1, 33, 0), (4, 2, 80, 600, 31, 1)])
def test_decode(ctx, dt, Hq, Hkv, r, N, M, splits):
    B = 3
    g = np.random.default_rng(Hq * r + N)
    Rr = rotation(g, B, Hkv, r)
    c = Cache(ctx, B, Hkv, r, up32(N), dt, fill=0xff)             # rows behind the end: steps that are NaN
    lens = [N, N // 3, 0]
    dev = torch.tensor(lens, dtype=torch.int32, device=DEV)
    c.compress(normal(g, (B, Hkv, N, D), dt, 2.0), normal(g, (B, Hkv, N, D), dt), Rr, N, n_tokens_dev=dev)
    q = normal(g, (B, Hq, D), dt)
    dmu = torch.from_numpy(g.standard_normal((B, Hkv, D)).astype(np.float32) * 0.2).to(DEV)
    text = tl = None
    if M:
        tk, tv = normal(g, (B, Hkv, M + 3, D), dt), normal(g, (B, Hkv, M + 3, D), dt)
        tl = [M // 2, M, 0]
        for b in range(B):
            tk[b, :, tl[b]:], tv[b, :, tl[b]:] = float("nan"), float("inf")
        text = rk.Text(tk, tv, M, len=torch.tensor(tl, dtype=torch.int32, device=DEV))
    got = f64(decode(ctx, c, q, Rr, dmu, N, text, splits))
    k32, v32 = (torch.zeros(B, Hkv, c.cap, w, dtype=F32, device=DEV) for w in (r, D))      # the codes' own values: more bits than bf16 has
    rk.rk_unpack_cache_quant(ctx, rk.Layout(B, Hkv, Hkv, r, rk.RK_F32, c.cap, 0, seq_len=dev), c.k, c.v, k32, v32)
    ref, size, top = attend(f64(q)[:, None], f64(k32), f64(v32), lens, f64(Rr), f64(dmu), (f64(tk), f64(tv)) if M else None, tl)
    tol = tolerance(ref, size, top, N + M, dt)[:, 0]
    assert (np.abs(got - ref[:, 0]) <= tol).all(), (np.abs(got - ref[:, 0]) / np.maximum(tol, 1e-30)).max()
    assert (got[2] == 0).all()
