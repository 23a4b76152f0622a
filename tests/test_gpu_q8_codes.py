"""The codes and steps of the 8-bit caches, number for number: c = x / s to the nearest whole number, ties to even, s the bfloat16 at or next above
max |x| / 127.  A quotient of an fp32 number by a bfloat16 is either half way between two whole numbers or more than 2^-24 of itself away from that, and max |x| / 127
is a bfloat16 or as far from one, so that float64 gives both as they are defined."""
import numpy as np
import pytest
import torch

import paper_2605_19218_amd as rk
from rows_util import D, DEV, f64, kind, normal, up32

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    c = rk.rk_create(0)
    yield c
    rk.rk_destroy(c)


def in_8_bits(x):
    """[..., n] float64 -> the step of each row and its codes, by the definition."""
    top = np.abs(x).max(-1, keepdims=True)
    m, e = np.frexp(top / 127)
    s = np.where(top < 2.0 ** -100, 0.0, np.ldexp(np.ceil(np.ldexp(m, 8)), e - 8))      # (smaller rows are zeros)
    return s, np.rint(over(x, s))


def over(x, s):
    return np.where(s > 0, x / np.where(s > 0, s, 1), 0.0)


def read_back(ctx, lay, k, v):
    """What the codes stand for, in fp32: a code of 7 bits by a step of 8 is exact there."""
    L = rk.Layout(lay.batch, lay.n_q_heads, lay.n_kv_heads, lay.keep, rk.RK_F32, lay.capacity, 0)
    k32 = torch.zeros(lay.batch, lay.n_kv_heads, lay.capacity, lay.keep, dtype=F32, device=DEV)
    v32 = torch.zeros(lay.batch, lay.n_kv_heads, lay.capacity, D, dtype=F32, device=DEV)
    rk.rk_unpack_cache_quant(ctx, L, k, v, k32, v32)
    return f64(k32), f64(v32)


def caches(lay):
    return [torch.zeros(n, dtype=torch.uint8, device=DEV) for n in rk.rk_cache_bytes_quant(lay)]


def written(ctx, K, V, Rr, dt):
    """K, V [B, H, N, d] as a prompt writes them."""
    B, H, N, _ = K.shape
    lay = rk.Layout(B, H, H, Rr.shape[-1], kind(dt), up32(N), 0)
    k, v = caches(lay)
    rk.rk_compress_quant(ctx, lay, rk.Rows(K, N), Rr, k, values=rk.Rows(V, N), v_cache=v)
    return [x[:, :, :N] for x in read_back(ctx, lay, k, v)]


def appended(ctx, K, V, Rr, dt):
    """The same token by token, every row a sequence's first."""
    B, H, N, _ = K.shape
    flat = [x.transpose(1, 2).reshape(B * N, H, D).contiguous() for x in (K, V)]
    R = Rr[:, None].expand(B, N, *Rr.shape[1:]).reshape(B * N, *Rr.shape[1:]).contiguous()
    n = torch.zeros(B * N, dtype=torch.int32, device=DEV)
    lay = rk.Layout(B * N, H, H, Rr.shape[-1], kind(dt), 32, 0, seq_len=n)
    k, v = caches(lay)
    rk.rk_append_quant(ctx, lay, *flat, R, k, v, n)
    return [x[:, :, 0].reshape(B, N, H, -1).transpose(0, 2, 1, 3) for x in read_back(ctx, lay, k, v)]


def differ(a, b):
    return int((a != b).sum())


def identity(B, H, r):
    return torch.eye(D, device=DEV)[:, :r].expand(B, H, D, r).contiguous()


def ties(dt):
    """Rows whose elements lie half way between two codes: s (k + 1/2), for every step and k for which `dt` holds that and a largest element which
    gives that step."""
    bits = 8 if dt == BF else 24
    rows = []
    for m in range(128, 256):
        s = m * 2.0 ** -7
        top = np.floor(127 * s * 2.0 ** (bits - 1 - np.floor(np.log2(127 * s)))) / 2.0 ** (bits - 1 - np.floor(np.log2(127 * s)))
        if in_8_bits(np.array([top]))[0] != s:
            continue
        half = [x for x in (s * (k + 0.5) for k in range(126)) if np.frexp(x)[0] * 2.0 ** bits % 1 == 0 and x < top]
        if half:
            rows.append(np.resize(np.concatenate([half, -np.array(half)]), D))
            rows[-1][m % D] = top
    return np.array(rows)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("way", [written, appended])
def test_ties_go_to_the_even_code(ctx, dt, way):
    x = ties(dt)
    assert len(x) > 20 and (in_8_bits(x)[1] % 2 == 0).mean() > 0.9
    x = np.concatenate([x, x * 2.0 ** -30, x * 2.0 ** 40])
    V = torch.from_numpy(x.astype(np.float32)).to(dt).to(DEV).view(1, 1, -1, D)
    assert differ(f64(V)[0, 0], x) == 0
    K = V if dt == BF else torch.ones_like(V)
    s, c = in_8_bits(x)
    k, v = way(ctx, K, V, identity(1, 1, D), dt)
    assert differ(v[0, 0], c * s) == 0
    if dt == BF:
        assert differ(k[0, 0], c * s) == 0


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("way", [written, appended])
@pytest.mark.parametrize("N", [1, 45, 1500])
def test_codes_of_values(ctx, dt, way, N):
    g = np.random.default_rng(N)
    V = normal(g, (2, 2, N, D), dt) * torch.from_numpy(np.exp(3 * g.standard_normal((2, 2, N, 1))).astype(np.float32)).to(dt).to(DEV)
    s, c = in_8_bits(f64(V))
    _, v = way(ctx, V, V, identity(2, 2, 16), dt)
    assert differ(v, c * s) == 0


@pytest.mark.parametrize("way", [written, appended])
def test_steps_next_to_a_bfloat16(ctx, way):
    """Largest elements at 127 steps, and one unit in the last place above and below."""
    x = []
    for m in range(128, 256):
        top = np.float32(127 * m * 2.0 ** -7)
        for t in (np.nextafter(top, np.float32(0)), top, np.nextafter(top, np.float32(np.inf))):
            row = np.linspace(-0.99, 0.99, D).astype(np.float32) * t
            row[m % D] = t
            x.append(row)
    V = torch.from_numpy(np.array(x, dtype=np.float32)).to(DEV).view(1, 1, -1, D)
    s, c = in_8_bits(f64(V))
    _, v = way(ctx, V, V, identity(1, 1, 16), F32)
    assert differ(v, c * s) == 0


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("way", [written, appended])
@pytest.mark.parametrize("r", [16, 37, 64, 96, 128])
@pytest.mark.parametrize("e", [-90, 0, 90])
def test_codes_of_rotated_keys(ctx, dt, way, r, e):
    """A Key with one channel is a row of R_r times a number: fp32 arithmetic has it but for a rounding or two (R_r in three bf16 parts: exact products, three
    sums of 2^-23 at most), 2^-21 of itself with room, by a prompt as by a token. So a code is off by what that makes of 127, and the step is certain unless the largest element is as near
    to a border."""
    B, H, N = 2, 2, 1000
    g = np.random.default_rng(r + e + 90)
    Rr = torch.from_numpy(g.standard_normal((B, H, D, r)).astype(np.float32)).to(DEV)
    v = torch.from_numpy((g.standard_normal((B, H, N)) * 2.0 ** e).astype(np.float32)).to(dt).to(DEV)
    at = torch.from_numpy(g.integers(0, D, (B, H, N))).to(DEV)
    K = torch.zeros(B, H, N, D, dtype=dt, device=DEV).scatter_(-1, at[..., None], v[..., None])
    got, _ = way(ctx, K, K, Rr, dt)
    x = f64(v)[..., None] * np.take_along_axis(f64(Rr), at.cpu().numpy()[..., None], 2)
    off = 2.0 ** -21
    s, _ = in_8_bits(x)
    sure = (in_8_bits(x * (1 - off))[0] == s) & (in_8_bits(x * (1 + off))[0] == s)
    assert sure.mean() > 0.99
    c = over(got, s)
    far = np.abs(over(x, s) - c) > 0.5 + 127 * off
    sure = np.broadcast_to(sure, c.shape)
    assert int((far & sure).sum()) == 0 and differ((np.rint(c) * s)[sure], got[sure]) == 0


@pytest.mark.parametrize("way", [written, appended])
def test_the_largest_keys_are_numbers(ctx, way):
    """Finite fp32 Keys next to the largest: rows that are finite too."""
    top = torch.finfo(F32).max
    K = torch.zeros(1, 1, 40, D, device=DEV)
    K[0, 0, range(40), range(40)] = torch.tensor([top, -top] * 20, device=DEV)
    x = f64(K)[..., :64] * 0.5
    s, c = in_8_bits(x[:, :, :40])
    k, _ = way(ctx, K, K, 0.5 * identity(1, 1, 64), F32)
    assert differ(k, c * s) == 0
