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
    m, e = np.frexp(np.abs(x).max(-1, keepdims=True) / 127)
    s = np.ldexp(np.ceil(np.ldexp(m, 8)), e - 8)
    return s, np.rint(x / s)


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
