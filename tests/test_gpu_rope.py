"""Positions of several axes on queries and Keys, alone and on the way into the text segment, against plain forms in 64 bits and more."""
import numpy as np
import pytest
import torch

import paper_2605_19218_amd as rk
from rows_util import D, DEV, f64, kind, normal
from window_util import turned

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    c = rk.rk_create(0)
    yield c
    rk.rk_destroy(c)


def int32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)


def spec(g, B, n, axes, pairs, adjacent, most=60000, least=0):
    pos = g.integers(least, most + 1, (axes, B, n)).astype(np.int32)
    inv = (10000.0 ** (-np.arange(pairs) / pairs)).astype(np.float32)
    axis = [int(a) for a in g.integers(0, axes, pairs)]
    rope = rk.Rope(int32(pos), torch.from_numpy(inv).to(DEV), axis=axis, pairing=rk.RK_ROPE_ADJACENT if adjacent else rk.RK_ROPE_HALVES)
    return rope, pos, inv, axis


def projection(g, B, n, heads, dt):
    """[B, heads, n, d] as a projection leaves it: token by token."""
    return normal(g, (B, n, heads, D), dt).transpose(1, 2)


def check(got, x, b, m, pos, inv, axis, adjacent, dt, sign=1.0):
    """got, x [heads, n, d] of sequence b, its first m rows."""
    ref, err = turned(f64(x[:, :m]), pos[:, b, :m], inv, axis, adjacent, sign)
    tol = torch.finfo(dt).eps / 2 * np.abs(ref) + err * (1 + torch.finfo(dt).eps)
    assert (np.abs(f64(got[:, :m]) - ref) <= tol).all(), (np.abs(f64(got[:, :m]) - ref) / np.maximum(tol, 1e-30)).max()


SHAPES = [
    # B, Hq, Hkv, n, lens, axes, pairs, adjacent
    (1, 2, 2, 1, None, 1, 64, False),
    (2, 32, 8, 1, [1, 0], 3, 64, False),
    (3, 7, 1, 7, [7, 3, 0], 3, 64, True),
    (2, 28, 4, 8, [8, 1], 2, 32, False),
    (2, 3, 3, 33, [33, 32], 4, 48, True),
    (1, 8, 2, 71, None, 3, 64, False),
    (2, 4, 4, 100, [100, 37], 3, 13, False),
    (1, 5, 1, 9, None, 2, 13, True),
    (1, 1, 1, 300, [299], 1, 1, False),
    (1, 130, 65, 3, None, 3, 40, False),
    (40, 4, 2, 2, None, 2, 8, True),
]


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("shape", SHAPES)
def test_rope(ctx, shape, dt, inverse):
    B, Hq, H, n, lens, axes, pairs, adjacent = shape
    g = np.random.default_rng([3, B, Hq, n, pairs, inverse])
    rope, pos, inv, axis = spec(g, B, n, axes, pairs, adjacent)
    lay = rk.Layout(B, Hq, H, 64, kind(dt), 32, 0)
    q, k = projection(g, B, n, Hq, dt), projection(g, B, n, H, dt)
    qo, ko = torch.full((B, n, Hq, D), 5.0, dtype=dt, device=DEV), torch.full((B, H, n, D), 5.0, dtype=dt, device=DEV)
    rk.rk_rope(ctx, lay, rope, n, rk.Heads(q), rk.Heads(qo.transpose(1, 2)), rk.Heads(k), rk.Heads(ko), flags=rk.RK_ROPE_INVERSE if inverse else 0,
               n_tokens_dev=int32(lens) if lens else None)
    for b in range(B):
        m = lens[b] if lens else n
        for got, x in ((qo.transpose(1, 2), q), (ko, k)):
            check(got[b], x[b], b, m, pos, inv, axis, adjacent, dt, -1.0 if inverse else 1.0)
            assert (got[b, :, m:] == 5.0).all()


def test_counts_out_of_range(ctx):
    g = np.random.default_rng(5)
    rope, pos, inv, axis = spec(g, 3, 10, 2, 64, False)
    lay = rk.Layout(3, 4, 2, 64, rk.RK_F32, 32, 0)
    q, out = projection(g, 3, 10, 4, F32), torch.full((3, 4, 10, D), 5.0, device=DEV)
    rk.rk_rope(ctx, lay, rope, 10, rk.Heads(q), rk.Heads(out), None, None, n_tokens_dev=int32([-3, 10 ** 6, 4]))
    for b, m in enumerate((0, 10, 4)):
        check(out[b], q[b], b, m, pos, inv, axis, False, F32)
        assert (out[b, :, m:] == 5.0).all()
    before = out.clone()
    rk.rk_rope(ctx, lay, rope, 0, rk.Heads(q), rk.Heads(out), None, None)
    assert torch.equal(out, before)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("pairs,adjacent", [(64, False), (64, True), (16, False), (21, False), (21, True)])
def test_in_place_on_a_projection(ctx, dt, pairs, adjacent):
    """Queries and Keys inside one buffer, over themselves; the Values between them and their neighbours stay."""
    g = np.random.default_rng([7, pairs, adjacent])
    B, Hq, H, n = 2, 6, 2, 45
    rope, pos, inv, axis = spec(g, B, n, 3, pairs, adjacent)
    buf = normal(g, (B, n, Hq + 2 * H, D), dt)
    old = buf.clone()
    cut = lambda x: (x[:, :, :Hq].transpose(1, 2), x[:, :, Hq:Hq + H].transpose(1, 2))
    (q, k), (q0, k0) = cut(buf), cut(old)
    lay = rk.Layout(B, Hq, H, 64, kind(dt), 32, 0)
    rk.rk_rope(ctx, lay, rope, n, rk.Heads(q), rk.Heads(q), rk.Heads(k), rk.Heads(k))
    for b in range(B):
        check(q[b], q0[b], b, n, pos, inv, axis, adjacent, dt)
        check(k[b], k0[b], b, n, pos, inv, axis, adjacent, dt)
    assert torch.equal(buf[:, :, Hq + H:], old[:, :, Hq + H:])


@pytest.mark.parametrize("n", [2, 40])
def test_far_and_negative_positions(ctx, n):
    g = np.random.default_rng(11)
    rope, pos, inv, axis = spec(g, 1, n, 2, 64, False, most=2 ** 31 - 1, least=-2 ** 31)
    lay = rk.Layout(1, 2, 1, 64, rk.RK_F32, 32, 0)
    q, out = projection(g, 1, n, 2, F32), torch.zeros(1, 2, n, D, device=DEV)
    rk.rk_rope(ctx, lay, rope, n, rk.Heads(q), rk.Heads(out), None, None)
    check(out[0], q[0], 0, n, pos, inv, axis, False, F32)


def test_inverse_is_the_gradient(ctx):
    """sum(w . rope(x)) grows along w taken back: against the formula's transpose by differences of the linear map itself."""
    g = np.random.default_rng(13)
    B, H, n = 1, 2, 12
    rope, pos, inv, axis = spec(g, B, n, 3, 64, False)
    lay = rk.Layout(B, H, H, 64, rk.RK_F32, 32, 0)
    x, w = projection(g, B, n, H, F32), projection(g, B, n, H, F32)
    grad = torch.zeros(B, H, n, D, device=DEV)
    rk.rk_rope(ctx, lay, rope, n, rk.Heads(w), rk.Heads(grad), None, None, flags=rk.RK_ROPE_INVERSE)
    for _ in range(8):
        h, t, c = int(g.integers(H)), int(g.integers(n)), int(g.integers(D))
        y = []
        for step in (0.5, -0.5):                     # (the map is linear: a difference of any step is the gradient)
            z = x.clone()
            z[0, h, t, c] += step
            out = torch.zeros(B, H, n, D, device=DEV)
            rk.rk_rope(ctx, lay, rope, n, rk.Heads(z), rk.Heads(out), None, None)
            y.append(float((f64(out) * f64(w)).sum()))
        # two of the outputs change with x; each is off by 2^-21 (|x| + |y|), twice, and so is the gradient
        size = float(f64(x[0, h, t]).__abs__().max() + 1) * float(f64(w[0, h, t]).__abs__().max())
        assert abs((y[0] - y[1]) - float(grad[0, h, t, c])) <= 10 * 2.0 ** -21 * size


APPENDS = [
    # B, Hq, Hkv, n, counts, lens, capacity, pairs, adjacent
    (1, 32, 8, 1, None, [500], 501, 64, False),
    (64, 8, 8, 1, None, [3 * i for i in range(64)], 200, 64, False),
    (2, 28, 4, 1, [1, 0], [0, 9], 30, 64, True),
    (3, 4, 2, 5, [5, 2, 0], [0, 31, 7], 40, 48, False),
    (2, 6, 3, 70, [70, 33], [10, 0], 90, 64, False),
    (1, 2, 1, 300, None, [0], 300, 20, True),
    (1, 200, 100, 4, None, [2], 64, 64, False),
]


@pytest.mark.parametrize("alias", [False, True])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("shape", APPENDS)
def test_append(ctx, shape, dt, alias):
    B, Hq, H, n, counts, lens, cap, pairs, adjacent = shape
    g = np.random.default_rng([17, B, Hq, n])
    rope, pos, inv, axis = spec(g, B, n, 3, pairs, adjacent)
    lay = rk.Layout(B, Hq, H, 64, kind(dt), 32, 0)
    q, k, v = (projection(g, B, n, h, dt) for h in (Hq, H, H))
    kt, vt = normal(g, (B, cap, H, D), dt).transpose(1, 2), normal(g, (B, cap, H, D), dt).transpose(1, 2)
    k0, v0 = kt.clone(), vt.clone()
    qo = torch.full((B, n, Hq, D), 5.0, dtype=dt, device=DEV)
    at = int32(lens)
    out = at if alias else torch.full((B,), -7, dtype=torch.int32, device=DEV)
    rk.rk_rope_append_text(ctx, lay, rope, n, rk.Heads(q), rk.Heads(qo.transpose(1, 2)), rk.Heads(k), rk.Heads(v),
                           rk.Text(kt, vt, min(max(lens), cap - n), len=at), out, n_tokens_dev=int32(counts) if counts else None)
    for b in range(B):
        m, p = counts[b] if counts else n, lens[b]
        check(qo[b].transpose(0, 1), q[b], b, m, pos, inv, axis, adjacent, dt)
        assert (qo[b, m:] == 5.0).all()
        check(kt[b, :, p:], k[b], b, m, pos, inv, axis, adjacent, dt)
        assert torch.equal(vt[b, :, p:p + m], v[b, :, :m])
        assert int(out[b]) == p + m
        for new, was in ((kt, k0), (vt, v0)):
            assert torch.equal(new[b, :, :p], was[b, :, :p]) and torch.equal(new[b, :, p + m:], was[b, :, p + m:])


@pytest.mark.parametrize("n", [3, 20])
def test_append_at_a_full_segment(ctx, n):
    """On the device a segment takes what fits; its length says so, and the queries are turned all the same."""
    g = np.random.default_rng([19, n])
    B, H, cap = 4, 2, 30
    rope, pos, inv, axis = spec(g, B, n, 2, 64, False)
    lay = rk.Layout(B, H, H, 64, rk.RK_BF16, 32, 0)
    q, k, v = (projection(g, B, n, H, BF) for _ in range(3))
    kt, vt = (torch.full((B, H, cap, D), 3.0, dtype=BF, device=DEV) for _ in range(2))
    qo, lens = torch.full((B, H, n, D), 5.0, dtype=BF, device=DEV), [cap, cap - 2, 40, -5]
    at = int32(lens)
    rk.rk_rope_append_text(ctx, lay, rope, n, rk.Heads(q), rk.Heads(qo), rk.Heads(k), rk.Heads(v), rk.Text(kt, vt, 0, len=at), at)
    assert at.tolist() == [cap, cap, 40, -5]
    for b, m in enumerate((0, 2, 0, 0)):
        check(qo[b], q[b], b, n, pos, inv, axis, False, BF)
        check(kt[b, :, cap - 2:], k[b], b, m, pos, inv, axis, False, BF)
        assert torch.equal(vt[b, :, cap - 2:cap - 2 + m], v[b, :, :m])
        assert (kt[b, :, :cap - 2] == 3.0).all() and (m or (vt[b] == 3.0).all())


def test_on_another_stream(ctx):
    g = np.random.default_rng(23)
    rope, pos, inv, axis = spec(g, 1, 50, 3, 64, False)
    lay = rk.Layout(1, 4, 2, 64, rk.RK_BF16, 32, 0)
    q, out = projection(g, 1, 50, 4, BF), torch.zeros(1, 4, 50, D, dtype=BF, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    rk.rk_rope(ctx, lay, rope, 50, rk.Heads(q), rk.Heads(out), None, None, stream=side)
    side.synchronize()
    check(out[0], q[0], 0, 50, pos, inv, axis, False, BF)
