"""Each attention kernel of many query rows by itself, its rows a work-group asked of the plan: results written without a merge, a caller's own scale and no
shift of the means, drafts that are no numbers on both sides of a tile's end, fixed splits."""
import numpy as np
import pytest
import torch

import paper_2605_19218_amd as rk
from rows_util import D, DEV, attend, f64, tolerance
from test_gpu_tree import BF, F32, Layer, ctx, words  # noqa: F401

pytestmark = pytest.mark.gpu


def layer(ctx, seed, per, dt, q8, lens, tl, T, nd, G, Hkv=2, r=64, mask="tree", B=None):  # noqa: F811
    """A layer whose host's bound of the lengths makes its work-groups take `per` rows: from 2500 tokens and 16 rows a compute unit on, more than 16."""
    n_cu = torch.cuda.get_device_properties(0).multi_processor_count

    class Bound(Layer):
        @staticmethod
        def bound(rows, units):
            return 0 if per == 16 else 2500 * n_cu // ((rows + 15) // 16 * units) + 1

    return Bound(ctx, np.random.default_rng(seed), dt, q8, B or len(lens), G * Hkv, Hkv, r, lens, tl, T, nd, mask)


def planned(ctx, x, tokens=None):  # noqa: F811
    return rk.rk_tree_plan(ctx, x.lay, x.T if tokens is None else tokens, x.M if x.text else 0, x.q8)


def close(got, ref, size, top, n, dt):
    tol = tolerance(ref, size, top, n, dt)
    live = ~np.isnan(ref)
    e = np.abs(got - ref)[live]
    assert np.isfinite(got[live]).all() and (e <= tol[live]).all(), (e / np.maximum(tol[live], 1e-30)).max()


@pytest.fixture
def one_split(ctx):  # noqa: F811
    rk.rk_set_option(ctx, rk.RK_OPT_DECODE_SPLITS, 1)
    yield
    rk.rk_set_option(ctx, rk.RK_OPT_DECODE_SPLITS, 0)


@pytest.mark.parametrize("dt,G,per", [(BF, 1, 16), (BF, 16, 16), (F32, 7, 16), (F32, 48, 16), (BF, 48, 64), (BF, 130, 128)])
@pytest.mark.parametrize("r", [37, 64, 128])
def test_results_without_a_merge(ctx, one_split, dt, G, per, r):  # noqa: F811
    """One split and nothing beside the cache: the work-group writes the result, at any element, and nothing beside it; of an empty sequence zeros."""
    x = layer(ctx, G + r, per, dt, True, [333, 0, 64], None, 1, [1, 1, 1], G, Hkv=1 if G > 64 else 2, r=r)
    assert planned(ctx, x, 0) == (per, 1, 0)
    B, Hq = 3, x.lay.n_q_heads
    big = torch.full((B * Hq * D + 2,), 5.0, dtype=dt, device=DEV)
    rk.rk_decode_attn_quant(ctx, x.lay, x.q[:, 0].contiguous(), x.k, x.v, x.Rr, x.dmu, None, 0.0, big[1:-1], x.ws)
    assert big[0] == 5 and big[-1] == 5
    got = f64(big[1:-1]).reshape(B, 1, Hq, D)
    close(got, *attend(f64(x.q), *x.stored(), x.lens, f64(x.Rr), f64(x.dmu)), x.N, dt)
    assert (got[1] == 0).all()


KERNELS = [(16, BF, False, 5, 4), (16, F32, False, 5, 4), (16, BF, True, 5, 4), (16, F32, True, 5, 4), (64, BF, True, 40, 1), (128, BF, True, 40, 3),
           (128, BF, False, 40, 3)]


@pytest.mark.parametrize("per,dt,q8,T,G", KERNELS)
@pytest.mark.parametrize("scale", [0.03, 0.2])
@pytest.mark.parametrize("shift", [True, False])
def test_scales_and_shifts(ctx, per, dt, q8, T, G, scale, shift):  # noqa: F811
    """A scale of the caller's own meets the cache, the text and the drafts alike; delta_mu may be missing."""
    x = layer(ctx, T + G, per, dt, q8, [300, 77], [40, 9], T, [T, T - 3], G)
    assert planned(ctx, x)[0] == per
    dmu = x.dmu if shift else None
    f = rk.rk_decode_attn_tree_quant if q8 else rk.rk_decode_attn_tree
    f(ctx, x.lay, x.q, x.k, x.v, x.Rr, dmu, x.text, x.drafts, scale, x.out, x.ws)
    ref = attend(f64(x.q), *x.stored(), x.lens, f64(x.Rr), f64(dmu) if shift else None, (f64(x.tk), f64(x.tv)), x.tl, (f64(x.kd), f64(x.vd)), x.nd,
                 x.mask, scale)
    close(f64(x.out), *ref, x.N + x.M + T, dt)


@pytest.mark.parametrize("per,dt,G", [(16, BF, 4), (16, F32, 4), (64, BF, 40), (128, BF, 70)])
@pytest.mark.parametrize("scale", [0.03, 0.2])
@pytest.mark.parametrize("shift", [True, False])
def test_scales_and_shifts_of_one_token(ctx, per, dt, G, scale, shift):  # noqa: F811
    x = layer(ctx, G, per, dt, True, [300, 77], [40, 9], 1, [1, 1], G)
    assert planned(ctx, x, 0)[0] == per
    dmu = x.dmu if shift else None
    out = torch.zeros_like(x.q[:, 0])
    rk.rk_decode_attn_quant(ctx, x.lay, x.q[:, 0].contiguous(), x.k, x.v, x.Rr, dmu, x.text, scale, out, x.ws)
    ref = attend(f64(x.q), *x.stored(), x.lens, f64(x.Rr), f64(dmu) if shift else None, (f64(x.tk), f64(x.tv)), x.tl, scale=scale)
    close(f64(out)[:, None], *ref, x.N + x.M, dt)


@pytest.mark.parametrize("per,dt,q8,T,G", [(16, BF, False, 40, 1), (16, F32, True, 64, 1), (64, BF, True, 40, 1), (64, BF, True, 64, 1),
                                           (128, BF, True, 40, 3), (128, BF, False, 64, 2)])
def test_drafts_that_are_no_numbers_in_both_tiles(ctx, per, dt, q8, T, G):  # noqa: F811
    """Drafts before and behind the 32nd whose Values hold infinities: the rows that see them have these in their channels, the others nothing of them."""
    x = layer(ctx, T, per, dt, q8, [150], [20], T, [T], G)
    assert planned(ctx, x)[0] == per
    bad = {1: (3, np.inf), 31: (40, -np.inf), 32: (41, np.inf), T - 1: (127, np.nan)}
    hidden = ~sum(1 << j for j in bad)
    x.mask = [[m & hidden for m in x.mask[0]]]
    see = {0: [1], 5: [31], 6: [32], 7: [T - 1], 33: [1, 32], T - 1: list(bad), 8: [31, 32]}
    for i, js in see.items():
        x.mask[0][i] |= sum(1 << j for j in js)
    x.drafts.mask = words(x.mask)
    for j, (c, w) in bad.items():
        x.vd[0, :, j, c] = w
    x.call()
    got = f64(x.out)[0].copy()
    for j, (c, _) in bad.items():                  # the same with numbers there
        x.vd[0, :, j, c] = 0.0
    x.out.fill_(5.0)
    x.call()
    same, _ = x.check()
    for i in range(T):
        hit = {bad[j][0]: bad[j][1] for j in see.get(i, [])}
        for c, w in hit.items():
            assert np.array_equal(got[i, :, c], np.full(2 * G, w), equal_nan=True), (i, c)
        rest = [c for c in range(D) if c not in hit]
        assert np.array_equal(got[i][:, rest], same[0, i][:, rest]), i


@pytest.mark.parametrize("q8,T,G,per", [(True, 16, 4, 64), (False, 16, 4, 128), (True, 40, 3, 128), (False, 40, 3, 128)])
@pytest.mark.parametrize("splits", [1, 2, 5, 40])
def test_fixed_splits(ctx, q8, T, G, per, splits):  # noqa: F811
    rk.rk_set_option(ctx, rk.RK_OPT_DECODE_SPLITS, splits)
    try:
        x = layer(ctx, splits, per, BF, q8, [900, 200], [100, 7], T, [T, T - 4], G)
        assert planned(ctx, x)[:2] == (per, splits)
        x.call()
        first = x.out.clone()
        for _ in range(2):
            x.out.fill_(5.0)
            x.call()
            assert torch.equal(x.out, first)
    finally:
        rk.rk_set_option(ctx, rk.RK_OPT_DECODE_SPLITS, 0)
    x.check()


@pytest.mark.parametrize("q8,T,G,per", [(True, 40, 1, 64), (False, 16, 4, 128), (True, 64, 7, 128)])
def test_calls_at_once_and_replays(ctx, q8, T, G, per):  # noqa: F811
    """Two calls on streams of their own, and one in a graph that is replayed between eager work."""
    a, b = [layer(ctx, s, per, BF, q8, [3000, 2000], [40, 3], T, [T, T // 2], G) for s in (1, 2)]
    assert planned(ctx, a)[0] == per
    s = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(4):
        a.call(stream=s[0])
        b.call(stream=s[1])
    torch.cuda.synchronize()
    a.check()
    b.check()
    want, graph = a.out.clone(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(s[0]):
        with torch.cuda.graph(graph, stream=s[0]):
            a.call(stream=s[0])
    for _ in range(3):
        a.out.fill_(5.0)
        assert np.isfinite(torch.randn(64, device=DEV).sum().item())
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a.out, want)
