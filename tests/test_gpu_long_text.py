"""Texts that are longer than the cache: their splits are many, and the partials of a row more than a wave's lanes."""
import numpy as np
import pytest
import torch

import paper_2605_19218_amd as rk
from rows_util import attend, f64, tolerance
from test_gpu_tree import BF, F32, Layer, ctx  # noqa: F401

pytestmark = pytest.mark.gpu
FORMATS = [(BF, False), (F32, False), (BF, True), (F32, True)]


@pytest.mark.parametrize("dt,q8", FORMATS)
@pytest.mark.parametrize("B,Hq,Hkv,lens,tl,T", [(1, 4, 1, [500], [20000], 3), (2, 8, 2, [0, 130], [6000, 15], 8), (1, 6, 2, [200], [9001], 30), (1, 16, 1, [33], [70000], 12)])
def test_trees(ctx, dt, q8, B, Hq, Hkv, lens, tl, T):  # noqa: F811
    x = Layer(ctx, np.random.default_rng(T), dt, q8, B, Hq, Hkv, 64, lens, tl, T, [T] * B)
    assert rk.rk_tree_plan(ctx, x.lay, T, max(tl), q8)[2] > 8
    x.call()
    x.check()


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("Hq", [1, 40])
def test_one_token(ctx, dt, Hq):  # noqa: F811
    x = Layer(ctx, np.random.default_rng(Hq), dt, True, 1, Hq, 1, 64, [700], [30000], 1, [1])
    assert rk.rk_tree_plan(ctx, x.lay, 0, 30000, True)[2] > 8
    q, out = x.q[:, 0].contiguous(), torch.zeros(1, Hq, 128, dtype=dt, device=x.q.device)
    rk.rk_decode_attn_quant(ctx, x.lay, q, x.k, x.v, x.Rr, x.dmu, x.text, 0.0, out, x.ws)
    ref, size, top = attend(f64(x.q), *x.stored(), x.lens, f64(x.Rr), f64(x.dmu), (f64(x.tk), f64(x.tv)), x.tl)
    e, tol = np.abs(f64(out)[:, None] - ref), tolerance(ref, size, top, 30700, dt)
    assert (e <= tol).all(), (e / tol).max()


@pytest.mark.parametrize("splits", [1, 60])
def test_a_fixed_split_of_the_cache(ctx, splits):  # noqa: F811
    rk.rk_set_option(ctx, rk.RK_OPT_DECODE_SPLITS, splits)
    try:
        x = Layer(ctx, np.random.default_rng(splits), BF, True, 1, 4, 1, 32, [3000], [12000], 5, [5])
        assert rk.rk_tree_plan(ctx, x.lay, 5, 12000, True)[1] == splits
        x.call()
    finally:
        rk.rk_set_option(ctx, rk.RK_OPT_DECODE_SPLITS, 0)
    x.check()
