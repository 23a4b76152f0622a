"""How the attention of drafted tokens and over 8-bit caches shares its work out (no GPU; without a context: 256 compute units)."""
import random

import pytest

import paper_2605_19218_amd as rk

N_CU = 256


def lay(B, Hq, Hkv, r, dtype, cached):
    return rk.Layout(B, Hq, Hkv, r, dtype, max(32, (cached + 31) // 32 * 32), cached)


def plan(B, Hq, Hkv, T, cached, text, quant, dtype=rk.RK_BF16, r=64, ctx=None):
    """(rows a work-group, splits of the cache, of the other rows, work-groups a split)"""
    per, sv, sr = rk.rk_tree_plan(ctx, lay(B, Hq, Hkv, r, dtype, cached), T, text, quant)
    rows = max(T, 1) * Hq // Hkv
    return per, sv, sr, (rows + per - 1) // per * B * Hkv


@pytest.mark.parametrize("B,Hq,Hkv,T,cached,text,quant,dtype", [
    (1, 32, 8, 8, 0, 30000, False, rk.RK_BF16), (1, 32, 8, 0, 2880, 100000, True, rk.RK_BF16), (1, 32, 8, 0, 2880, 10000, True, rk.RK_BF16),
    (1, 8, 1, 8, 2880, 8000, False, rk.RK_BF16), (1, 8, 1, 8, 2880, 8000, True, rk.RK_BF16), (1, 32, 8, 16, 1000, 30000, False, rk.RK_BF16),
    (4, 8, 8, 4, 4000, 12000, False, rk.RK_F32), (1, 32, 8, 0, 2880, 20000, True, rk.RK_F32), (1, 8, 2, 3, 500, 60000, False, rk.RK_BF16),
    (8, 28, 4, 16, 1000, 8000, False, rk.RK_BF16)])
def test_a_long_text_is_shared_out(B, Hq, Hkv, T, cached, text, quant, dtype):
    """A text that takes longer than the cache leaves no more than half of the compute units without a work-group of it, as far as there are partials for it."""
    per, sv, sr, groups = plan(B, Hq, Hkv, T, cached, text, quant, dtype)
    slots = rk.rk_tree_workspace_size(None, lay(B, Hq, Hkv, 64, dtype, cached), max(T, 1)) // (B * max(T, 1) * Hq * 130 * 4)
    assert groups * sr >= 0.5 * N_CU or sv + sr >= 0.75 * slots, (per, sv, sr, groups)


def test_the_cache_beside_a_long_text_keeps_its_splits():
    """A long text keeps the memory busy: one work-group that walks through the whole cache beside it would end last."""
    assert plan(4, 8, 8, 4, 4000, 12000, False)[1] >= 4 and plan(1, 32, 8, 0, 2880, 20000, True, rk.RK_F32)[1] >= 4


@pytest.mark.parametrize("quant", [False, True])
def test_rows_a_work_group_go_by_all_tokens(quant):
    """Many rows share what is staged once the tokens that they read are many, cached or text."""
    for T, G in ((16, 4), (16, 7), (64, 7)):
        assert plan(1, 8 * G, 8, T, 600, 600, quant)[0] == 16
        assert plan(1, 8 * G, 8, T, 60000, 0, quant)[0] == plan(1, 8 * G, 8, T, 0, 60000, quant)[0] > 16
    assert plan(1, 8, 8, 8, 10 ** 6, 10 ** 6, quant)[0] == 16 and plan(1, 64, 8, 64, 10 ** 6, 10 ** 6, quant, rk.RK_F32)[0] == 16


def test_plans_fit_the_workspace():
    g = random.Random(3)
    ctx = rk.rk_create(rk.RK_DEVICE_NONE)
    try:
        for _ in range(3000):
            Hkv = g.choice([1, 2, 4, 8, 16, 32])
            B, Hq, T, quant = g.choice([1, 1, 2, 5, 16, 64, 300]), Hkv * g.choice([1, 2, 4, 7, 16, 48]), g.choice([0, 1, 3, 8, 17, 64]), g.random() < 0.5
            cached, text = [int(10 ** g.uniform(0, 6)) if g.random() < 0.9 else 0 for _ in range(2)]
            text = g.choice([text, 0, 2 ** 31 - 1])
            dtype = g.choice([rk.RK_F32, rk.RK_BF16])
            forced = g.choice([0, 0, 1, 5, 40, 64, 500])
            rk.rk_set_option(ctx, rk.RK_OPT_DECODE_SPLITS, forced)
            per, sv, sr, _ = plan(B, Hq, Hkv, T, cached, text, quant, dtype, ctx=ctx)
            rows = B * max(T, 1) * Hq
            assert per in (16, 64, 128) and sv >= 1 and sr >= (1 if T or text else 0)
            assert (sv + sr) * rows * 130 * 4 + 256 <= rk.rk_tree_workspace_size(ctx, lay(B, Hq, Hkv, 64, dtype, cached), max(T, 1))
            assert not forced or sv == forced
    finally:
        rk.rk_destroy(ctx)


def test_workspace_by_rows_and_options():
    """As the header has it: 520 bytes a row and partial, 10 to 64 partials, N + 8 at least once the splits are set to N; a workspace of before is refused then."""
    ctx, P = rk.rk_create(rk.RK_DEVICE_NONE), 4096
    try:
        for B, Hq, Hkv, T in ((1, 32, 8, 1), (8, 28, 4, 16), (64, 32, 32, 64), (1, 1, 1, 1)):
            L, rows = lay(B, Hq, Hkv, 64, rk.RK_BF16, 4000), B * T * Hq
            size = rk.rk_tree_workspace_size(ctx, L, T)
            assert size == rk.rk_tree_workspace_size(None, L, T) and 10 * 520 * rows <= size <= 64 * 520 * rows + 512
            for N in (1, 60, 300):
                rk.rk_set_option(ctx, rk.RK_OPT_DECODE_SPLITS, N)
                assert rk.rk_tree_workspace_size(ctx, L, T) >= max(size, (N + 8) * 520 * rows)
            L.seq_len = P
            d = rk.Drafts(P, P, T, strides=(0, 0, 128))
            for n, status in ((size, rk.RK_ERR_WORKSPACE), (rk.rk_tree_workspace_size(ctx, L, T), rk.RK_ERR_NO_DEVICE)):
                with pytest.raises(rk.RotateKError) as e:
                    rk.rk_decode_attn_tree(ctx, L, P, P, P, P, P, None, d, 0.0, P, P, workspace_bytes=n)
                assert e.value.status == status
            rk.rk_set_option(ctx, rk.RK_OPT_DECODE_SPLITS, 0)
    finally:
        rk.rk_destroy(ctx)


def test_refusals():
    L = lay(1, 8, 8, 64, rk.RK_BF16, 100)
    for a in ((L, -1), (L, 65), (L, 4, -1), (lay(1, 8, 8, 0, rk.RK_BF16, 100), 4)):
        with pytest.raises(rk.RotateKError):
            rk.rk_tree_plan(None, *a)
    assert rk.lib().rk_tree_plan(None, None, 1, 0, 0, None, None, None) == rk.RK_ERR_INVALID_ARG
