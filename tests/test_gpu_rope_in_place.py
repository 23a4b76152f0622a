"""Positions put on rows over themselves, for pairs that several lanes of a row read: bit for bit what a result of its own gets."""
import numpy as np
import pytest
import torch

import paper_2605_19218_amd as rk
from rows_util import D, kind, normal
from test_gpu_rope import check, spec

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = rk.rk_create(0)
    yield c
    rk.rk_destroy(c)


@pytest.mark.parametrize("n", [3, 45])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pairs,adjacent", [(1, False), (7, False), (9, False), (13, False), (21, False), (31, False), (33, False), (60, False), (63, False), (13, True), (63, True),
                                            (64, True), (24, False), (64, False)])
def test_over_itself(ctx, pairs, adjacent, dt, n):
    g = np.random.default_rng([29, pairs, adjacent, n])
    B, Hq, H = 2, 7, 3
    rope, pos, inv, axis = spec(g, B, n, 3, pairs, adjacent)
    lay = rk.Layout(B, Hq * H, H, 64, kind(dt), 32, 0)
    q, k = (normal(g, (B, n, h, D), dt).transpose(1, 2) for h in (Hq * H, H))
    own = [torch.zeros_like(x) for x in (q, k)]
    for flags in (0, rk.RK_ROPE_INVERSE):
        rk.rk_rope(ctx, lay, rope, n, rk.Heads(q), rk.Heads(own[0]), rk.Heads(k), rk.Heads(own[1]), flags=flags)
        over = [x.clone() for x in (q, k)]
        for _ in range(3):
            for x, y in zip(over, (q, k)):
                x.copy_(y)
            rk.rk_rope(ctx, lay, rope, n, rk.Heads(over[0]), rk.Heads(over[0]), rk.Heads(over[1]), rk.Heads(over[1]), flags=flags)
            assert torch.equal(over[0], own[0]) and torch.equal(over[1], own[1])
        for b in range(B):
            for got, x in zip(own, (q, k)):
                check(got[b], x[b], b, n, pos, inv, axis, adjacent, dt, -1.0 if flags else 1.0)
