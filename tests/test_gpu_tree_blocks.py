"""The tests of drafted tokens once more where the host's bound of the lengths is so large that many rows share what is staged (the kernels of 64 and
128 rows a work-group): from 2500 tokens and 16 rows a compute unit on, of 256."""
import numpy as np
import pytest

import test_gpu_tree as tree
from test_gpu_tree import (BF, Layer, ctx, test_again_on_one_workspace, test_far_scores_do_not_lose_the_weights,  # noqa: F401
                           test_masked_drafts_that_are_no_numbers, test_splits, test_streams_and_graph_replay, test_tree, test_two_calls_at_once)

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def long_bound(monkeypatch):
    monkeypatch.setattr(Layer, "bound", staticmethod(lambda rows, units: 0 if rows <= 32 else 640000 // ((rows + 15) // 16 * units) + 1))


@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("r", [1, 32, 45, 64, 96, 100, 128])
@pytest.mark.parametrize("T,Hq,nd", [(11, 6, 11), (32, 4, 31), (33, 4, 17), (13, 20, 13), (64, 4, 64), (64, 10, 63), (64, 14, 33)])
def test_rows(ctx, q8, r, T, Hq, nd):  # noqa: F811
    """33 to 448 rows a KV head, blocks that end inside, waves without rows, tokens that end inside a stage."""
    g = np.random.default_rng(T + Hq + r)
    x = Layer(ctx, g, BF, q8, 2, Hq, 2, r, [int(g.integers(1, 400)), int(g.integers(300, 700))], [int(g.integers(0, 200)), 65], T, [nd, T], "odd")
    x.call()
    x.check()


@pytest.mark.parametrize("q8", [False, True])
def test_nothing_but_masks(ctx, q8):  # noqa: F811
    x = Layer(ctx, np.random.default_rng(3), BF, q8, 1, 16, 2, 32, [0], None, 6, [6])
    x.mask = [[0, 2, 0, 4 + 8, 1 << 40, 32]]
    x.drafts.mask = tree.words(x.mask)
    x.call()
    got, _ = x.check()
    assert (got[0, [0, 2, 4]] == 0).all()
