"""Each kernel of prompts (few rows, many rows, fp32), with and without splits: edges, masked values that are no numbers, results over the queries."""
import numpy as np
import pytest
import torch

import paper_2605_19218_amd as rk
from rows_util import D, DEV, f64, kind, normal
from window_util import attend, sees, tolerance

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    c = rk.rk_create(0)
    yield c
    rk.rk_destroy(c)


class Prompt:
    def __init__(self, ctx, dt, B, Hq, H, n, held, window, sinks, rows, splits):
        """held: rows of the segment, of every sequence but the second, which has a quarter of the new tokens and half of the rows."""
        g = np.random.default_rng([B, Hq, n, held, window])
        self.ctx, self.dt, self.n, self.window, self.sinks, self.G = ctx, dt, n, window, sinks, Hq // H
        self.lay = rk.Layout(B, Hq, H, 64, kind(dt), 32, 0)
        p = rk.rk_prefill_plan(ctx, self.lay, n, held, window, sinks)
        assert p[0] == rows and (p[1] > 1) == splits, p          # (the kernel that the test is for)
        self.counts, self.lens = [n] * B, [held] * B
        if B > 1:
            self.counts[1], self.lens[1] = max(n // 4, 1), held // 2
        # few different sequences, repeated: the device makes the rest
        self.q, self.k, self.v = (normal(g, (min(B, 3), x, h, D), dt).repeat((B + 2) // 3, 1, 1, 1)[:B].transpose(1, 2) for x, h in ((n, Hq), (held, H), (held, H)))
        self.text = rk.Text(self.k, self.v, held, len=torch.tensor(self.lens, dtype=torch.int32, device=DEV))
        self.n_dev = torch.tensor(self.counts, dtype=torch.int32, device=DEV)
        self.out = torch.full((B, n, Hq, D), 5.0, dtype=dt, device=DEV)
        self.ws = torch.full((rk.rk_window_workspace_size(ctx, self.lay, n),), 0xff, dtype=torch.uint8, device=DEV)

    def call(self, q=None, out=None):
        rk.rk_prefill_attn_window(self.ctx, self.lay, rk.Heads(self.q if q is None else q), self.n, self.text, self.window, self.sinks, 0.0,
                                  rk.Heads(self.out.transpose(1, 2) if out is None else out), self.ws, n_tokens_dev=self.n_dev)

    def positions(self, b):
        return self.lens[b] - self.counts[b] + np.arange(self.counts[b])

    def check(self, at, rows=None):
        """at: (sequence, head) pairs; rows: of the new tokens"""
        for b, h in at:
            m, hk = self.counts[b], h // self.G
            t = np.arange(m) if rows is None else np.array([r % m for r in rows])
            q, see = f64(self.q[b, h, t]), sees(self.positions(b)[t][:, None], np.arange(self.lens[b])[None], self.window, self.sinks)
            ref, size, mean = attend(q, [(f64(self.k[b, hk, :self.lens[b]]), q, np.zeros(len(t)), f64(self.v[b, hk, :self.lens[b]]), see)])
            tol = tolerance(ref, size, mean, self.lens[b], self.dt, self.dt == BF)
            e = np.abs(f64(self.out[b, t, h]) - ref)
            assert (e <= tol).all(), (b, h, (e / np.maximum(tol, 1e-30)).max())
            assert (self.out[b, m:] == 5.0).all()


KERNELS = [
    # dtype, B, Hq, H, n, held, window, sinks, rows of a work-group, splits
    (BF, 1, 8, 2, 45, 60, 0, 0, 32, False),
    (BF, 1, 14, 2, 90, 900, 600, 5, 32, True),
    (BF, 40, 8, 4, 90, 100, 0, 0, 256, False),
    (BF, 40, 8, 4, 130, 200, 33, 70, 256, False),
    (BF, 2, 28, 4, 300, 3000, 0, 0, 256, True),
    (BF, 1, 32, 8, 500, 4000, 2500, 70, 256, True),
    (F32, 40, 8, 4, 9, 40, 7, 2, 32, False),
    (F32, 2, 16, 2, 230, 400, 0, 0, 32, False),
    (F32, 2, 8, 2, 40, 300, 0, 0, 32, True),
    (F32, 1, 16, 2, 150, 1500, 900, 40, 32, True),
    (F32, 40, 8, 4, 90, 100, 20, 2, 128, False),
    (F32, 1, 8, 2, 45, 300, 0, 0, 128, True),
    (F32, 16, 16, 8, 300, 400, 100, 5, 256, False),
    (F32, 1, 32, 8, 500, 2000, 900, 30, 256, True),
    # few work-groups: blocks that see more are in more splits, up to eight
    (BF, 1, 1, 1, 3000, 3100, 0, 0, 32, True),
    (BF, 1, 8, 8, 2500, 2500, 0, 0, 256, True),
    (F32, 1, 8, 2, 300, 300, 0, 0, 32, True),
    (F32, 1, 8, 4, 600, 1100, 700, 9, 128, True),
    (F32, 1, 16, 2, 700, 900, 300, 40, 256, True),
    # ... and more than eight, the same for all
    (BF, 1, 2, 2, 30, 5000, 0, 0, 32, True),
]


@pytest.mark.parametrize("shape", KERNELS)
def test_results(ctx, shape):
    p = Prompt(ctx, *shape)
    p.call()
    last = shape[1] - 1
    p.check([(0, 0), (min(1, last), shape[2] - 1), (last, shape[2] // 2)],
            rows=None if shape[4] <= 130 else [0, 1, 31, 32, 36, 63, 64, 255, 256, 500, shape[4] // 4 - 1, shape[4] - 2, shape[4] - 1])


@pytest.mark.parametrize("what", [float("nan"), float("-inf")])
@pytest.mark.parametrize("shape", KERNELS)
def test_masked_values(ctx, shape, what):
    """Values and Keys that are no numbers: what does not see them is as if they were 0, and what sees such a Value is no number."""
    p = Prompt(ctx, *shape)
    B, held, n = shape[1], shape[5], shape[4]
    # rows that some new tokens see and some do not
    bad = sorted({held - n // 3, held - n // 4, held - 1} | ({held - n - p.window + n // 5, held - n - p.window + n // 4} if p.window else set()))
    bad = [j for j in bad if p.sinks <= j < held]
    k0, v0 = p.k.clone(), p.v.clone()
    for j in bad:
        p.k[:, :, j], p.v[:, :, j] = 0.0, 0.0
    p.call()
    clean = p.out.clone()
    p.k.copy_(k0)
    p.v.copy_(v0)
    for j in bad:
        p.k[:, :, j], p.v[:, :, j] = 0.0, what
    p.call()
    for b in {0, min(1, B - 1), B - 1}:
        m = p.counts[b]
        hit = (sees(p.positions(b)[:, None], np.array(bad)[None], p.window, p.sinks) & (np.array(bad)[None] < p.lens[b])).any(1)
        assert b == 1 or (hit.any() and not hit.all())
        hit = torch.from_numpy(hit).to(DEV)
        assert torch.equal(p.out[b, :m][~hit], clean[b, :m][~hit]) and not torch.isfinite(p.out[b, :m][hit]).any()
    for j in bad:
        p.k[:, :, j], p.v[:, :, j] = what, 0.0
    p.call()
    for b in {0, B - 1}:
        m = p.counts[b]
        hit = torch.from_numpy((sees(p.positions(b)[:, None], np.array(bad)[None], p.window, p.sinks) & (np.array(bad)[None] < p.lens[b])).any(1)).to(DEV)
        assert torch.equal(p.out[b, :m][~hit], clean[b, :m][~hit])


@pytest.mark.parametrize("shape", KERNELS)
def test_over_the_queries(ctx, shape):
    """The result over its own queries, bit for bit, and twice the same."""
    p = Prompt(ctx, *shape)
    p.call()
    first = p.out.clone()
    p.call()
    assert torch.equal(first, p.out)
    q = p.q.clone()
    p.call(q, q)
    for b, m in enumerate(p.counts):
        assert torch.equal(q[b, :, :m], first[b, :m].transpose(0, 1)) and torch.equal(q[b, :, m:], p.q[b, :, m:])


@pytest.mark.parametrize("shape", KERNELS)
def test_scores_that_rise(ctx, shape):
    """Scores in the hundreds that rise along the segment: the running maximum moves at every tile."""
    p = Prompt(ctx, *shape)
    p.q.mul_(8)
    p.k.mul_(torch.linspace(0.1, 6, shape[5], device=DEV)[None, None, :, None].to(p.dt))
    p.call()
    p.check([(0, 0), (shape[1] - 1, shape[2] - 1)], rows=[0, 5, shape[4] // 2, shape[4] - 1])
