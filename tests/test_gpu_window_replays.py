"""Captured prompts replayed on segments of other lengths, and sums over a hundred thousand rows."""
import numpy as np
import pytest
import torch

import paper_2605_19218_amd as rk
from rows_util import D, DEV, f64, kind, normal
from test_gpu_window_blocks import KERNELS, Prompt
from window_util import attend, sees, tolerance

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    c = rk.rk_create(0)
    yield c
    rk.rk_destroy(c)


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("shape", KERNELS)
def test_other_lengths(ctx, shape):
    """The plan is the longest length's: shorter ones, fewer rows than new tokens, none at all, and the longest again; each replay bit for bit the eager call, and
    right."""
    p = Prompt(ctx, *shape)
    B, Hq, n, held = shape[1], shape[2], shape[4], shape[5]
    p.call()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        rk.rk_prefill_attn_window(ctx, p.lay, rk.Heads(p.q), n, p.text, p.window, p.sinks, 0.0, rk.Heads(p.out.transpose(1, 2)), p.ws, n_tokens_dev=p.n_dev, stream=side)
    g = np.random.default_rng([31, B, n])
    for turn, (longest, counted) in enumerate([(held - 1, n), (held // 3, n), (max(n // 2, 1), n), (0, n), (held, max(n // 3, 1)), (1, 1), (held, n)]):
        p.lens, p.counts = [max(longest - 3 * b, 0) for b in range(B)], [max(counted - b, 1) for b in range(B)]
        p.text.len.copy_(int32(p.lens))
        p.n_dev.copy_(int32(p.counts))
        p.q.copy_(normal(g, (1, Hq, n, D), p.dt).expand_as(p.q))
        p.out.fill_(5.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = p.out.clone()
        p.out.fill_(5.0)
        p.call()
        torch.cuda.synchronize()
        assert torch.equal(got, p.out), (turn, longest, counted)
        p.check([(0, 0), (min(1, B - 1), Hq - 1)], rows=[0, n // 2, counted - 1, n - 1])


LONG = [
    # dtype, Hq, H, new tokens, rows of a work-group
    (BF, 8, 2, 5, 32),
    (BF, 8, 2, 700, 256),
    (F32, 8, 2, 5, 32),
    (F32, 128, 128, 100, 128),
    (F32, 8, 2, 700, 256),
]


@pytest.mark.parametrize("dt,Hq,H,n,per", LONG)
def test_a_hundred_thousand_rows(ctx, dt, Hq, H, n, per):
    """All rows seen, their scores within some tenths of each other, Values about 1: a mean in which every row counts."""
    g = np.random.default_rng([33, Hq, n])
    held = 100003
    lay = rk.Layout(1, Hq, H, 64, kind(dt), 32, 0)
    assert rk.rk_prefill_plan(ctx, lay, n, held, 0, 0)[0] == per
    q = normal(g, (1, n, Hq, D), dt).transpose(1, 2)
    k, v = (normal(g, (1, 1, held, D), dt) for _ in range(2))
    k.mul_(0.1)
    v.mul_(0.5).add_(1.0)
    k, v = (x.expand(1, H, held, D) for x in (k, v))         # (one head's rows for all)
    text = rk.Text(k, v, held)
    out, one = torch.zeros(1, n, Hq, D, dtype=dt, device=DEV), torch.zeros(1, Hq, D, dtype=dt, device=DEV)
    ws = torch.empty(rk.rk_window_workspace_size(ctx, lay, n), dtype=torch.uint8, device=DEV)
    rk.rk_prefill_attn_window(ctx, lay, rk.Heads(q), n, text, 0, 0, 0.0, rk.Heads(out.transpose(1, 2)), ws)
    rk.rk_decode_attn_window(ctx, lay, q[:, :, n - 1].contiguous(), None, None, None, None, text, 0, 0, 0.0, one, ws)
    t = np.array(sorted({0, n // 2, n - 1}))
    for h in (0, Hq - 1):
        hk, x = h // (Hq // H), f64(q[0, h, t])
        see = sees(held - n + t[:, None], np.arange(held)[None], 0, 0)
        ref, size, mean = attend(x, [(f64(k[0, hk]), x, np.zeros(len(t)), f64(v[0, hk]), see)])
        e = np.abs(f64(out[0, t, h]) - ref)
        assert (e <= tolerance(ref, size, mean, held, dt, dt == BF)).all(), e.max()
        e = np.abs(f64(one[0, h]) - ref[-1])
        assert (e <= tolerance(ref[-1:], size[-1:], mean[-1:], held, dt, False)[0]).all(), e.max()
