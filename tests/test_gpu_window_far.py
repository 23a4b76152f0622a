"""Segments whose offsets pass 32 bits, captured steps, and calls that share a context."""
import numpy as np
import pytest
import torch

import paper_2605_19218_amd as rk
from rows_util import D, DEV, f64, kind, normal
from window_util import attend, sees, tolerance, turned

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    c = rk.rk_create(0)
    yield c
    rk.rk_destroy(c)


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def inv_freq():
    return (10000.0 ** (-np.arange(64) / 64)).astype(np.float32)


@pytest.mark.parametrize("n,window,sinks", [(3, 50, 4), (300, 120, 40)])
def test_seventeen_million_rows(ctx, n, window, sinks):
    """One head's segment of 4.3 GB: positions put on behind it, then the prompt's and a token's attention, whose windows and sinks lie 4 GB apart."""
    g = np.random.default_rng(n)
    rows, Hq = (1 << 24) + 1000, 2
    lay = rk.Layout(1, Hq, 1, 64, rk.RK_BF16, 32, 0)
    k, v = (torch.zeros(1, 1, rows, D, dtype=BF, device=DEV) for _ in range(2))
    held = (1 << 24) + 77
    near = max(window, n) + n
    for x in (k, v):
        x[0, 0, :sinks] = normal(g, (sinks, D), BF)
        x[0, 0, held - near:held] = normal(g, (near, D), BF)
    q, kn, vn = (normal(g, (1, n, h, D), BF).transpose(1, 2) for h in (Hq, 1, 1))
    pos = g.integers(held, held + 5000, (2, 1, n)).astype(np.int32)
    axis = [i % 2 for i in range(64)]
    rope = rk.Rope(torch.from_numpy(pos).to(DEV), torch.from_numpy(inv_freq()).to(DEV), axis=axis)
    length = int32([held])
    qo = torch.zeros(1, n, Hq, D, dtype=BF, device=DEV)
    rk.rk_rope_append_text(ctx, lay, rope, n, rk.Heads(q), rk.Heads(qo.transpose(1, 2)), rk.Heads(kn), rk.Heads(vn), rk.Text(k, v, held, len=length), length)
    assert length.tolist() == [held + n]
    for got, x in ((qo.transpose(1, 2)[0], q[0]), (k[0, :, held:held + n], kn[0])):
        ref, err = turned(f64(x), pos[:, 0], inv_freq(), axis, False)
        assert (np.abs(f64(got) - ref) <= 2.0 ** -8 * np.abs(ref) + err * 1.01).all()
    assert torch.equal(v[0, :, held:held + n], vn[0])
    ws = torch.empty(rk.rk_window_workspace_size(ctx, lay, n), dtype=torch.uint8, device=DEV)
    text = rk.Text(k, v, held + n, len=length)
    out, one = torch.zeros(1, n, Hq, D, dtype=BF, device=DEV), torch.zeros(1, Hq, D, dtype=BF, device=DEV)
    rk.rk_prefill_attn_window(ctx, lay, rk.Heads(qo.transpose(1, 2)), n, text, window, sinks, 0.0, rk.Heads(out.transpose(1, 2)), ws)
    rk.rk_decode_attn_window(ctx, lay, qo[:, n - 1].contiguous(), None, None, None, None, text, window, sinks, 0.0, one, ws)
    at = np.concatenate([np.arange(sinks), np.arange(held - near, held + n)])
    rowsel = torch.from_numpy(at).to(DEV)
    ks, vs = f64(k[0, 0, rowsel]), f64(v[0, 0, rowsel])
    p = held + np.arange(n)[:, None]
    for h in range(Hq):
        x = f64(qo[0, :, h])
        ref, size, mean = attend(x, [(ks, x, np.zeros(n), vs, sees(p, at[None], window, sinks))])
        assert (np.abs(f64(out[0, :, h]) - ref) <= tolerance(ref, size, mean, len(at), BF, True)).all()
        assert (np.abs(f64(one[0, h]) - ref[-1]) <= tolerance(ref[-1:], size[-1:], mean[-1:], len(at), BF, True)[0]).all()


@pytest.mark.parametrize("dt", [BF, F32])
def test_steps_in_a_graph(ctx, dt):
    """A token's positions, its row, its attention and the length that grows, captured once and replayed; every replay against the eager calls on copies."""
    g = np.random.default_rng(3)
    B, Hq, H, cap, w, s = 3, 8, 2, 200, 40, 3
    lay = rk.Layout(B, Hq, H, 64, kind(dt), 32, 0)
    start = [60, 7, 0]
    kt, vt = (normal(g, (B, H, cap, D), dt) for _ in range(2))
    held = int32(start)
    qkv = torch.zeros(B, 1, Hq + 2 * H, D, dtype=dt, device=DEV)
    q, k, v = (x.transpose(1, 2) for x in qkv.split([Hq, H, H], 2))
    pos = torch.zeros(3, B, 1, dtype=torch.int32, device=DEV)
    rope = rk.Rope(pos, torch.from_numpy(inv_freq()).to(DEV), axis=[i % 3 for i in range(64)])
    qo, out = (torch.zeros(B, Hq, D, dtype=dt, device=DEV) for _ in range(2))
    ws = torch.empty(rk.rk_window_workspace_size(ctx, lay, 1), dtype=torch.uint8, device=DEV)

    def step(kt, vt, held, qo, out, stream=None):
        rk.rk_rope_append_text(ctx, lay, rope, 1, rk.Heads(q), rk.Heads(qo[:, :, None]), rk.Heads(k), rk.Heads(v), rk.Text(kt, vt, cap - 1, len=held), held,
                               stream=stream)
        rk.rk_decode_attn_window(ctx, lay, qo, None, None, None, None, rk.Text(kt, vt, cap, len=held), w, s, 0.0, out, ws, stream=stream)

    copies = [x.clone() for x in (kt, vt, held, qo, out)]
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        step(kt, vt, held, qo, out, stream=side)
    for turn in range(5):
        qkv.copy_(normal(g, tuple(qkv.shape), dt))
        pos.copy_(int32(g.integers(0, 4000, (3, B, 1)).tolist()))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        step(*copies)
        torch.cuda.synchronize()
        for a, b in zip((kt, vt, held, qo, out), copies):
            assert torch.equal(a, b)
        assert held.tolist() == [x + turn + 1 for x in start]


def test_lengths_beyond_their_bound(ctx):
    """A length above max_len is held within it, a negative one counts as none."""
    g = np.random.default_rng(5)
    lay = rk.Layout(3, 2, 1, 64, rk.RK_BF16, 32, 0)
    k, v = (normal(g, (3, 1, 90, D), BF) for _ in range(2))
    q = normal(g, (3, 2, D), BF)
    ws = torch.empty(rk.rk_window_workspace_size(ctx, lay, 1), dtype=torch.uint8, device=DEV)
    one, many = torch.full((3, 2, D), 5.0, dtype=BF, device=DEV), torch.full((3, 2, 1, D), 5.0, dtype=BF, device=DEV)
    text = rk.Text(k, v, 80, len=int32([10 ** 6, -3, 80]))
    rk.rk_decode_attn_window(ctx, lay, q, None, None, None, None, text, 30, 2, 0.0, one, ws)
    rk.rk_prefill_attn_window(ctx, lay, rk.Heads(q[:, :, None]), 1, text, 30, 2, 0.0, rk.Heads(many), ws)
    assert (one[1] == 0).all() and (many[1] == 0).all()
    at = np.nonzero(sees(79, np.arange(80), 30, 2))[0]
    for b in (0, 2):
        x = f64(q[b])
        ref, size, mean = attend(x, [(f64(k[b, 0])[at], x, np.zeros(2), f64(v[b, 0])[at], np.ones((2, len(at)), bool))])
        for got in (one[b], many[b, :, 0]):
            assert (np.abs(f64(got) - ref) <= tolerance(ref, size, mean, 32, BF, True)).all()


def test_broadcast_sources(ctx):
    """One head's queries, Keys or Values for all (strides of 0) are read as often as they are asked for."""
    g = np.random.default_rng(7)
    lay = rk.Layout(2, 4, 2, 64, rk.RK_F32, 32, 0)
    n = 20
    x = normal(g, (1, 1, n, D), F32)
    pos = g.integers(0, 900, (1, 2, n)).astype(np.int32)
    rope = rk.Rope(torch.from_numpy(pos).to(DEV), torch.from_numpy(inv_freq()).to(DEV))
    out = torch.zeros(2, 4, n, D, device=DEV)
    rk.rk_rope(ctx, lay, rope, n, rk.Heads(x.expand(2, 4, n, D)), rk.Heads(out), None, None)
    for b in range(2):
        ref, err = turned(np.repeat(f64(x[0]), 4, 0), pos[:, b], inv_freq(), [0] * 64, False)
        assert (np.abs(f64(out[b]) - ref) <= 2.0 ** -24 * np.abs(ref) + err * 1.01).all()


@pytest.mark.parametrize("apart", [(1 << 24) - 8, 1 << 24])
def test_rows_far_apart(ctx, apart):
    """Rows of the segment as far apart as the kernel of many rows takes them, and farther: 23 GB of which 700 rows are read."""
    g = np.random.default_rng(23)
    n, Hq, H = 700, 32, 8
    lay = rk.Layout(1, Hq, H, 64, rk.RK_BF16, 32, 0)
    assert rk.rk_prefill_plan(ctx, lay, n, n, 0, 0)[0] == 256
    q, k, v = (normal(g, (1, n, h, D), BF).transpose(1, 2) for h in (Hq, H, H))
    room = torch.empty((n - 1) * apart + 2 * H * D, dtype=BF, device=DEV)
    far = [torch.as_strided(room, (1, H, n, D), (0, D, apart, 1), i * H * D) for i in range(2)]
    for x, y in zip(far, (k, v)):
        x.copy_(y)
    out = torch.zeros(2, 1, n, Hq, D, dtype=BF, device=DEV)
    ws = torch.empty(rk.rk_window_workspace_size(ctx, lay, n), dtype=torch.uint8, device=DEV)
    for o, (a, b) in zip(out, (far, (k, v))):
        rk.rk_prefill_attn_window(ctx, lay, rk.Heads(q), n, rk.Text(a, b, n, strides=tuple(a.stride()[:3])), 0, 0, 0.0, rk.Heads(o.transpose(1, 2)), ws)
    if apart < 1 << 24:
        assert torch.equal(out[0], out[1])
    t = np.array([0, 1, 31, 32, 63, 64, 65, 300, 511, 640, 698, 699])
    for h in (0, 13, 31):
        see = np.arange(n)[None] <= t[:, None]
        x = f64(q[0, h, t])
        ref, size, mean = attend(x, [(f64(k[0, h // 4]), x, np.zeros(len(t)), f64(v[0, h // 4]), see)])
        for o in out:
            assert (np.abs(f64(o[0, t, h]) - ref) <= tolerance(ref, size, mean, n, BF, True)).all()
