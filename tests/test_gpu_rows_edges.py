"""The 8-bit caches and the drafted tokens at the edges of what their calls allow: counts out of range, addresses that are aligned to an element only,
a captured round of a server, offsets beyond 32 bits, many query heads of one token."""
import numpy as np
import pytest
import torch

import paper_2605_19218_amd as rk
from rows_util import D, DEV, attend, f64, kind, normal, rotation, tolerance, up32
from test_gpu_tree import BF, F32, Layer, ctx  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture
def blocks(monkeypatch):
    """Bounds for which the kernels of 64 and 128 rows a work-group are taken."""
    monkeypatch.setattr(Layer, "bound", staticmethod(lambda rows, units: 0 if rows <= 32 else 640000 // ((rows + 15) // 16 * units) + 1))


@pytest.mark.parametrize("dt,q8", [(BF, False), (BF, True), (F32, True)])
@pytest.mark.parametrize("T", [5, 40])
def test_counts_out_of_range(ctx, dt, q8, T):  # noqa: F811
    """Device counts below zero are none, above the host's as many as there are."""
    x = Layer(ctx, np.random.default_rng(T), dt, q8, 3, 8, 2, 64, [96, 0, 96], [50, 50, 0], T, [T, T, 0])
    for t, v in ((x.len, [1 << 30, -7, 97]), (x.text_len, [51, 1 << 30, -1]), (x.n_drafts, [T + 1, 1 << 30, -2])):
        t.copy_(torch.tensor(v, dtype=torch.int32))
    x.call()
    for t, v in ((x.len, x.lens), (x.text_len, x.tl), (x.n_drafts, x.nd)):
        t.copy_(torch.tensor(v, dtype=torch.int32))
    x.check()


@pytest.mark.parametrize("dt,q8", [(BF, False), (F32, False), (BF, True), (F32, True)])
@pytest.mark.parametrize("T,splits", [(3, 1), (3, 4), (40, 1), (40, 4)])
def test_results_of_any_place(ctx, blocks, dt, q8, T, splits):  # noqa: F811
    """Results may lie at any element, and touch nothing beside them."""
    rk.rk_set_option(ctx, rk.RK_OPT_DECODE_SPLITS, splits)
    try:
        x = Layer(ctx, np.random.default_rng(T), dt, q8, 2, 4, 2, 64, [300, 20], None, T, [T, T - 1])
        big = torch.full((x.out.numel() + 2,), 5.0, dtype=dt, device=DEV)
        x.call(out=big[1:-1])
    finally:
        rk.rk_set_option(ctx, rk.RK_OPT_DECODE_SPLITS, 0)
    assert big[0] == 5 and big[-1] == 5
    x.out = big[1:-1].view(x.out.shape)
    x.check()


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("r", [37, 64])
def test_rows_read_back_to_any_place(ctx, dt, r):  # noqa: F811
    x = Layer(ctx, np.random.default_rng(r), dt, True, 2, 2, 2, r, [96, 45], None, 1, [1, 1])
    out = []
    for off in (0, 1):
        k = torch.full((2 * 2 * 96 * r + 2,), 3.0, dtype=dt, device=DEV)
        v = torch.full((2 * 2 * 96 * D + 2,), 3.0, dtype=dt, device=DEV)
        rk.rk_unpack_cache_quant(ctx, x.lay, x.k, x.v, k[off:], v[off:])
        out.append((k[off:off + 2 * 2 * 96 * r], v[off:off + 2 * 2 * 96 * D]))
        assert (k[off + 2 * 2 * 96 * r:] == 3).all() and (v[off + 2 * 2 * 96 * D:] == 3).all() and (k[:off] == 3).all() and (v[:off] == 3).all()
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
    assert (out[0][0].view(2, 2, 96, r)[1, :, 45:] == 3).all() and (out[0][1].view(2, 2, 96, D)[1, :, 45:] == 3).all()


@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("T", [6, 40])
def test_captured_round(ctx, q8, T):  # noqa: F811
    """A round of a server in one graph, lengths growing in place: replays give what eager calls give, with other work between them."""
    def state():
        x = Layer(ctx, np.random.default_rng(T), BF, q8, 2, 8, 2, 64, [200, 31], [20, 5], T, [T, T - 2], poison=False)
        g = np.random.default_rng(1)
        x.kn, x.vn = normal(g, (2, 2, D), BF), normal(g, (2, 2, D), BF)
        x.path = torch.tensor([[0, 2, 2], [3, 1, 99]], dtype=torch.int32, device=DEV)
        x.n_path = torch.tensor([3, 3], dtype=torch.int32, device=DEV)
        roomy = [torch.zeros(2, 2, 64, D, dtype=BF, device=DEV) for _ in range(2)]
        for to, of in zip(roomy, (x.tk, x.tv)):
            to[:, :, :of.shape[2]] = of[:, :, :64]
        x.tk, x.tv = roomy
        x.text = rk.Text(x.tk, x.tv, 50, len=x.text_len)
        return x

    def turn(x, s):
        (rk.rk_append_quant(ctx, x.lay, x.kn, x.vn, x.Rr, x.k, x.v, x.len, stream=s) if q8 else
         rk.rk_append(ctx, x.lay, x.kn, x.vn, x.Rr, x.k, x.v, x.len, stream=s))
        x.call(stream=s)
        rk.rk_append_text_path(ctx, x.lay, x.text, x.drafts, x.path, x.n_path, x.text_len, stream=s)

    a, b = state(), state()
    for x in (a, b):
        x.lay.max_seq_len = 210
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        turn(a, s)                                # (warm)
        s.synchronize()
        with torch.cuda.graph(graph, stream=s):
            turn(a, s)
    turn(b, None)
    for i in range(5):
        b.out.fill_(0.0)
        turn(b, None)
        noise = torch.randn(4096, device=DEV).sum().item()
        graph.replay()
        torch.cuda.synchronize()
        assert np.isfinite(noise) and a.len.tolist() == b.len.tolist() == [202 + i, 33 + i]
        assert a.text_len.tolist() == b.text_len.tolist() == [20 + 3 * (i + 2), 5 + 2 * (i + 2)]
        live = [a.out[j, :n] for j, n in enumerate(a.nd)], [b.out[j, :n] for j, n in enumerate(b.nd)]
        assert all(torch.equal(p, q) for p, q in zip(*live))
        assert torch.equal(a.k, b.k) and torch.equal(a.v, b.v) and torch.equal(a.tk, b.tk) and torch.equal(a.tv, b.tv)


@pytest.mark.parametrize("T", [1, 3, 16, 40])
def test_calls_on_one_context_at_once(ctx, blocks, T):  # noqa: F811
    """Attention keeps nothing in the context: calls with workspaces of their own may overlap."""
    xs = [Layer(ctx, np.random.default_rng(31 + i), BF, bool(i & 1), 2, 16, 4, 64, [3000, 2000], [40, 3], T, [T, (T + 1) // 2]) for i in range(3)]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    for _ in range(6):
        for x, s in zip(xs, streams):
            x.call(stream=s)
    torch.cuda.synchronize()
    for x in xs:
        x.check()


@pytest.mark.parametrize("bound", [0, 220000])
@pytest.mark.parametrize("M", [0, 70])
@pytest.mark.parametrize("Hq", [33, 48, 130])
def test_many_query_heads(ctx, bound, M, Hq):  # noqa: F811
    """One token of more query heads a KV head than a work-group of few rows takes; the text's length is the host's."""
    N, r = 150, 48
    g = np.random.default_rng(Hq + M)
    Rr, dev = rotation(g, 1, 1, r), torch.tensor([N], dtype=torch.int32, device=DEV)
    lay = rk.Layout(1, Hq, 1, r, rk.RK_BF16, up32(max(N, bound)), max(N, bound), seq_len=dev)
    kb, vb = rk.rk_cache_bytes_quant(lay)
    kc, vc = (torch.full((n,), 0xff, dtype=torch.uint8, device=DEV) for n in (kb, vb))
    rk.rk_compress_quant(ctx, lay, rk.Rows(normal(g, (1, 1, N, D), BF), N), Rr, kc, rk.Rows(normal(g, (1, 1, N, D), BF), N), vc)
    tk, tv = normal(g, (1, 1, M + 1, D), BF), normal(g, (1, 1, M + 1, D), BF)
    q, out = normal(g, (1, Hq, D), BF), torch.zeros(1, Hq, D, dtype=BF, device=DEV)
    ws = torch.empty(rk.rk_tree_workspace_size(ctx, lay, 1), dtype=torch.uint8, device=DEV)
    rk.rk_decode_attn_quant(ctx, lay, q, kc, vc, Rr, None, rk.Text(tk, tv, M) if M else None, 0.0, out, ws)
    k32, v32 = (torch.zeros(1, 1, lay.capacity, w, device=DEV) for w in (r, D))
    rk.rk_unpack_cache_quant(ctx, rk.Layout(1, 1, 1, r, rk.RK_F32, lay.capacity, 0, seq_len=dev), kc, vc, k32, v32)
    ref, size, top = attend(f64(q)[:, None], f64(k32[:, :, :N]), f64(v32[:, :, :N]), [N], f64(Rr), None, (f64(tk), f64(tv)) if M else None, [M])
    assert (np.abs(f64(out) - ref[:, 0]) <= tolerance(ref, size, top, N + M, BF)[:, 0]).all()


@pytest.mark.parametrize("q8", [False, True])
def test_offsets_beyond_32_bits(ctx, q8):  # noqa: F811
    """A head of 17.5 million tokens, of which only the last weighs: 2.3 GB and more of Keys (bf16 4.5), and an index of elements beyond 2^31."""
    N = 17_499_990 if q8 else 17_000_000
    T = 40
    lens = torch.tensor([N], dtype=torch.int32, device=DEV)
    lay = rk.Layout(1, 1, 1, D, rk.RK_BF16, up32(N), N, seq_len=lens)
    K, V = (torch.zeros(1, 1, N, D, dtype=BF, device=DEV) for _ in range(2))
    g = np.random.default_rng(0)
    one, last = normal(g, (D,), BF), normal(g, (D,), BF)
    K[0, 0, -1], V[0, 0, -1] = 4 * one, last
    eye = torch.eye(D, device=DEV)[None, None].contiguous()
    kb, vb = (rk.rk_cache_bytes_quant if q8 else rk.rk_cache_bytes)(lay)
    kc, vc = (torch.empty(n, dtype=torch.uint8, device=DEV) for n in (kb, vb))
    put = rk.rk_compress_quant if q8 else rk.rk_compress
    put(ctx, lay, rk.Rows(K, N), eye, kc, values=rk.Rows(V, N), v_cache=vc)
    del K, V
    # 4 |one|^2 / sqrt(128) is some 45: e^-45 17.5e6 = 5e-13 beside a weight of one
    q = one.expand(1, T, 1, D).contiguous()
    text = None
    kd, vd = (torch.zeros(1, 1, T, D, dtype=BF, device=DEV) for _ in range(2))
    ws = torch.empty(rk.rk_tree_workspace_size(ctx, lay, T), dtype=torch.uint8, device=DEV)
    out = torch.zeros(1, T, 1, D, dtype=BF, device=DEV)
    f = rk.rk_decode_attn_tree_quant if q8 else rk.rk_decode_attn_tree
    want = last.float()
    held = want
    if q8:
        rows = torch.zeros(lay.capacity, D, dtype=F32, device=DEV)
        rk.rk_unpack_cache_quant(ctx, rk.Layout(1, 1, 1, D, rk.RK_F32, lay.capacity, 0, seq_len=lens), kc, vc, None, rows)
        held = rows[N - 1].clone()
        assert (held - want).abs().max() <= want.abs().max() / 127 * (1 + 2.0 ** -7) / 2 * 1.0001 and (rows[:N - 1] == 0).all()
    for n in (1, T):
        d = rk.Drafts(kd, vd, n, mask=torch.zeros(1, n, dtype=torch.int64, device=DEV), strides=(T * D, T * D, D))
        out.fill_(0.0)
        f(ctx, lay, q[:, :n].contiguous(), kc, vc, eye, None, None, d, 0.0, out, ws)
        got = out[0, :n, 0].float()
        assert (got - held).abs().max() <= 2.0 ** -8 * held.abs().max() + 2.0 ** -15 * held.abs().max()
    if q8:
        one_out = torch.zeros(1, 1, D, dtype=BF, device=DEV)
        rk.rk_decode_attn_quant(ctx, lay, q[:, 0].contiguous(), kc, vc, eye, None, None, 0.0, one_out, ws)
        assert torch.equal(one_out[0, 0], out[0, 0, 0]) or (one_out.float() - out[0, 0].float()).abs().max() <= 2.0 ** -7 * held.abs().max()
        rk.rk_append_quant(ctx, lay, one.view(1, 1, D), last.view(1, 1, D), eye, kc, vc, lens)
        rk.rk_unpack_cache_quant(ctx, rk.Layout(1, 1, 1, D, rk.RK_F32, lay.capacity, 0, seq_len=lens), kc, vc, None, rows)
        assert lens.tolist() == [N + 1] and torch.equal(rows[N], held) and torch.equal(rows[N - 1], held)
