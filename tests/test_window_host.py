"""Refusals of positions and of attention with a window, and the workspace it asks for (no GPU)."""
import pytest

import paper_2605_19218_amd as rk

P = 0x7f0000001000                   # an address that is looked at, never read
FAR = P + (1 << 33)
BAD, CAP, WS, NONE = rk.RK_ERR_INVALID_ARG, rk.RK_ERR_CAPACITY, rk.RK_ERR_WORKSPACE, rk.RK_ERR_NO_DEVICE


@pytest.fixture()
def ctx():
    c = rk.rk_create(rk.RK_DEVICE_NONE)
    yield c
    rk.rk_destroy(c)


def lay(**more):
    a = dict(batch=2, n_q_heads=8, n_kv_heads=2, keep=64, dtype=rk.RK_BF16, capacity=128, max_seq_len=100, seq_len=P)
    a.update(more)
    return rk.Layout(**a)


def text(**more):
    a = dict(k=P, v=P, max_len=10, len=P, capacity=40, strides=(2 * 40 * 128, 40 * 128, 128))
    a.update(more)
    return rk.Text(**a)


def heads(H, n=8, data=FAR, strides=None):
    return rk.Heads(data, strides=strides or (H * n * 128, n * 128, 128))


def rope(**more):
    a = dict(pos=P, inv_freq=P, axis=[0] * 32 + [1] * 16 + [2] * 16, n_axes=3, strides=(16, 8))
    a.update(more)
    return rk.Rope(**a)


def status(f, *a, **k):
    try:
        f(*a, **k)
    except rk.RotateKError as e:
        return e.status
    return rk.RK_OK


def test_rope(ctx):
    call = lambda L=lay(), r=rope(), n=8, q=heads(8), qo=heads(8), k=heads(2), ko=heads(2), **m: status(rk.rk_rope, ctx, L, r, n, q, qo, k, ko, **m)
    assert call() == NONE and call(k=None, ko=None) == NONE and call(q=None, qo=None) == NONE and call(n=0) == NONE
    assert call(r=None) == BAD and call(r=rope(pos=None)) == BAD and call(r=rope(inv_freq=None)) == BAD
    assert call(r=rope(n_axes=0)) == BAD and call(r=rope(n_axes=5)) == BAD and call(r=rope(n_axes=2)) == BAD     # (pairs of axis 2)
    assert call(r=rope(axis=[])) == BAD and call(r=rope(pairing=2)) == BAD and call(r=rope(strides=(-1, 8))) == BAD
    assert call(r=rope(axis=[0, 1, 3] + [0] * 61)) == BAD and call(r=rope(axis=[3], n_axes=4)) == NONE
    with pytest.raises(ValueError):
        call(r=rope(axis=[0] * 65))
    with pytest.raises(ValueError):
        call(r=rope(axis=[-1]))
    assert call(n=-1) == BAD and call(n=(1 << 30) + 1) == BAD
    assert call(L=lay(batch=1000), n=1 << 22) == rk.RK_ERR_UNSUPPORTED
    assert call(q=None, qo=None, k=None, ko=None) == BAD
    assert call(q=None) == BAD and call(qo=None) == BAD and call(k=None) == BAD and call(ko=None) == BAD
    assert call(q=heads(8, data=FAR + 8)) == BAD and call(q=heads(8, strides=(4, 128, 128))) == BAD and call(q=heads(8, strides=(-8, 128, 128))) == BAD
    assert call(flags=2) == BAD and call(flags=rk.RK_ROPE_INVERSE) == NONE
    assert call(L=lay(dtype=9)) == rk.RK_ERR_UNSUPPORTED and call(L=lay(head_dim=64)) == rk.RK_ERR_UNSUPPORTED
    # a source may be broadcast; a result may not
    assert call(q=heads(8, strides=(0, 0, 128))) == NONE and call(qo=heads(8, strides=(0, 1024, 128))) == BAD
    assert call(qo=heads(8, strides=(8 * 8 * 128, 128, 8 * 128))) == NONE                 # token by token
    assert call(qo=heads(8, strides=(8 * 12 * 128, 128, 12 * 128))) == NONE               # inside a projection
    assert call(qo=heads(8, strides=(8 * 4 * 128, 128, 4 * 128))) == BAD                  # heads over the next token's
    assert call(qo=heads(8, strides=(8 * 8 * 128, 8 * 128, 120))) == BAD
    assert call(L=lay(batch=1), qo=heads(8, strides=(0, 8 * 128, 128))) == NONE           # (one sequence does not step)
    assert status(rk.rk_rope, None, lay(), rope(), 8, heads(8), heads(8), None, None) == BAD


def test_rope_append_text(ctx):
    call = lambda L=lay(), r=rope(), n=8, q=heads(8), qo=heads(8), k=heads(2), v=heads(2), t=text(), out=P, **m: status(
        rk.rk_rope_append_text, ctx, L, r, n, q, qo, k, v, t, out, **m)
    assert call() == NONE and call(q=None, qo=None) == NONE
    assert call(q=None) == BAD and call(k=None) == BAD and call(v=None) == BAD and call(t=None) == BAD and call(out=None) == BAD
    assert call(t=text(len=None)) == BAD and call(t=text(k=P + 2)) == BAD and call(t=text(max_len=41)) == BAD and call(t=text(strides=(4, 4, 128))) == BAD
    assert call(n=0) == BAD and call(n=-4) == BAD
    assert call(t=text(max_len=32)) == NONE and call(t=text(max_len=33)) == CAP and call(n=41, q=None, qo=None, t=text(max_len=0)) == CAP
    assert call(t=text(max_len=2 ** 31 - 1, capacity=2 ** 31 - 1)) == CAP
    assert call(k=heads(2, data=P + 128)) == BAD and call(v=heads(2, data=P + 128)) == BAD      # over the segment
    assert call(qo=heads(8, strides=(0, 0, 128))) == BAD and call(r=rope(n_axes=9)) == BAD
    # strides whose products pass 64 bits: the stretch still meets the segment, and rows do not lie apart for it
    assert call(n=5, k=heads(2, data=P - 4096, strides=(0, 0, 1 << 62))) == BAD and call(n=5, k=heads(2, strides=(0, 0, 1 << 62))) == NONE
    assert call(qo=heads(8, strides=(1 << 62, 1 << 61, 128))) == BAD and call(qo=heads(8, strides=((1 << 63) - 8, 1 << 59, 128))) == NONE
    # the lengths that come out may lie over those that go in, not over the counts that every work-group reads
    assert call(n_tokens_dev=FAR) == NONE and call(n_tokens_dev=FAR, out=FAR) == BAD


def test_prefill(ctx):
    need = rk.rk_window_workspace_size(ctx, lay(), 8)
    call = lambda L=lay(), q=heads(8), n=8, t=text(), w=4, s=2, out=heads(8), ws=P, wb=need, **m: status(
        rk.rk_prefill_attn_window, ctx, L, q, n, t, w, s, 0.0, out, ws, workspace_bytes=wb, **m)
    assert call() == NONE and call(w=0, s=0) == NONE and call(t=text(len=None)) == NONE and call(w=2 ** 31 - 1, s=2 ** 31 - 1) == NONE
    assert call(w=-1) == BAD and call(s=-1) == BAD and call(n=0) == BAD and call(n=-1) == BAD
    assert call(q=None) == BAD and call(out=None) == BAD and call(t=None) == BAD
    assert call(out=heads(8, strides=(0, 0, 128))) == BAD and call(q=heads(8, strides=(0, 0, 128))) == NONE
    assert call(q=heads(8, data=FAR + 4)) == BAD and call(t=text(v=P + 4)) == BAD
    assert call(ws=None) == WS and call(wb=0) == WS and call(ws=P + 8) == WS
    assert call(t=text(max_len=2 ** 31 - 1, capacity=2 ** 31 - 1)) == BAD
    assert call(L=lay(batch=1000), n=1 << 22) == rk.RK_ERR_UNSUPPORTED


@pytest.mark.parametrize("f", [rk.rk_decode_attn_window, rk.rk_decode_attn_window_quant])
def test_decode(ctx, f):
    need = rk.rk_window_workspace_size(ctx, lay(), 1)
    call = lambda L=lay(), q=P, k=P, v=P, R=P, dmu=P, t=text(), w=4, s=2, out=P, ws=P, wb=need: status(
        f, ctx, L, q, k, v, R, dmu, t, w, s, 0.0, out, ws, workspace_bytes=wb)
    assert call() == NONE and call(dmu=None) == NONE and call(w=0) == NONE
    assert call(k=None, v=None) == NONE and call(k=None, v=None, R=None, dmu=None, L=lay(seq_len=None, max_seq_len=200)) == NONE
    assert call(k=None) == BAD and call(v=None) == BAD and call(R=None) == BAD and call(L=lay(seq_len=None)) == BAD
    assert call(q=None) == BAD and call(out=None) == BAD and call(t=None) == BAD and call(q=P + 2) == BAD and call(k=P + 2) == BAD
    assert call(w=-1) == BAD and call(s=-5) == BAD and call(t=text(max_len=50)) == BAD
    assert call(L=lay(max_seq_len=129)) == CAP
    assert call(ws=None) == WS and call(wb=16) == WS and call(ws=P + 4) == WS
    assert call(L=lay(batch=65535, n_q_heads=65534, n_kv_heads=2), wb=1 << 60) == rk.RK_ERR_UNSUPPORTED


def test_workspace():
    assert rk.rk_window_workspace_size(None, lay(), 0) == 0 and rk.rk_window_workspace_size(None, lay(keep=0), 1) == 0
    assert rk.rk_window_workspace_size(None, lay(), (1 << 30) + 1) == 0
    last = 0
    for n in list(range(1, 300)) + [1000, 4096, 1 << 30]:
        size = rk.rk_window_workspace_size(None, lay(), n)
        assert size >= last and size >= rk.rk_tree_workspace_size(None, lay(), 1)
        last = size
    assert last < 160 << 20


def test_prefill_plan():
    """Which kernel a prompt goes to, for 256 compute units: few rows on short prompts, many from where the device is full."""
    plan = lambda n, most, w=0, s=0, **m: rk.rk_prefill_plan(None, lay(**{**dict(batch=1, n_q_heads=32, n_kv_heads=8), **m}), n, most, w, s)
    assert plan(1, 1)[0] == 32 and plan(40, 1040, 512, 4)[0] == 32 and plan(300, 300)[0] == 32
    assert plan(500, 8500)[0] == 256 and plan(16384, 16384, 4096, 4) == (256, 1) and plan(100, 100, batch=64)[0] == 256
    assert plan(40, 1040, 512, 4, dtype=rk.RK_F32)[0] == 32 and plan(100, 100, batch=4, n_q_heads=56, dtype=rk.RK_F32)[0] == 128 and plan(500, 8500, dtype=rk.RK_F32)[0] == 256
    assert plan(1 << 20, 1 << 30)[1] == 1                      # (a full device takes no splits)
    for dtype in (rk.RK_F32, rk.RK_BF16):
        for batch, hq, hkv in ((1, 1, 1), (1, 32, 8), (8, 28, 4), (3, 64, 64)):
            for n in (1, 7, 64, 1000, 30000):
                for w in (0, 1, 100, 1 << 30, 2 ** 31 - 1):
                    L = lay(batch=batch, n_q_heads=hq, n_kv_heads=hkv, dtype=dtype)
                    rows, splits = rk.rk_prefill_plan(None, L, n, n + 5000, w, 2 ** 31 - 1)
                    assert splits >= 1 and (splits == 1 or 520 * batch * hq * n * splits + 256 <= rk.rk_window_workspace_size(None, L, n))
    for bad in (dict(n=0), dict(most=-1), dict(most=(1 << 30) + 1), dict(w=-1), dict(s=-1), dict(head_dim=64)):
        with pytest.raises(rk.RotateKError):
            plan(**{**dict(n=5, most=5), **bad})
