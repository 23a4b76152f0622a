"""Refusals of the 8-bit caches and of drafted tokens, and the sizes they ask for (no GPU)."""
import ctypes as C

import pytest

import paper_2605_19218_amd as rk

P = 0x7f0000001000                   # an address that is looked at, never read


@pytest.fixture()
def ctx():
    c = rk.rk_create(rk.RK_DEVICE_NONE)
    yield c
    rk.rk_destroy(c)


def lay(**more):
    a = dict(batch=2, n_q_heads=8, n_kv_heads=2, keep=64, dtype=rk.RK_BF16, capacity=128, max_seq_len=100, seq_len=P)
    a.update(more)
    return rk.Layout(**a)


def rows(**more):
    a = dict(data=P, n_tokens=100, strides=(2 * 128 * 128, 128 * 128, 128))
    a.update(more)
    return rk.Rows(**a)


def text(**more):
    a = dict(k=P, v=P, max_len=10, len=P, capacity=40, strides=(2 * 40 * 128, 40 * 128, 128))
    a.update(more)
    return rk.Text(**a)


def drafts(**more):
    a = dict(k=P + (1 << 30), v=P + (1 << 30), n_tokens=8, mask=P, n_tokens_dev=P, strides=(2 * 8 * 128, 8 * 128, 128))
    a.update(more)
    return rk.Drafts(**a)


def status(f, *a, **k):
    try:
        f(*a, **k)
    except rk.RotateKError as e:
        return e.status
    return rk.RK_OK


def test_sizes():
    L = lay()
    assert rk.rk_cache_bytes_quant(L) == (2 * 2 * 128 * (64 + 4), 2 * 2 * 128 * 128)
    assert rk.rk_cache_bytes_quant(lay(keep=37)) == (2 * 2 * 128 * (48 + 4), 2 * 2 * 128 * 128)
    assert rk.rk_cache_bytes_quant(lay(capacity=16384 + 128))[1] == 4 * (16384 + 256 + 64) * 128
    with pytest.raises(rk.RotateKError):
        rk.rk_cache_bytes_quant(lay(keep=0))
    assert rk.rk_tree_workspace_size(None, L, 0) == 0 and rk.rk_tree_workspace_size(None, L, 65) == 0
    assert rk.rk_tree_workspace_size(None, lay(capacity=31), 1) == 0
    for n in (1, 8, 64):
        one = rk.rk_tree_workspace_size(None, L, n)
        assert one >= 2 * n * 8 * 2 * 130 * 4
        assert one == rk.rk_tree_workspace_size(None, lay(capacity=1 << 20, max_seq_len=1 << 20), n)     # of no length


def test_compress_append_unpack(ctx):
    ok = rk.RK_ERR_NO_DEVICE
    call = lambda L=lay(), k=rows(), R=P, kc=P, v=rows(), vc=P: status(rk.rk_compress_quant, ctx, L, k, R, kc, values=v, v_cache=vc)  # noqa: E731
    bad = rk.RK_ERR_INVALID_ARG
    assert call() == ok
    assert call(k=None) == bad and call(v=None) == bad and call(R=None) == bad and call(kc=None) == bad and call(vc=None) == bad
    assert call(kc=P + 8) == bad and call(vc=P + 8) == bad and call(v=rows(n_tokens=99)) == bad and call(v=rows(tok_idx=P, tok_off=P)) == bad
    assert call(k=rows(n_tokens=129), v=rows(n_tokens=129)) == rk.RK_ERR_CAPACITY
    assert call(k=rows(strides=(0, 0, 64))) == bad and call(L=lay(head_dim=64)) == rk.RK_ERR_UNSUPPORTED
    call = lambda L=lay(), k=P, v=P, R=P, kc=P, vc=P, n=P: status(rk.rk_append_quant, ctx, L, k, v, R, kc, vc, n)  # noqa: E731
    assert call() == ok and call(L=lay(seq_len=None)) == bad and call(n=None) == bad and call(k=None) == bad and call(R=None) == bad
    assert call(L=lay(max_seq_len=128)) == rk.RK_ERR_CAPACITY and call(kc=P + 4) == bad
    call = lambda L=lay(), k=P, v=P, kr=P, vr=P: status(rk.rk_unpack_cache_quant, ctx, L, k, v, kr, vr)  # noqa: E731
    assert call() == ok and call(vr=None) == ok and call(kr=None) == ok and call(v=None, vr=None) == ok
    assert call(kr=None, vr=None) == bad and call(k=None, kr=None) == bad and call(v=None) == bad and call(k=P + 8) == bad


@pytest.mark.parametrize("q8", [False, True])
def test_tree(ctx, q8):
    f = rk.rk_decode_attn_tree_quant if q8 else rk.rk_decode_attn_tree
    need = rk.rk_tree_workspace_size(ctx, lay(), 8)

    def call(L=None, q=P, k=P, v=P, R=P, m=P, t=text(), d=drafts(), out=P, ws=P, n=need):
        return status(f, ctx, L or lay(), q, k, v, R, m, t, d, 0.0, out, ws, workspace_bytes=n)

    ok, bad = rk.RK_ERR_NO_DEVICE, rk.RK_ERR_INVALID_ARG
    assert call() == ok and call(t=None) == ok and call(m=None) == ok and call(t=text(len=None)) == ok
    assert call(d=drafts(mask=None, n_tokens_dev=None)) == ok and call(d=drafts(n_tokens=1)) == ok
    for arg in ("q", "k", "v", "R", "out", "d"):
        assert call(**{arg: None}) == bad, arg
    for arg in ("q", "k", "v"):
        assert call(**{arg: P + 8}) == bad, arg
    assert call(L=lay(seq_len=None)) == bad and call(L=lay(max_seq_len=129)) == rk.RK_ERR_CAPACITY
    assert call(ws=None) == rk.RK_ERR_WORKSPACE and call(ws=P + 8) == rk.RK_ERR_WORKSPACE and call(n=need - 1) == rk.RK_ERR_WORKSPACE
    for more in (dict(n_tokens=0), dict(n_tokens=65), dict(k=None), dict(v=None), dict(k=P + 8), dict(mask=P + 4), dict(strides=(0, 0, 64)),
                 dict(strides=(-8, 0, 128)), dict(strides=(0, 4, 128))):
        assert call(d=drafts(**more)) == bad, more
    for more in (dict(max_len=41), dict(k=None), dict(v=P + 2), dict(strides=(0, 0, 130))):
        assert call(t=text(**more)) == bad, more
    assert call(L=lay(batch=65535, n_q_heads=65528), n=1 << 60) == rk.RK_ERR_UNSUPPORTED


def test_decode_q8(ctx):
    need = rk.rk_tree_workspace_size(ctx, lay(), 1)
    call = lambda q=P, t=text(), n=need, ws=P: status(rk.rk_decode_attn_quant, ctx, lay(), q, P, P, P, P, t, 0.0, P, ws, workspace_bytes=n)  # noqa: E731
    assert call() == rk.RK_ERR_NO_DEVICE and call(t=None) == rk.RK_ERR_NO_DEVICE
    assert call(q=P + 2) == rk.RK_ERR_INVALID_ARG and call(n=need - 1) == rk.RK_ERR_WORKSPACE and call(ws=None) == rk.RK_ERR_WORKSPACE


def test_append_path(ctx):
    def call(t=text(), d=drafts(), path=P, n_path=P, out=P, n=8):
        return status(rk.rk_append_text_path, ctx, lay(), t, d, path, n_path, out, path_len=n)

    ok, bad = rk.RK_ERR_NO_DEVICE, rk.RK_ERR_INVALID_ARG
    assert call() == ok and call(n=30) == ok and call(n=31) == rk.RK_ERR_CAPACITY
    assert call(n=0) == bad and call(n=65, t=text(capacity=400, strides=(102400, 51200, 128))) == bad
    assert call(t=text(len=None)) == bad and call(path=None) == bad and call(n_path=None) == bad and call(out=None) == bad and call(d=None) == bad
    assert call(d=drafts(k=P + 2 * 128 * 11)) == bad          # rows of the segment itself
    assert call(t=None) == bad


def test_null_context():
    L = rk.lib()
    assert L.rk_decode_attn_tree(None, C.byref(lay().c()), P, P, P, P, P, None, C.byref(drafts().c()), 0.0, P, P, 1, None) == rk.RK_ERR_INVALID_ARG
    assert L.rk_compress_quant(None, None, None, None, None, None, None, None, None) == rk.RK_ERR_INVALID_ARG


def test_text_of_the_largest_bound(ctx):
    """A bound next to the largest int does not pass for a small one."""
    most = (1 << 31) - 1
    t = text(max_len=most, capacity=most)
    assert status(rk.rk_append_text_path, ctx, lay(), t, drafts(k=1 << 60, v=1 << 60), P, P, P, path_len=8) == rk.RK_ERR_CAPACITY
