"""Calls of positions and windows that no kernel can take: rows that many work-groups would write, launches past what the device takes (no GPU)."""
import pytest

import paper_2605_19218_amd as rk
from test_window_host import BAD, CAP, FAR, NONE, P, heads, lay, rope, status, text


@pytest.fixture()
def ctx():
    c = rk.rk_create(rk.RK_DEVICE_NONE)
    yield c
    rk.rk_destroy(c)


def test_segment_rows_lie_apart(ctx):
    """A segment that is read may be one for all heads or sequences; one that rows are appended to may not."""
    call = lambda L=lay(), n=8, H=2, **m: status(rk.rk_rope_append_text, ctx, L, rope(), n, None, None, heads(H), heads(H), text(**m), P)
    d = 128
    assert call() == NONE
    assert call(strides=(2 * 40 * d, 0, d)) == BAD and call(strides=(0, 40 * d, d)) == BAD and call(strides=(0, 0, d)) == BAD
    assert call(strides=(2 * 40 * d, 17 * d, d)) == BAD and call(strides=(2 * 40 * d, 18 * d, d)) == NONE        # 10 + 8 rows are in use
    assert call(strides=(2 * 40 * d, d, 2 * d)) == NONE and call(strides=(2 * 40 * d, d, d)) == BAD              # token by token; heads over the next token's
    assert call(strides=(2 * d, d, 4 * d)) == NONE and call(strides=(d, d, 4 * d)) == BAD                        # the sequences of a token side by side
    assert call(L=lay(batch=1), strides=(0, 40 * d, d)) == NONE                                                  # (one sequence, one head do not step)
    assert call(L=lay(batch=1, n_kv_heads=1), H=1, strides=(0, 0, d)) == NONE
    assert call(max_len=33, strides=(0, 0, d)) == CAP
    # attention only reads them
    need = rk.rk_window_workspace_size(ctx, lay(), 8)
    for strides in ((2 * 40 * d, 0, d), (0, 40 * d, d), (0, 0, d)):
        assert status(rk.rk_prefill_attn_window, ctx, lay(), heads(8), 8, text(strides=strides), 4, 2, 0.0, heads(8, data=FAR), P, workspace_bytes=need) == NONE
        assert status(rk.rk_decode_attn_window, ctx, lay(), P, None, None, None, None, text(strides=strides), 4, 2, 0.0, P, P, workspace_bytes=need) == NONE


LAUNCH = (1 << 32) - 1               # threads that a launch holds along an axis, at most
UNS = rk.RK_ERR_UNSUPPORTED


def test_more_tokens_than_a_launch(ctx):
    """Positions: 256 threads for eight tokens."""
    one = lambda h, n: rk.Heads(FAR, strides=(h * n * 128, n * 128, 128))
    L = lay(batch=1, n_q_heads=1, n_kv_heads=1)
    turn = lambda n: status(rk.rk_rope, ctx, L, rope(), n, one(1, n), one(1, n), None, None)
    most = LAUNCH // 256 * 8
    assert most == (1 << 27) - 8 and turn(most) == NONE and turn(most + 1) == UNS and turn(1 << 30) == UNS
    far = 1 << 50
    put = lambda n: status(rk.rk_rope_append_text, ctx, L, rope(), n, None, None, rk.Heads(far, strides=(0, 0, 128)), rk.Heads(far, strides=(0, 0, 128)),
                           text(max_len=0, capacity=1 << 30, strides=(1 << 40, 1 << 38, 128)), P)
    assert put(most) == NONE and put(most + 1) == UNS


@pytest.mark.parametrize("dtype", [rk.RK_BF16, rk.RK_F32])
def test_more_row_blocks_than_a_launch(ctx, dtype):
    """Prompts: the work-groups of all KV heads, as rk_prefill_plan says their rows are."""
    for n, lens in ((1, 10), (1, 5000), (300, 300)):
        for hkv in (1, 300, 65535):
            for batch in (1, 2, 255, 256, 257, 1000, 30000, 65535):
                if batch * hkv * n > 2 ** 31 - 1:
                    continue
                L = lay(batch=batch, n_q_heads=hkv, n_kv_heads=hkv, dtype=dtype)
                seen = []
                got = status(lambda: seen.append(rk.rk_prefill_plan(ctx, L, n, lens, 0, 0)))
                rows, splits = seen[0] if seen else (32, 1)
                groups = batch * hkv * ((n + rows - 1) // rows) * splits
                fits = groups * (512 if dtype == rk.RK_F32 and rows == 256 else 256) <= LAUNCH
                assert got == (rk.RK_OK if fits else UNS), (n, lens, hkv, batch)
                t = text(max_len=lens, capacity=lens, strides=(hkv * lens * 128, lens * 128, 128))
                x = rk.Heads(FAR, strides=(hkv * n * 128, n * 128, 128))
                assert status(rk.rk_prefill_attn_window, ctx, L, x, n, t, 0, 0, 0.0, x, P, workspace_bytes=1 << 62) == (NONE if fits else UNS)
    assert status(rk.rk_prefill_plan, ctx, lay(batch=65535, n_q_heads=300, n_kv_heads=300), 1, 10, 0, 0) == UNS


@pytest.mark.parametrize("f", [rk.rk_decode_attn_window, rk.rk_decode_attn_window_quant])
def test_more_heads_than_a_launch(ctx, f):
    """One token: a work-group a KV head and split, and the fold, eight rows a work-group."""
    def call(batch, hq, hkv, cache):
        kv = P if cache else None
        return status(f, ctx, lay(batch=batch, n_q_heads=hq, n_kv_heads=hkv), P, kv, kv, kv, None, text(), 4, 2, 0.0, P, P, workspace_bytes=1 << 62)
    assert call(65535, 256, 256, False) == NONE and call(65535, 257, 257, False) == UNS
    assert call(65535, 128, 128, True) == NONE and call(65535, 129, 129, True) == UNS          # the cache's work-group and the text's
    assert call(65535, 16 * 2047, 2047, False) == UNS and call(65535, 16 * 200, 200, False) == NONE


@pytest.mark.parametrize("f", [rk.rk_decode_attn_window, rk.rk_decode_attn_window_quant])
def test_longest_text(ctx, f):
    """One token: the last rows of a text are numbered in 32 bits with a tile to spare, as a prompt's are."""
    call = lambda n: status(f, ctx, lay(), P, None, None, None, None, text(max_len=n, capacity=2 ** 31 - 1), 4, 2, 0.0, P, P, workspace_bytes=1 << 62)
    assert call(1 << 30) == NONE and call((1 << 30) + 1) == BAD and call(2 ** 31 - 1) == BAD
