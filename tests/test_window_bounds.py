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
