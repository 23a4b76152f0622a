"""Infinite Values that a prompt's tokens see, in tiles on an edge and inside, and numbers next to the largest one of fp32: the same answer from every kernel of prompts."""
import numpy as np
import pytest
import torch

import paper_2605_19218_amd as rk
from rows_util import f64
from test_gpu_window_blocks import KERNELS, Prompt
from window_util import attend, sees, tolerance

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
LARGE = 3.4e38                       # above the largest 16-bit number, 3.39e38, below the largest of fp32


@pytest.fixture(scope="module")
def ctx():
    c = rk.rk_create(0)
    yield c
    rk.rk_destroy(c)


@pytest.mark.parametrize("shape", KERNELS)
def test_infinite_values(ctx, shape):
    """A token that sees a Value with an infinity in some channel has it there, one that sees both signs no number, and all else is as without them, bit for bit."""
    p = Prompt(ctx, *shape)
    B, n, held = shape[1], shape[4], shape[5]
    bad = sorted({1, held // 5, held // 3, held // 2, held - n // 2, held - n // 3, held - 2})
    sign = {j: (float("inf"), float("-inf"))[i % 2] for i, j in enumerate(bad)}
    channel = {j: 5 + 16 * i for i, j in enumerate(bad)}
    both = 127                       # (of the first and the last)
    for j in bad:
        p.v[:, :, j, channel[j]] = 0.0
    p.v[:, :, bad[0], both], p.v[:, :, bad[-1], both] = 0.0, 0.0
    p.call()
    clean = p.out.clone()
    for j in bad:
        p.v[:, :, j, channel[j]] = sign[j]
    p.v[:, :, bad[0], both], p.v[:, :, bad[-1], both] = float("inf"), float("-inf")
    p.call()
    for b in {0, B - 1}:
        m = p.counts[b]
        hit = sees(p.positions(b)[:, None], np.array(bad)[None], p.window, p.sinks) & (np.array(bad)[None] < p.lens[b])
        assert hit.any()
        want = clean[b, :m].clone()
        for i, j in enumerate(bad):
            want[torch.from_numpy(hit[:, i]).to(want.device), :, channel[j]] = sign[j]
        one, two = (torch.from_numpy(hit[:, i]).to(want.device) for i in (0, -1))
        want[one, :, both], want[two, :, both], want[one & two, :, both] = float("inf"), float("-inf"), float("nan")
        assert torch.equal(torch.isnan(p.out[b, :m]), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(p.out[b, :m], nan=7.0, posinf=1e30, neginf=-1e30), torch.nan_to_num(want, nan=7.0, posinf=1e30, neginf=-1e30))


@pytest.mark.parametrize("shape", [s for s in KERNELS if s[0] == F32])
def test_values_near_the_largest(ctx, shape):
    """One Value of 3.4e38 a channel among plain ones; equal Keys, so that all weights are 1 and no sum passes the range."""
    p = Prompt(ctx, *shape)
    held, n = shape[5], shape[4]
    p.k.zero_()
    for i, j in enumerate(sorted({1, held // 3, held // 2, held - n // 2, held - 2})):
        p.v[:, :, j, 3 + 16 * i] = LARGE if i % 2 else -LARGE
    p.call()
    last = shape[1] - 1
    p.check([(0, 0), (last, shape[2] - 1)], rows=[0, 1, n // 2, n - 2, n - 1])


@pytest.mark.parametrize("keys", [False, True])
@pytest.mark.parametrize("shape", [s for s in KERNELS if s[0] == F32])
def test_queries_and_keys_near_the_largest(ctx, shape, keys):
    """Queries (or Keys) of 3.4e38 in one channel, Keys (queries) of 2^-100 there, and a scale that makes scores of some tenths of them."""
    p = Prompt(ctx, *shape)
    n, scale = shape[4], 2.0 ** -30
    large, small = (p.k, p.q) if keys else (p.q, p.k)
    large.mul_(2.0 ** -20)
    small.mul_(2.0 ** -20)
    large[..., 70] = torch.sign(large[..., 70]) * LARGE
    small[..., 70] *= 2.0 ** -80
    rk.rk_prefill_attn_window(ctx, p.lay, rk.Heads(p.q), n, p.text, p.window, p.sinks, scale, rk.Heads(p.out.transpose(1, 2)), p.ws, n_tokens_dev=p.n_dev)
    last = shape[1] - 1
    for b, h in ((0, 0), (last, shape[2] - 1)):
        t = np.array([0, 1, n // 2, n - 2, n - 1]) % p.counts[b]
        hk = h // p.G
        q, see = f64(p.q[b, h, t]), sees(p.positions(b)[t][:, None], np.arange(p.lens[b])[None], p.window, p.sinks)
        ref, size, mean = attend(q, [(f64(p.k[b, hk, :p.lens[b]]), q, np.zeros(len(t)), f64(p.v[b, hk, :p.lens[b]]), see)], scale)
        assert (np.abs(f64(p.out[b, t, h]) - ref) <= tolerance(ref, size, mean, p.lens[b], F32, False)).all()
