"""Operators in front of and beside the rotated cache: positions of several axes, prompts into the text segment, attention with a window.

Four operators on one attention layer, each as a user calls it through the binding and in its plain form:
  rope     the positions of a prompt's queries and Keys, put on or taken off         rk_rope
  append   positions, and new tokens behind the text segment                         rk_rope_append_text
  prefill  the attention of new tokens over the text segment, window and sinks       rk_prefill_attn_window
  decode   one token over the rotated cache and the windowed text segment            rk_decode_attn_window, rk_decode_attn_window_quant

Positions: pair i of a row's channels turns by pos[axis of i] * inv_freq[i]. A window of w tokens and s sinks: the token at position p
attends the text rows j <= p with j < s or p - j < w (w = 0: all of them).
"""
import math
import random

import torch

own = False

DEV, D = "cuda", 128
_ctx = None


def _rk():
    import paper_2605_19218_amd as rk
    return rk


def _context():
    global _ctx
    if _ctx is None:
        _ctx = _rk().rk_create(0)
    return _ctx


# ---- the cases --------------------------------------------------------------------------------------------
def _case(name, op, B, Hq, Hkv, n, dtype="bf16", **more):
    """n: new tokens a sequence; text: rows that the segment holds (in front of the new ones); L, r: the rotated cache."""
    c = dict(name=name, op=op, B=B, Hq=Hq, Hkv=Hkv, n=n, dtype=dtype, ragged=False, text=0, window=0, sinks=0, L=0, r=0, q8=False,
             axes=3, order="blocks", pairs=64, adjacent=False, inverse=False)
    c.update(more)
    return c


def listed():
    return [
        # a follow-up question of a chat: launches and latency
        _case("rope_question", "rope", 1, 32, 8, 71),
        # the positions of a LLaVA-shaped fp32 prompt are taken off its Keys and queries again (also the gradient's way)
        _case("rope_off_llava_f32", "rope", 1, 32, 32, 2944, "f32", inverse=True),
        # image and video prompts of the benchmark's layer, a batch of 8 of all lengths up to 16K tokens, out of one projection
        _case("rope_16k_gqa", "rope", 8, 28, 4, 16384, ragged=True),
        # one generated token of a chat
        _case("append_token", "append", 1, 32, 8, 1, text=500),
        # one generated token each of a full serving batch of a multi-head model
        _case("append_token_batch_mha", "append", 64, 32, 32, 1, text=150, ragged=True),
        # prompts of up to 1000 tokens behind what the segments hold
        _case("append_prompts_gqa", "append", 8, 28, 4, 1000, text=500, ragged=True),
        # a short question behind a chat of 1000 tokens, on a layer with a sliding window
        _case("prefill_question", "prefill", 1, 32, 8, 40, text=1000, window=512, sinks=4),
        # a LLaVA-shaped fp32 layer's prompt, all of it visible
        _case("prefill_llava_f32", "prefill", 1, 32, 32, 2944, "f32"),
        # a prompt of 16K tokens on the benchmark's layer, a sliding window of a quarter of it: compute-bound
        _case("prefill_16k_gqa", "prefill", 1, 28, 4, 16384, window=4096, sinks=4),
        # one token of a sliding-window layer, which has no rotated cache
        _case("decode_window_chat", "decode", 1, 32, 8, 1, text=1500, window=1024, sinks=4),
        # one token of a LLaVA-shaped fp32 layer beside a long answer
        _case("decode_llava_f32", "decode", 1, 32, 32, 1, "f32", text=700, window=256, sinks=16, L=2880, r=64),
        # the benchmark's layer with its cache in 8 bits, late in a long conversation
        _case("decode_16k_gqa_q8", "decode", 8, 28, 4, 1, text=6000, window=2048, sinks=4, L=16384, r=64, q8=True, ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    op = rng.choice(["rope", "append", "prefill", "prefill", "decode", "decode"])
    f32 = rng.random() < 0.25
    Hkv = rng.choice([1, 2, 4, 8, 8, 16, 32])
    Hq = Hkv * (rng.choice([1, 2]) if Hkv == 32 else rng.choice([1, 2, 3, 4, 7, 8]))
    B = rng.choice([1, 1, 2, 3, 4, 8, 16])
    c = _case("", op, B, Hq, Hkv, 1, "f32" if f32 else "bf16")
    del c["name"]
    c["axes"] = rng.choice([1, 2, 3, 3, 3, 4])
    c["order"] = rng.choice(["blocks", "turns"])
    c["pairs"] = rng.choice([64, 64, 64, 32, 48, 13])
    c["adjacent"] = rng.random() < 0.3
    if op in ("prefill", "decode"):
        c["window"] = rng.choice([0, _log(rng, 1, 8192)])
        c["sinks"] = rng.choice([0, 1, 4, 4, 16, 128]) if c["window"] else 0
    if op == "rope":
        c["n"] = _log(rng, 1, 16384)
        c["inverse"] = rng.random() < 0.3
        while c["B"] * Hq * c["n"] > (800_000 if f32 else 1_600_000):
            c["n"] = c["n"] // 2 + rng.randrange(2)
    elif op == "append":
        c["n"] = rng.choice([1, 1, _log(rng, 2, 4096)])
        c["text"] = rng.randint(0, 2000)
        while c["B"] * Hq * (c["n"] + c["text"]) > (400_000 if f32 else 800_000):
            c["n"], c["text"] = c["n"] // 2 + 1, c["text"] // 2
    elif op == "prefill":
        c["n"] = _log(rng, 1, 16384)
        c["text"] = rng.choice([0, _log(rng, 1, 8000)])
        while c["B"] * Hq * _pairs_of(c["n"], c["n"] + c["text"], c["window"], c["sinks"]) > (100_000_000 if f32 else 1_200_000_000):
            c["n"], c["text"] = c["n"] // 2 + rng.randrange(2), c["text"] * 3 // 4
    else:
        c["text"] = _log(rng, 1, 10000)
        if rng.random() < 0.7:
            c["L"], c["r"], c["q8"] = _log(rng, 1, 33000), rng.choice([16, 24, 32, 37, 48, 64, 64, 80, 96, 128]), rng.random() < 0.5
        while c["B"] * Hkv * (c["L"] + c["text"]) > (200_000 if f32 else 520_000):
            if c["B"] > 1:
                c["B"] = max(1, c["B"] // 2)
            else:
                c["L"], c["text"] = c["L"] // 2, max(1, c["text"] // 2)
        if not c["L"]:
            c["r"], c["q8"] = 0, False
    c["ragged"] = c["B"] > 1 and rng.random() < 0.5
    return c


# ---- inputs -------------------------------------------------------------------------------------------------
def _lens(c, key, most, least=1):
    """A length a sequence: part of the case, so that its work is known. One of a ragged batch has the most."""
    if not c["ragged"] or most <= least:
        return [most] * c["B"]
    g = random.Random("%s %d %d %d" % (key, c["B"], c["Hkv"], most))
    n = [g.randint(max(least, most // 16), most) for _ in range(c["B"])]
    n[g.randrange(c["B"])] = most
    return n


def _axis_of_pairs(c):
    """The axis of each pair: three consecutive sections (the first axis the smaller one), or the axes in turn."""
    a, p = c["axes"], c["pairs"]
    if c["order"] == "turns":
        return [i % a for i in range(p)]
    first = p if a == 1 else max(1, p // (a + 1))
    return [0 if i < first else 1 + (i - first) * (a - 1) // (p - first) for i in range(p)]


def _pairs_of(n, length, window, sinks):
    """(query, row) pairs of a sequence: what the queries at the last n of `length` positions see."""
    total = 0
    first = length - n
    if not window:
        return n * first + n * (n + 1) // 2
    for lo, hi, seen in ((first, min(length, window), None), (max(first, window), length, window)):
        if hi > lo:
            total += (hi - lo) * seen if seen else (hi * (hi + 1) - lo * (lo + 1)) // 2
    for lo, hi in ((max(first, window), min(length, window + sinks)),):      # sinks that the window has left behind, one more a step
        if hi > lo:
            total += sum(p - window + 1 for p in range(lo, hi))
    lo = max(first, window + sinks)
    return total + max(0, length - lo) * sinks


def _rows_of(n, length, window, sinks):
    """Rows that any of these queries sees."""
    if not window:
        return length
    lo = max(0, length - n - window + 1)
    return length - lo + min(sinks, lo)


def _up(n):
    return max(32, (n + 31) // 32 * 32)


def _dt(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class _State:
    pass


def _rotation(g, B, H, r):
    """The first r columns of a product of four reflections: orthonormal."""
    R = torch.eye(D, device=DEV).expand(B, H, D, D)
    for _ in range(4):
        v = torch.randn(B, H, D, 1, device=DEV, generator=g)
        v = v / v.norm(dim=2, keepdim=True)
        R = R - 2 * torch.matmul(R, v) * v.transpose(2, 3).contiguous()
    return R[..., :r].contiguous()


def _coded(g, shape, low, high, dt):
    """Rows as an 8-bit cache holds them: whole numbers up to 127 (once in each row) by a power of two, exact in any type."""
    c = torch.randn(*shape, device=DEV, generator=g).mul_(36).round_().clamp_(-127, 127)
    at = torch.randint(0, shape[-1], shape[:-1] + (1,), device=DEV, generator=g)
    c.scatter_(-1, at, 127.0)
    e = torch.randint(low, high + 1, shape[:-1] + (1,), device=DEV, generator=g).float()
    return (c * torch.exp2(e)).to(dt)


def _positions(c, g, first):
    """[axes, B, n] int32: images of 24 columns behind some text; time stands still inside an image, behind it all axes go on from the largest."""
    B, n, axes = c["B"], c["n"], c["axes"]
    t = torch.arange(n, device=DEV)[None] + torch.randint(0, 32, (B, 1), device=DEV, generator=g)
    base = first[:, None].long() + t // 640 * 64
    place = t % 640                                                     # of each 640 tokens: 64 of text, 576 of an image
    image = place >= 64
    row, col = (place - 64) // 24, (place - 64) % 24
    per = [base + torch.where(image, 64, place)]
    for a in range(1, axes):
        per.append(base + torch.where(image, 64 + (row if a % 2 else col), place))
    return torch.stack(per).to(torch.int32).contiguous()


def prepare(case, seed):
    c, s = case, _State()
    s.c = c
    g = torch.Generator(device=DEV)
    g.manual_seed(1_000_003 * seed + 29)
    B, Hq, H, n, dt = c["B"], c["Hq"], c["Hkv"], c["n"], _dt(c)

    def normal(*shape, std=1.0):
        x = torch.empty(*shape, device=DEV, dtype=dt)
        for b in range(shape[0]):
            x[b] = (torch.randn(*shape[1:], device=DEV, generator=g) * std).to(dt)
        return x

    s.scale = 1.0 / math.sqrt(D)
    s.n = _lens(c, "new", n)
    s.n_dev = _int32(s.n)
    if c["op"] in ("rope", "append"):
        # a projection's rows: the queries' heads, the Keys', the Values'
        s.qkv = normal(B, n, Hq + 2 * H, D)
        s.held = _lens(c, "held", c["text"], 0)
        s.text_len = _int32(s.held)
        s.axis = _axis_of_pairs(c)
        s.inv_freq = (10000.0 ** (-torch.arange(c["pairs"], device=DEV, dtype=torch.float64) / c["pairs"])).float()
        s.pos = _positions(c, g, s.text_len if c["op"] == "append" else torch.randint(0, 60000, (B,), device=DEV, generator=g))
        s.q = s.qkv[:, :, :Hq].transpose(1, 2)
        s.k = s.qkv[:, :, Hq:Hq + H].transpose(1, 2)
        s.v = s.qkv[:, :, Hq + H:].transpose(1, 2)
        s.axis_dev = torch.tensor(s.axis, device=DEV)
        s.q_out = torch.zeros(B, n, Hq, D, device=DEV, dtype=dt)
    if c["op"] == "rope":
        s.k_out = torch.zeros(B, H, n, D, device=DEV, dtype=dt)
    if c["op"] == "append":
        s.kt, s.vt = normal(B, H, c["text"] + n, D), normal(B, H, c["text"] + n, D)
        s.len_out = torch.zeros(B, dtype=torch.int32, device=DEV)
    if c["op"] == "prefill":
        s.held = [a + b for a, b in zip(_lens(c, "held", c["text"], 0), s.n)]
        s.text_len = _int32(s.held)
        s.q = normal(B, n, Hq, D).transpose(1, 2)
        s.kt, s.vt = normal(B, H, c["text"] + n, D), normal(B, H, c["text"] + n, D)
        s.out = torch.zeros(B, n, Hq, D, device=DEV, dtype=dt)
    if c["op"] == "decode":
        s.held = _lens(c, "held", c["text"])
        s.text_len = _int32(s.held)
        s.q = normal(B, Hq, D)
        s.kt, s.vt = normal(B, H, c["text"], D), normal(B, H, c["text"], D)
        s.out = torch.zeros(B, Hq, D, device=DEV, dtype=dt)
        if c["L"]:
            L, r = c["L"], c["r"]
            s.cached = _lens(c, "cached", L)
            s.len = _int32(s.cached)
            s.Rr = _rotation(g, B, H, r)
            if c["q8"]:
                s.Kt, s.Vt = _coded(g, (B, H, L, r), -6, -3, dt), _coded(g, (B, H, L, D), -6, -4, dt)
            else:
                s.Kt, s.Vt = normal(B, H, L, r, std=1.5), normal(B, H, L, D)
            s.dmu = 0.3 * torch.randn(B, H, D, device=DEV, generator=g)
    if own:
        _hold(s)
    return s


def _hold(s):
    """What a program that uses the framework has at hand: the caches as the framework holds them, the segment, workspace."""
    rk, c = _rk(), s.c
    ctx = s.ctx = _context()
    B, Hq, H, n, L, r, dt = c["B"], c["Hq"], c["Hkv"], c["n"], c["L"], c["r"], _dt(c)
    kind = rk.RK_F32 if c["dtype"] == "f32" else rk.RK_BF16
    s.lay = rk.Layout(B, Hq, H, r or D, kind, _up(L), L, seq_len=getattr(s, "len", None))
    if c["op"] in ("rope", "append"):
        s.rope = rk.Rope(s.pos, s.inv_freq, axis=s.axis, pairing=rk.RK_ROPE_ADJACENT if c["adjacent"] else rk.RK_ROPE_HALVES)
        s.heads = [rk.Heads(x) for x in (s.q, s.k, s.v, s.q_out.transpose(1, 2))]
    if c["op"] == "rope":
        s.k_heads = rk.Heads(s.k_out)
        s.flags = rk.RK_ROPE_INVERSE if c["inverse"] else 0
    if c["op"] == "append":
        s.segment = rk.Text(s.kt, s.vt, c["text"], len=s.text_len)
    if c["op"] == "prefill":
        s.segment = rk.Text(s.kt, s.vt, c["text"] + n, len=s.text_len)
        s.heads = [rk.Heads(s.q), rk.Heads(s.out.transpose(1, 2))]
        s.ws = torch.empty(rk.rk_window_workspace_size(ctx, s.lay, n), dtype=torch.uint8, device=DEV)
    if c["op"] == "decode":
        s.segment = rk.Text(s.kt, s.vt, c["text"], len=s.text_len)
        s.ws = torch.empty(rk.rk_window_workspace_size(ctx, s.lay, 1), dtype=torch.uint8, device=DEV)
        s.kc = s.vc = None
        if L:
            kb, vb = rk.rk_cache_bytes_quant(s.lay) if c["q8"] else rk.rk_cache_bytes(s.lay)
            s.kc = torch.zeros(kb, dtype=torch.uint8, device=DEV)
            s.vc = torch.zeros(vb, dtype=torch.uint8, device=DEV)
            # rows that are exact in the cache's form, through the columns of the identity
            pick = torch.eye(D, device=DEV)[:, :r].expand(B, H, D, r).contiguous()
            wide = torch.zeros(B, H, L, D, device=DEV, dtype=dt)
            wide[..., :r] = s.Kt
            put = rk.rk_compress_quant if c["q8"] else rk.rk_compress
            put(ctx, s.lay, rk.Rows(wide, L, n_tokens_dev=s.len), pick, s.kc, values=rk.Rows(s.Vt, L, n_tokens_dev=s.len), v_cache=s.vc)
            torch.cuda.synchronize()


# ---- one pass -----------------------------------------------------------------------------------------------
def run(s):
    return {"rope": _rope, "append": _append, "prefill": _prefill, "decode": _decode}[s.c["op"]](s)


def _turns(s, sign):
    """cos and sin [B, 1, n, pairs] in fp32 of angles in 64 bits."""
    at = s.pos.double()[s.axis_dev]                                  # [pairs, B, n]
    angle = (at * s.inv_freq.double()[:, None, None]).permute(1, 2, 0)[:, None]
    return torch.cos(angle).float(), (sign * torch.sin(angle)).float()


def _turned(c, x, cos, sin):
    """Rows [B, heads, n, d] turned, in fp32."""
    x, p = x.float(), c["pairs"]
    if c["adjacent"]:
        a, b = x[..., 0:2 * p:2], x[..., 1:2 * p:2]
        both = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = x[..., :p], x[..., p:2 * p]
        both = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([both, x[..., 2 * p:]], -1) if p < D // 2 else both


def _rope(s):
    c = s.c
    if own:
        _rk().rk_rope(s.ctx, s.lay, s.rope, c["n"], s.heads[0], s.heads[3], s.heads[1], s.k_heads, flags=s.flags, n_tokens_dev=s.n_dev)
        return s.q_out, s.k_out
    cos, sin = _turns(s, -1.0 if c["inverse"] else 1.0)
    there = (torch.arange(c["n"], device=DEV)[None] < s.n_dev[:, None])[:, None, :, None]
    q = torch.where(there, _turned(c, s.q, cos, sin), 0).to(_dt(c)).transpose(1, 2).contiguous()
    return q, torch.where(there, _turned(c, s.k, cos, sin), 0).to(_dt(c))


def _append(s):
    c = s.c
    if own:
        _rk().rk_rope_append_text(s.ctx, s.lay, s.rope, c["n"], s.heads[0], s.heads[3], s.heads[1], s.heads[2], s.segment, s.len_out,
                                  n_tokens_dev=s.n_dev)
        return s.q_out, s.kt, s.vt, s.len_out
    B, H, n = c["B"], c["Hkv"], c["n"]
    cos, sin = _turns(s, 1.0)
    t = torch.arange(n, device=DEV)
    there = (t[None] < s.n_dev[:, None])[:, None, :, None]
    q = torch.where(there, _turned(c, s.q, cos, sin), 0).to(_dt(c)).transpose(1, 2).contiguous()
    at = (s.text_len[:, None].long() + t)[:, None, :, None].expand(B, H, n, D)
    s.kt.scatter_(2, at, torch.where(there, _turned(c, s.k, cos, sin).to(_dt(c)), torch.gather(s.kt, 2, at)))
    s.vt.scatter_(2, at, torch.where(there, s.v, torch.gather(s.vt, 2, at)))
    return q, s.kt, s.vt, s.text_len + s.n_dev


def _prefill(s):
    c = s.c
    if own:
        _rk().rk_prefill_attn_window(s.ctx, s.lay, s.heads[0], c["n"], s.segment, c["window"], c["sinks"], s.scale, s.heads[1], s.ws,
                                     n_tokens_dev=s.n_dev)
        return s.out
    Hq, H = c["Hq"], c["Hkv"]
    G, w, first = Hq // H, c["window"], c["sinks"]
    out = torch.zeros_like(s.out)
    for b, (n, held) in enumerate(zip(s.n, s.held)):
        step = max(16, min(n, 100_000_000 // (Hq * min(held, (w or held) + first + 512))))
        for t0 in range(0, n, step):
            t1 = min(n, t0 + step)
            p = torch.arange(held - n + t0, held - n + t1, device=DEV)
            lo = max(0, held - n + t0 - w + 1) if w else 0               # the rows that these tokens may see
            j = torch.cat([torch.arange(min(first, lo), device=DEV), torch.arange(lo, held - n + t1, device=DEV)])
            q = s.q[b, :, t0:t1].float().reshape(H, G * (t1 - t0), D)
            x = torch.bmm(q, s.kt[b][:, j].float().transpose(1, 2).contiguous()).view(H, G, t1 - t0, -1)
            seen = j[None] <= p[:, None]
            if w:
                seen &= (j[None] < first) | (p[:, None] - j[None] < w)
            x.masked_fill_(~seen, float("-inf"))
            x = torch.exp((x - x.amax(-1, keepdim=True)).mul_(s.scale))
            o = torch.bmm((x / x.sum(-1, keepdim=True)).view(H, G * (t1 - t0), -1), s.vt[b][:, j].float())
            out[b, t0:t1] = o.view(Hq, t1 - t0, D).transpose(0, 1).to(out.dtype)
    return out


def _decode(s):
    c = s.c
    if own:
        rk = _rk()
        call = rk.rk_decode_attn_window_quant if c["q8"] else rk.rk_decode_attn_window
        call(s.ctx, s.lay, s.q, s.kc, s.vc, s.Rr if c["L"] else None, s.dmu if c["L"] else None, s.segment, c["window"], c["sinks"],
             s.scale, s.out, s.ws)
        return s.out
    B, Hq, H = c["B"], c["Hq"], c["Hkv"]
    G, w, first, low = Hq // H, c["window"], c["sinks"], float("-inf")
    q = s.q.float().view(B, H, G, D)
    j, held = torch.arange(c["text"], device=DEV)[None], s.text_len[:, None]
    seen = (j < held) & ((j < first) | (j >= held - w)) if w else j < held
    x = torch.matmul(q, s.kt.float().transpose(2, 3).contiguous())
    parts, values = [x.masked_fill_(~seen[:, None, None, :], low)], [s.vt]
    if c["L"]:
        there = torch.arange(c["L"], device=DEV)[None] < s.len[:, None]
        x = torch.matmul(torch.matmul(q, s.Rr), s.Kt.float().transpose(2, 3).contiguous()) + torch.matmul(q, s.dmu[..., None])
        parts.append(x.masked_fill_(~there[:, None, None, :], low))
        values.append(s.Vt)
    most = torch.stack([p.amax(-1, keepdim=True) for p in parts]).amax(0)
    parts = [torch.exp((p - most).mul_(s.scale)) for p in parts]
    total = sum(p.sum(-1, keepdim=True) for p in parts)
    out = sum(torch.matmul(p, v.float()) for p, v in zip(parts, values)) / total
    return out.view(B, Hq, D).to(_dt(c))


# ---- what a pass cannot do without ---------------------------------------------------------------------------
def work(case):
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    H, Hq = c["Hkv"], c["Hq"]
    new = sum(_lens(c, "new", c["n"]))
    if c["op"] == "rope":
        return {"bytes": new * (2 * (Hq + H) * D * e + 4 * c["axes"]), "flops": new * (Hq + H) * 6 * c["pairs"]}
    if c["op"] == "append":
        return {"bytes": new * (2 * (Hq + 2 * H) * D * e + 4 * c["axes"]), "flops": new * (Hq + H) * 6 * c["pairs"]}
    size = flops = 0
    if c["op"] == "prefill":
        for n, held in zip(_lens(c, "new", c["n"]), _lens(c, "held", c["text"], 0)):
            size += 2 * (n * Hq + _rows_of(n, held + n, c["window"], c["sinks"]) * H) * D * e
            flops += 4 * D * Hq * _pairs_of(n, held + n, c["window"], c["sinks"])
        return {"bytes": size, "flops": flops}
    cached = _lens(c, "cached", c["L"]) if c["L"] else [0] * c["B"]
    each = c["r"] + D + 4 if c["q8"] else (c["r"] + D) * e
    for held, m in zip(_lens(c, "held", c["text"]), cached):
        rows = _rows_of(1, held, c["window"], c["sinks"])
        size += H * (2 * rows * D * e + m * each + (D * (c["r"] + 1) * 4 if c["L"] else 0)) + 2 * Hq * D * e
        flops += 2 * Hq * (2 * D * rows + m * (c["r"] + D) + D * c["r"])
    return {"bytes": size, "flops": flops}


# ---- the definition in 64 bits --------------------------------------------------------------------------------
def _exact_rotated(s, x, b, n, sign):
    """Rows [heads, n, d] as complex numbers times e^(i angle)."""
    c, p = s.c, s.c["pairs"]
    x = x[:, :n].to(torch.float64)
    one, two = (range(0, 2 * p, 2), range(1, 2 * p, 2)) if c["adjacent"] else (range(p), range(p, 2 * p))
    one, two = torch.tensor(list(one), device=DEV), torch.tensor(list(two), device=DEV)
    angle = torch.stack([s.pos[a, b, :n].to(torch.float64) * s.inv_freq[i].to(torch.float64) for i, a in enumerate(s.axis)], -1)
    z = torch.complex(x[..., one], x[..., two]) * torch.polar(torch.ones_like(angle), sign * angle)
    y = x.clone()
    y[..., one], y[..., two] = z.real, z.imag
    return y


def _exact_attention(q, keys, vals, seen):
    """[rows, d] of float64 against [m, d]; seen [rows, m]."""
    w = (q @ keys.T.contiguous() / math.sqrt(D)).masked_fill(~seen, -math.inf)
    return torch.softmax(w, -1) @ vals


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    B, Hq, H, n, f64 = c["B"], c["Hq"], c["Hkv"], c["n"], torch.float64
    G = Hq // H
    if c["op"] in ("rope", "append"):
        sign = -1.0 if c["inverse"] else 1.0
        q = torch.zeros(B, n, Hq, D, device=DEV, dtype=f64)
        k = torch.zeros(B, H, n, D, device=DEV, dtype=f64) if c["op"] == "rope" else s.kt.to(f64)
        v = None if c["op"] == "rope" else s.vt.to(f64)
        for b, m in enumerate(s.n):
            q[b, :m] = _exact_rotated(s, s.q[b], b, m, sign).transpose(0, 1)
            at = 0 if c["op"] == "rope" else s.held[b]
            k[b, :, at:at + m] = _exact_rotated(s, s.k[b], b, m, sign)
            if v is not None:
                v[b, :, at:at + m] = s.v[b, :, :m].to(f64)
        return (q, k) if v is None else (q, k, v, _int32([a + m for a, m in zip(s.held, s.n)]))
    if c["op"] == "prefill":
        if work(c)["flops"] > 4e12:
            return None
        out = torch.zeros(B, n, Hq, D, device=DEV, dtype=f64)
        for b, (m, held) in enumerate(zip(s.n, s.held)):
            for h in range(Hq):
                keys, vals = s.kt[b, h // G, :held].to(f64), s.vt[b, h // G, :held].to(f64)
                for t in range(0, m, 1024):
                    p = held - m + torch.arange(t, min(m, t + 1024), device=DEV)[:, None]
                    a = max(0, int(p[0]) - c["window"] + 1) if c["window"] else 0
                    j = torch.cat([torch.arange(min(a, c["sinks"]), device=DEV), torch.arange(a, int(p[-1]) + 1, device=DEV)])
                    near = p - j < c["window"] if c["window"] else j >= 0
                    seen = (near | (j < c["sinks"])) & (j <= p)
                    out[b, t:t + p.shape[0], h] = _exact_attention(s.q[b, h, t:t + p.shape[0]].to(f64), keys[j], vals[j], seen)
        return out
    out = torch.zeros(B, Hq, D, device=DEV, dtype=f64)
    for b, held in enumerate(s.held):
        rows = [j for j in range(held) if not c["window"] or j < c["sinks"] or held - 1 - j < c["window"]]
        rows = torch.tensor(rows, device=DEV)
        for h in range(H):
            keys, vals = [s.kt[b, h, rows].to(f64)], [s.vt[b, h, rows].to(f64)]
            if c["L"]:
                # a rotated Key stands for R k~ + delta_mu in the space of the queries
                m = s.cached[b]
                keys.append(s.Kt[b, h, :m].to(f64) @ s.Rr[b, h].to(f64).T.contiguous() + s.dmu[b, h].to(f64))
                vals.append(s.Vt[b, h, :m].to(f64))
            keys, vals = torch.cat(keys), torch.cat(vals)
            q = s.q[b, h * G:(h + 1) * G].to(f64)
            out[b, h * G:(h + 1) * G] = _exact_attention(q, keys, vals, torch.ones(G, keys.shape[0], dtype=torch.bool, device=DEV))
    return out
