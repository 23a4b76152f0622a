"""Serving operators over a rotated, pruned cache: the 8-bit cache and the attention of drafted tokens.

Five operators on one attention layer, each as a user calls it through the binding and in its plain form:
  write    a prompt's Keys and Values into the 8-bit caches, and these read back   rk_compress_quant, rk_unpack_cache_quant
  append   one token a sequence into the 8-bit caches, and these read back          rk_append_quant, rk_unpack_cache_quant
  decode   one token's attention over the 8-bit caches (and a text segment)         rk_decode_attn_quant
  tree     the attention of a tree of drafted tokens over cache, text and drafts    rk_decode_attn_tree, rk_decode_attn_tree_quant
  commit   the accepted drafts go behind the text segment                           rk_append_text_path

A row x of a head (the rotated Key k R_r, or a Value) is held in 8 bits as whole numbers c = round(x / s), |c| <= 127, and one bfloat16
s for the row: max |x| / 127, rounded up.
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
def _case(name, op, B, Hq, Hkv, L, r, dtype="bf16", **more):
    c = dict(name=name, op=op, B=B, Hq=Hq, Hkv=Hkv, L=L, r=r, dtype=dtype, ragged=False, lists=False, text=0, T=0, q8=op != "tree")
    c.update(more)
    return c


def listed():
    return [
        # the repository's tiny fp32 layer goes into 8 bits: launches and latency
        _case("write_tiny_f32", "write", 1, 2, 2, 512, 32, "f32"),
        # the prompt of the benchmark's layer: batch of 8, 4 KV heads, 16K tokens
        _case("write_16k_gqa", "write", 8, 28, 4, 16384, 64),
        # the first answer tokens of a chat behind a short prompt
        _case("append_chat", "append", 1, 32, 8, 71, 32),
        # a full serving batch, each sequence a token further, all of them at other lengths
        _case("append_batch_mha", "append", 64, 32, 32, 150, 64, ragged=True),
        # a chat turn on a short 8-bit cache of a grouped-query model
        _case("decode_1k_q8", "decode", 1, 32, 8, 1024, 32),
        # a LLaVA-shaped layer in fp32: 2880 image tokens in 8 bits and a 64-token prompt beside them
        _case("decode_llava_q8_f32", "decode", 1, 32, 32, 2880, 64, "f32", text=64),
        # the benchmark's layer with its cache in 8 bits
        _case("decode_16k_q8", "decode", 8, 28, 4, 16384, 64),
        # eight drafted tokens behind a short chat
        _case("tree_chat", "tree", 1, 32, 8, 1024, 32, text=40, T=8),
        # sixteen drafted tokens a sequence on the benchmark's layer, with a prompt of 1024 tokens
        _case("tree_16k_gqa", "tree", 8, 28, 4, 16384, 64, text=1024, T=16),
        # the largest trees, over an 8-bit cache: compute-bound
        _case("tree_64_q8", "tree", 8, 28, 4, 16384, 64, text=300, T=64, q8=True),
        # four accepted tokens of one sequence
        _case("commit_chat", "commit", 1, 32, 8, 0, 32, text=200, T=8),
        # accepted tokens of a full serving batch of a multi-head model
        _case("commit_batch_mha", "commit", 64, 32, 32, 0, 64, text=220, T=24, ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    op = rng.choice(["write", "append", "decode", "decode", "tree", "tree", "tree", "commit"])
    f32 = rng.random() < 0.25
    Hkv = rng.choice([1, 2, 4, 8, 8, 16, 32])
    Hq = Hkv * (rng.choice([1, 2]) if Hkv == 32 else rng.choice([1, 2, 3, 4, 7, 8]))
    B = rng.choice([1, 1, 2, 3, 4, 8, 16])
    r = rng.choice([16, 24, 32, 37, 48, 64, 64, 80, 96, 128])
    L, text, T = 0, 0, 0
    if op in ("write", "decode", "tree"):
        L = _log(rng, 1, 33000)
        while B * Hkv * L > (200_000 if f32 else 520_000):        # (head, token) pairs, under the largest listed case
            if B > 1:
                B = max(1, B // 2)
            else:
                L = L // 2 + rng.randrange(2)
    elif op == "append":
        L = rng.randint(1, 200)
    if op in ("decode", "tree"):
        text = rng.choice([0, _log(rng, 1, 1500)])
    if op == "tree":
        T = _log(rng, 1, 64)
        while B * Hq * T * (L + 2 * text) > (60_000_000 if f32 else 200_000_000):
            T = T // 2 + rng.randrange(2)
    if op == "commit":
        B, T, text = rng.choice([1, 2, 5, 16, 64]), rng.randint(1, 64), rng.randint(64, 400)
    c = _case("", op, B, Hq, Hkv, L, r, "f32" if f32 else "bf16", text=text, T=T, ragged=B > 1 and rng.random() < 0.5)
    if op == "tree":
        c["q8"] = rng.random() < 0.5
    if op == "write" and rng.random() < 0.3:
        c["lists"] = True
    del c["name"]
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


def _kept(n):
    """The rows of a token list: the last 64 and half of the others."""
    return min(n, 64) + max(n - 64, 0) // 2


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


def prepare(case, seed):
    c, s = case, _State()
    s.c = c
    g = torch.Generator(device=DEV)
    g.manual_seed(1_000_003 * seed + 17)
    B, Hq, H, L, r, T, dt = c["B"], c["Hq"], c["Hkv"], c["L"], c["r"], c["T"], _dt(c)

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, device=DEV, generator=g) * std).to(dt)

    s.scale = 1.0 / math.sqrt(D)
    s.Rr = _rotation(g, B, H, r)
    if c["op"] == "write":
        lens = _lens(c, "rows", L)
        s.lens = lens
        mix = torch.randn(B, H, 16, D, device=DEV, generator=g)
        s.K = torch.empty(B, H, L, D, device=DEV, dtype=dt)
        for b in range(B):
            s.K[b] = (torch.matmul(torch.randn(H, L, 16, device=DEV, generator=g), mix[b])
                      + 0.1 * torch.randn(H, L, D, device=DEV, generator=g)).to(dt)
        s.V = normal(B, H, L, D)
        s.n = [_kept(n) for n in lens] if c["lists"] else lens
        s.n_dev = _int32(s.n)
        s.idx = s.off = None
        if c["lists"]:
            rows = [torch.randperm(n, generator=g, device=DEV)[:k].sort().values for n, k in zip(lens, s.n)]
            s.idx = torch.cat(rows).to(torch.int32)
            s.off = torch.tensor([sum(s.n[:i]) for i in range(B + 1)], dtype=torch.int64, device=DEV)
        s.cap = _up(max(s.n))
    elif c["op"] == "append":
        s.cap = _up(L + 1)
        s.len = _int32(_lens(c, "held", L, 0))
        s.Kt, s.Vt = _coded(g, (B, H, s.cap, r), -6, -3, dt), _coded(g, (B, H, s.cap, D), -6, -4, dt)
        held = torch.arange(s.cap, device=DEV)[None, None, :, None] < s.len[:, None, None, None]
        s.Kt, s.Vt = s.Kt * held, s.Vt * held
        s.k_new, s.v_new = normal(B, H, D), normal(B, H, D)
    elif c["op"] in ("decode", "tree"):
        s.cap = _up(L)
        s.len = _int32(_lens(c, "held", L))
        if c["q8"]:
            s.Kt, s.Vt = _coded(g, (B, H, L, r), -6, -3, dt), _coded(g, (B, H, L, D), -6, -4, dt)
        else:
            s.Kt, s.Vt = normal(B, H, L, r, std=1.5), normal(B, H, L, D)
        s.dmu = 0.3 * torch.randn(B, H, D, device=DEV, generator=g)
        s.q = normal(B, max(T, 1), Hq, D)
    if c["op"] != "commit" and c["text"]:
        s.text_len = _int32(_lens(c, "text", c["text"]))
        s.kt, s.vt = normal(B, H, c["text"], D), normal(B, H, c["text"], D)
    if c["op"] == "commit":
        s.text_cap = c["text"] + T
        s.text_len = _int32(_lens(c, "text", c["text"], 0))
        s.kt, s.vt = normal(B, H, s.text_cap, D), normal(B, H, s.text_cap, D)
        s.path = torch.rand(B, T, device=DEV, generator=g).argsort(-1).sort(-1).values.to(torch.int32)
        s.n_path = _int32(_lens(c, "path", max(T // 2, 1)))
        keep = torch.rand(B, T, device=DEV, generator=g).argsort(-1)     # each path: n rows of the drafts in rising order
        s.path = torch.where(torch.arange(T, device=DEV)[None] < s.n_path[:, None], keep, T + keep).sort(-1).values
        s.path = torch.where(s.path < T, s.path, 0).to(torch.int32)
    if T:
        s.kd, s.vd = normal(B, H, T, D), normal(B, H, T, D)
        s.n_drafts = _int32(_lens(c, "drafts", T))
        parent = [[-1] + [random.Random("%d %d %d" % (seed, b, i)).randint(max(0, i - 6), i - 1) for i in range(1, T)] for b in range(B)]
        bits = []
        for b in range(B):
            seen = []
            for i, p in enumerate(parent[b]):
                seen.append((seen[p] if p >= 0 else 0) | 1 << i)
            bits.append([x - (1 << 64) if x >> 63 else x for x in seen])
        s.bits = torch.tensor(bits, dtype=torch.int64, device=DEV)
    if own:
        _hold(s)
    return s


def _hold(s):
    """What a program that uses the framework has at hand: the caches as the framework holds them, outputs and workspace."""
    rk, c = _rk(), s.c
    ctx = _context()
    B, Hq, H, L, r, T, dt = c["B"], c["Hq"], c["Hkv"], c["L"], c["r"], c["T"], _dt(c)
    kind = rk.RK_F32 if c["dtype"] == "f32" else rk.RK_BF16
    s.ctx = ctx
    s.lay = rk.Layout(B, Hq, H, r, kind, getattr(s, "cap", 32), L if c["op"] != "write" else 0, seq_len=getattr(s, "len", None))
    if c["op"] != "commit":
        kb, vb = rk.rk_cache_bytes_quant(s.lay) if c["q8"] else rk.rk_cache_bytes(s.lay)
        s.kc = torch.zeros(kb, dtype=torch.uint8, device=DEV)
        s.vc = torch.zeros(vb, dtype=torch.uint8, device=DEV)
    if c["op"] in ("append", "decode", "tree"):
        # rows that are exact in the cache's form, through the columns of the identity
        pick = torch.eye(D, device=DEV)[:, :r].expand(B, H, D, r).contiguous()
        wide = torch.zeros(B, H, s.Kt.shape[2], D, device=DEV, dtype=dt)
        wide[..., :r] = s.Kt
        n = L if c["op"] == "append" else s.Kt.shape[2]
        keys, values = rk.Rows(wide, n, n_tokens_dev=s.len), rk.Rows(s.Vt, n, n_tokens_dev=s.len)
        put = rk.rk_compress_quant if c["q8"] else rk.rk_compress
        put(ctx, s.lay, keys, pick, s.kc, values=values, v_cache=s.vc)
        torch.cuda.synchronize()
    if c["op"] in ("write", "append"):
        s.len_out = torch.zeros(B, dtype=torch.int32, device=DEV)
        s.k_rows = torch.zeros(B, H, s.cap, r, device=DEV, dtype=dt)
        s.v_rows = torch.zeros(B, H, s.cap, D, device=DEV, dtype=dt)
    if c["op"] == "write":
        s.keys = rk.Rows(s.K, max(s.n), n_tokens_dev=None if c["lists"] else s.n_dev, tok_idx=s.idx, tok_off=s.off)
        s.values = rk.Rows(s.V, max(s.n), n_tokens_dev=None if c["lists"] else s.n_dev, tok_idx=s.idx, tok_off=s.off)
    if c["op"] in ("write", "append"):
        s.held = rk.Layout(B, Hq, H, r, kind, s.cap, 0, seq_len=s.len_out)
    s.text = None
    if c["text"]:
        s.text = rk.Text(s.kt, s.vt, c["text"], len=s.text_len)
    if T:
        s.drafts = rk.Drafts(s.kd, s.vd, T, mask=s.bits, n_tokens_dev=s.n_drafts if c["op"] == "tree" else None)
    if c["op"] in ("decode", "tree"):
        s.out = torch.zeros(B, max(T, 1), Hq, D, device=DEV, dtype=dt)
        s.ws = torch.empty(rk.rk_tree_workspace_size(ctx, s.lay, max(T, 1)), dtype=torch.uint8, device=DEV)
    if c["op"] == "commit":
        s.len_out = torch.zeros(B, dtype=torch.int32, device=DEV)


# ---- one pass -----------------------------------------------------------------------------------------------
def run(s):
    return {"write": _write, "append": _append, "decode": _attend, "tree": _attend, "commit": _commit}[s.c["op"]](s)


def _read_back(s):
    """Values that are held in 8 bits, as bfloat16."""
    if own:
        _rk().rk_unpack_cache_quant(s.ctx, s.held, s.kc, s.vc, s.k_rows, s.v_rows)
        return s.k_rows.to(torch.bfloat16), s.v_rows.to(torch.bfloat16)


def _in_8_bits(x):
    """x row by row in 8 bits, and back."""
    step = x.abs().amax(-1, keepdim=True) / 127
    step = ((step.view(torch.int32) + 0xFFFF) & ~0xFFFF).view(torch.float32)
    return torch.where(step > 0, torch.round(x / step).clamp(-127, 127) * step, torch.zeros_like(x))


def _write(s):
    c = s.c
    if own:
        _rk().rk_compress_quant(s.ctx, s.lay, s.keys, s.Rr, s.kc, values=s.values, v_cache=s.vc, seq_len_out=s.len_out)
        k, v = _read_back(s)
        return k, v, s.len_out
    K, V = s.K.float(), s.V.float()
    B, H, r, cap = c["B"], c["Hkv"], c["r"], s.cap
    t = torch.arange(cap, device=DEV)
    at = t[None].expand(B, cap)
    if c["lists"]:
        at = s.idx[(s.off[:-1, None] + t[None]).clamp(max=s.idx.numel() - 1)]
    at = at.clamp(max=c["L"] - 1).to(torch.int64)[:, None, :, None].expand(B, H, cap, D)
    there = (t[None] < s.n_dev[:, None])[:, None, :, None]
    K, V = torch.gather(K, 2, at), torch.gather(V, 2, at)
    k, v = _in_8_bits(torch.matmul(K, s.Rr)), _in_8_bits(V)
    return torch.where(there, k, 0).to(torch.bfloat16), torch.where(there, v, 0).to(torch.bfloat16), s.n_dev.clone()


def _append(s):
    if own:
        _rk().rk_append_quant(s.ctx, s.lay, s.k_new, s.v_new, s.Rr, s.kc, s.vc, s.len_out)
        k, v = _read_back(s)
        return k, v, s.len_out
    k = _in_8_bits(torch.matmul(s.k_new.float()[:, :, None], s.Rr))
    v = _in_8_bits(s.v_new.float()[:, :, None])
    here = (torch.arange(s.cap, device=DEV)[None] == s.len[:, None])[:, None, :, None]
    return torch.where(here, k, s.Kt.float()).to(torch.bfloat16), torch.where(here, v, s.Vt.float()).to(torch.bfloat16), s.len + 1


def _attend(s):
    c = s.c
    if own:
        rk = _rk()
        if c["op"] == "decode":
            rk.rk_decode_attn_quant(s.ctx, s.lay, s.q, s.kc, s.vc, s.Rr, s.dmu, s.text, s.scale, s.out, s.ws)
        else:
            call = rk.rk_decode_attn_tree_quant if c["q8"] else rk.rk_decode_attn_tree
            call(s.ctx, s.lay, s.q, s.kc, s.vc, s.Rr, s.dmu, s.text, s.drafts, s.scale, s.out, s.ws)
        return s.out
    B, T, Hq, _ = s.q.shape
    H, G = c["Hkv"], c["Hq"] // c["Hkv"]
    q = s.q.float().view(B, T, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, T * G, D)      # rows of a KV head: token, head
    low = float("-inf")
    cached = torch.arange(c["L"], device=DEV)[None] < s.len[:, None]
    x = torch.matmul(torch.matmul(q, s.Rr), s.Kt.float().transpose(2, 3).contiguous()) + torch.matmul(q, s.dmu[..., None])
    parts, values = [x.masked_fill_(~cached[:, None, None, :], low)], [s.Vt]
    if c["text"]:
        there = torch.arange(c["text"], device=DEV)[None] < s.text_len[:, None]
        x = torch.matmul(q, s.kt.float().transpose(2, 3).contiguous())
        parts.append(x.masked_fill_(~there[:, None, None, :], low))
        values.append(s.vt)
    if c["T"]:
        j = torch.arange(T, device=DEV)
        seen = ((s.bits[:, :, None] >> j) & 1).bool() & (j < s.n_drafts[:, None])[:, None]
        seen = seen[:, None, :, None, :].expand(B, H, T, G, T).reshape(B, H, T * G, T)
        x = torch.matmul(q, s.kd.float().transpose(2, 3).contiguous())
        parts.append(x.masked_fill_(~seen, low))
        values.append(s.vd)
    most = torch.stack([p.amax(-1, keepdim=True) for p in parts]).amax(0).clamp(min=-3e38)
    parts = [torch.exp((p - most).mul_(s.scale)) for p in parts]
    total = sum(p.sum(-1, keepdim=True) for p in parts)
    out = sum(torch.matmul(p, v.float()) for p, v in zip(parts, values))
    out = torch.where(total > 0, out / total, 0)
    out = out.view(B, H, T, G, D).permute(0, 2, 1, 3, 4).reshape(B, T, Hq, D)
    if c["T"]:
        out = torch.where((torch.arange(T, device=DEV)[None] < s.n_drafts[:, None])[:, :, None, None], out, 0)
    return out.to(_dt(c))


def _commit(s):
    c = s.c
    if own:
        _rk().rk_append_text_path(s.ctx, s.lay, s.text, s.drafts, s.path, s.n_path, s.len_out)
        return s.kt, s.vt, s.len_out
    B, H, T = c["B"], c["Hkv"], c["T"]
    j = torch.arange(s.text_cap, device=DEV)[None] - s.text_len[:, None]
    here = ((j >= 0) & (j < s.n_path[:, None]))[:, None, :, None]
    at = torch.gather(s.path.to(torch.int64), 1, j.clamp(0, T - 1).to(torch.int64))[:, None, :, None].expand(B, H, s.text_cap, D)
    return torch.where(here, torch.gather(s.kd, 2, at), s.kt), torch.where(here, torch.gather(s.vd, 2, at), s.vt), s.text_len + s.n_path


# ---- what a pass cannot do without ---------------------------------------------------------------------------
def work(case):
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    H, Hq, r, T, B = c["Hkv"], c["Hq"], c["r"], c["T"], c["B"]
    held = r + D + 4                                      # a token and head in 8 bits
    if c["op"] == "write":
        n = sum(_kept(x) if c["lists"] else x for x in _lens(c, "rows", c["L"]))
        return {"bytes": H * n * (2 * D * e + 2 * held + (r + D) * e) + B * H * D * r * 4, "flops": 2 * H * n * D * r}
    if c["op"] == "append":
        n = sum(x + 1 for x in _lens(c, "held", c["L"], 0))
        return {"bytes": B * H * (2 * D * e + held + D * r * 4) + H * n * (held + (r + D) * e), "flops": 2 * H * B * D * r}
    if c["op"] == "commit":
        n = sum(_lens(c, "path", max(T // 2, 1)))
        return {"bytes": 4 * H * n * D * e, "flops": 0}
    cached, text, rows = _lens(c, "held", c["L"]), _lens(c, "text", c["text"]), _lens(c, "drafts", T) if T else [1] * B
    each = held if c["q8"] else (r + D) * e
    size = B * H * D * (r + 1) * 4
    flops = 0
    for n, m, t in zip(cached, text, rows):
        size += H * (n * each + 2 * (m + (t if T else 0)) * D * e) + 2 * t * Hq * D * e
        flops += 2 * t * Hq * (n * (r + D) + 2 * D * (m + (t if T else 0)) + D * r)
    return {"bytes": size, "flops": flops}


# ---- the definition in 64 bits --------------------------------------------------------------------------------
def _exact_8_bits(row):
    """[..., n] of float64 -> what its 8 bits stand for, from the definition."""
    top = row.abs().max(dim=-1, keepdim=True).values
    m, e = torch.frexp(top / 127)
    step = torch.ldexp(torch.ceil(torch.ldexp(m, torch.tensor(8))), e - 8)           # eight binary digits, upwards
    codes = torch.where(step > 0, row / torch.where(step > 0, step, 1), 0)
    return torch.round(codes) * step


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    B, H, G, r, f64 = c["B"], c["Hkv"], c["Hq"] // c["Hkv"], c["r"], torch.float64
    if c["op"] == "write":
        k = torch.zeros(B, H, s.cap, r, device=DEV, dtype=f64)
        v = torch.zeros(B, H, s.cap, D, device=DEV, dtype=f64)
        for b in range(B):
            n = s.n[b]
            rows = s.idx[s.off[b]:s.off[b + 1]].long() if c["lists"] else torch.arange(n, device=DEV)
            for h in range(H):
                k[b, h, :n] = _exact_8_bits(s.K[b, h, rows].to(f64) @ s.Rr[b, h].to(f64))
                v[b, h, :n] = _exact_8_bits(s.V[b, h, rows].to(f64))
        return k, v, torch.tensor(s.n, dtype=torch.int32, device=DEV)
    if c["op"] == "append":
        k, v = s.Kt.to(f64), s.Vt.to(f64)
        for b, n in enumerate(s.len.tolist()):
            for h in range(H):
                k[b, h, n] = _exact_8_bits(s.k_new[b, h].to(f64) @ s.Rr[b, h].to(f64))
                v[b, h, n] = _exact_8_bits(s.v_new[b, h].to(f64))
        return k, v, s.len + 1
    if c["op"] == "commit":
        k, v, n = s.kt.to(f64), s.vt.to(f64), s.text_len.clone()
        for b, (at, m) in enumerate(zip(s.text_len.tolist(), s.n_path.tolist())):
            for j, row in enumerate(s.path[b, :m].tolist()):
                k[b, :, at + j], v[b, :, at + j] = s.kd[b, :, row].to(f64), s.vd[b, :, row].to(f64)
            n[b] += m
        return k, v, n
    T = max(c["T"], 1)
    out = torch.zeros(B, T, c["Hq"], D, device=DEV, dtype=f64)
    for b in range(B):
        n, m = int(s.len[b]), int(s.text_len[b]) if c["text"] else 0
        t = int(s.n_drafts[b]) if c["T"] else 1
        for h in range(H):
            R = s.Rr[b, h].to(f64)
            # a rotated Key stands for R k~ + delta_mu in the space of the queries
            keys = [s.Kt[b, h, :n].to(f64) @ R.T.contiguous() + s.dmu[b, h].to(f64)]
            vals = [s.Vt[b, h, :n].to(f64)]
            if m:
                keys.append(s.kt[b, h, :m].to(f64))
                vals.append(s.vt[b, h, :m].to(f64))
            if c["T"]:
                keys.append(s.kd[b, h, :t].to(f64))
                vals.append(s.vd[b, h, :t].to(f64))
            keys, vals = torch.cat(keys), torch.cat(vals)
            hide = torch.zeros(t, keys.shape[0], dtype=torch.bool, device=DEV)
            if c["T"]:
                for i, word in enumerate(s.bits[b, :t].tolist()):
                    hide[i, n + m:] = torch.tensor([not word >> j & 1 for j in range(t)], device=DEV)
            q = s.q[b, :t, h * G:(h + 1) * G].to(f64).reshape(t * G, D)
            w = (q @ keys.T.contiguous() / math.sqrt(D)).view(t, G, -1).masked_fill(hide[:, None], -math.inf)
            out[b, :t, h * G:(h + 1) * G] = (torch.softmax(w, -1).view(t * G, -1) @ vals).view(t, G, D)
    return out
