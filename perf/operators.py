"""The measured cases of the serving operators around the adapter projections: block tables from request
lengths, per-head norm and rotation of queries and keys, the 4-bit cache write, and attention over
that cache, each in its plain form (elementary torch operations in 32 bits) and through the library.

Sizes follow the repository's workloads: 32 query heads and 8 key/value heads of 128 (the fused QKV
projection 4096 -> 6144), 16 / 256 / 512 decode tokens, prompt chunks of 512, 32 prompts of 32..2048
tokens.  Cache format: cells of 16 tokens of one head, [16 x D/2 K codes][16 x D/2 V codes][16 x
(scale, low) of K][16 x (scale, low) of V], cells of a page's head consecutive, heads inside a page.
"""
import math
import random

import torch

own = False

CELL = 16


# ------------------------------------------------------------------------------------------
# cases
# ------------------------------------------------------------------------------------------
def _case(name, op, **kw):
    c = {"name": name, "op": op, "hq": 32, "hkv": 8, "d": 128, "page": 16, "window": 0, "lens": 1,
         "decode": 0, "q_dec": 1, "ctx_lo": 1, "ctx_hi": 1, "prompts": 0, "q_lo": 0, "q_hi": 0,
         "pre_lo": 0, "pre_hi": 0}
    c.update(kw)
    return c


def listed():
    return [
        # one decode step of a busy server: every request one token, contexts of all lengths
        _case("tables_decode", "tables", decode=256, ctx_lo=1, ctx_hi=8192),
        # a chunked-prefill step: 512 decode tokens beside four prompt chunks
        _case("tables_mixed", "tables", decode=512, ctx_lo=1, ctx_hi=4096, prompts=4, q_lo=512, q_hi=512,
              pre_hi=4096),
        # the smallest decode batch: the time is launch latency
        _case("norm_rope_decode", "norm_rope", decode=16, ctx_lo=1, ctx_hi=2048),
        # a prefill step of 32 prompts: the time is memory traffic
        _case("norm_rope_prompts", "norm_rope", prompts=32, q_lo=32, q_hi=2048),
        # cache write of one decode step
        _case("append_decode", "append", decode=256, ctx_lo=1, ctx_hi=2048),
        # cache write of 32 prompts on pages of 64 tokens
        _case("append_prompts", "append", prompts=32, q_lo=32, q_hi=2048, page=64),
        # a handful of requests, seven query heads per key/value head, heads of 64, a sliding window
        _case("attn_decode_few", "attention", decode=16, ctx_lo=1, ctx_hi=2048, hq=28, hkv=4, d=64, page=32,
              window=1000),
        # the ordinary decode step of a busy server
        _case("attn_decode", "attention", decode=256, ctx_lo=256, ctx_hi=8192),
        # few requests with very long contexts: the work has to be split along the keys
        _case("attn_decode_long", "attention", decode=4, ctx_lo=60000, ctx_hi=131000),
        # a chunked-prefill step: decode tokens and prompt chunks in one call
        _case("attn_mixed", "attention", decode=512, ctx_lo=16, ctx_hi=4096, prompts=4, q_lo=512, q_hi=512,
              pre_hi=4096),
        # a prefill step of 32 fresh prompts
        _case("attn_prompts", "attention", prompts=32, q_lo=32, q_hi=2048),
        # one chunk of a long document on top of its cached part
        _case("attn_chunk", "attention", prompts=1, q_lo=2048, q_hi=2048, pre_lo=30001, pre_hi=30001, page=64),
    ]


def _log_uniform(rng, lo, hi):
    if hi <= lo:
        return lo
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(max(lo, 1)), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["tables", "norm_rope", "append", "attention", "attention", "attention"])
    d = rng.choice([64, 128])
    hkv = rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 2, 3, 4, 5, 7, 8, 16] if hkv < 8 else [1, 2, 4])
    page = rng.choice([16, 32, 64, 128])
    kw = dict(hq=hkv * group, hkv=hkv, d=d, page=page, lens=rng.randrange(1 << 20))
    kind = rng.choice(["decode", "prompts", "mixed"])
    if kind != "prompts":
        kw.update(decode=_log_uniform(rng, 1, 512), ctx_lo=rng.choice([0, 1, 100]),
                  ctx_hi=_log_uniform(rng, 128, 4096))
        if op == "attention":
            kw.update(q_dec=rng.choice([1, 1, 1, 2, 5]))
            if kw["decode"] <= 8:
                kw.update(ctx_hi=_log_uniform(rng, 4096, 100000))
    if kind == "prompts":
        kw.update(prompts=_log_uniform(rng, 1, 24), q_lo=_log_uniform(rng, 1, 64), q_hi=_log_uniform(rng, 65, 2000))
    if kind == "mixed":
        kw.update(prompts=rng.randint(1, 4), q_lo=33, q_hi=_log_uniform(rng, 64, 700), pre_hi=rng.choice([0, 1500, 4000]))
    if op == "attention" and rng.random() < 0.3:
        kw.update(window=_log_uniform(rng, 16, 2048))
    c = _case("", op, **kw)
    del c["name"]
    # no dearer than the largest listed case, in products and in the plain form's padded scores
    while op == "attention" and (work(c)["flops"] > 5e11 or _padded(c) > 2e9):
        c["prompts"], c["decode"] = -(-c["prompts"] // 2), -(-c["decode"] // 2)
        c["q_hi"], c["ctx_hi"] = max(c["q_lo"], c["q_hi"] // 2), max(c["ctx_lo"], c["ctx_hi"] // 2)
    return c


def _padded(case):
    lens, n = _lengths(case), case["decode"]
    return max(len(g) * case["hq"] * max(q for _, q in g) * max(kv + q for kv, q in g)
               for g in (lens[:n], lens[n:]) if g)


def _lengths(case):
    """[(keys already cached, new tokens)] of the batch: decode requests first, then prompts."""
    rng = random.Random(case["lens"])
    out = [(_log_uniform(rng, case["ctx_lo"], case["ctx_hi"]), case["q_dec"]) for _ in range(case["decode"])]
    out += [(_log_uniform(rng, case["pre_lo"], case["pre_hi"]), _log_uniform(rng, case["q_lo"], case["q_hi"]))
            for _ in range(case["prompts"])]
    return out


def _pairs(kv, q, window):
    """(visible (query, key) pairs of one head, keys that any of the queries sees) of one request."""
    if not window:
        return q * kv + q * (q + 1) // 2, kv + q
    return sum(min(kv + i + 1, window) for i in range(q)), min(kv + q, window + q - 1)


def work(case):
    hq, hkv, d, P = case["hq"], case["hkv"], case["d"], case["page"]
    lens = _lengths(case)
    R, T = len(lens), sum(q for _, q in lens)
    new_pages = sum(-(-(kv + q) // P) - -(-kv // P) for kv, q in lens)
    row = d + 8                     # one key's K and V codes with their scales and lows, one head
    if case["op"] == "tables":      # lengths and tables in; starts, lengths, positions, slots, pages out
        return {"bytes": 4 * (3 * R + 2 * new_pages) + 4 * (2 * R + 2 * T), "flops": 0}
    if case["op"] == "norm_rope":   # q and k in and out, positions, the rows of the angle table
        return {"bytes": 4 * T * (hq + hkv) * d + 4 * T + 4 * T * d, "flops": 8 * T * (hq + hkv) * d}
    if case["op"] == "append":      # q, k, v in; q and the cache rows out; the rows back in and out as bf16
        return {"bytes": 4 * T * hq * d + 4 * T * hkv * d + 2 * T * hkv * row + 4 * T * hkv * d + 8 * T + 4 * T * d,
                "flops": 8 * T * (hq + 3 * hkv) * d}
    pairs, keys = (sum(v) for v in zip(*(_pairs(kv, q, case["window"]) for kv, q in lens)))
    return {"bytes": 4 * T * hq * d + keys * hkv * row, "flops": 4 * d * hq * pairs}


# ------------------------------------------------------------------------------------------
# the cache format in plain operations
# ------------------------------------------------------------------------------------------
#: nibble n of a 32-bit word holds element NIBBLE[n] of its eight
NIBBLE = (0, 2, 4, 6, 1, 3, 5, 7)


def _quantise(x):
    """float32 [..., D] -> codes (float32, whole numbers 0..15), scale and low (bfloat16 [...])."""
    low = x.amin(-1).bfloat16()
    scale = ((x.amax(-1) - low.float()) / 15.0).bfloat16()
    scale = torch.where(scale.float() < 1.17549435e-38, torch.zeros_like(scale), scale)
    bad = ~(torch.isfinite(scale) & torch.isfinite(low))
    scale, low = scale.masked_fill(bad, math.nan), low.masked_fill(bad, math.nan)
    inv = torch.where(scale == 0, torch.zeros_like(scale, dtype=torch.float32), 1.0 / scale.float())
    codes = torch.round((x - low.float()[..., None]) * inv[..., None]).clamp(0.0, 15.0)
    return codes.masked_fill(bad[..., None], 0.0), scale, low


def _pack(codes):
    """codes [..., D] -> uint8 [..., D/2]"""
    n = codes.to(torch.uint8).unflatten(-1, (-1, 8))[..., list(NIBBLE)]
    return (n[..., 0::2] | (n[..., 1::2] << 4)).flatten(-2)


def _unpack(b):
    """uint8 [..., D/2] -> codes [..., D] in float32"""
    n = torch.stack([b & 15, b >> 4], -1).unflatten(-2, (-1, 4)).flatten(-2)     # [..., D/8, 8] in nibble order
    return n[..., [NIBBLE.index(i) for i in range(8)]].flatten(-2).float()


def _params(scale, low):
    """bfloat16 [...] twice -> uint8 [..., 4]"""
    return torch.stack([scale, low], -1).view(torch.uint8)


def _cell_bytes(case):
    return CELL * (case["d"] + 8)


def _cells(case, buf):
    """The cache of one layer as [pages * cells of a page, heads, bytes of a cell] (a view)."""
    hkv, P = case["hkv"], case["page"]
    return buf.view(-1, hkv, P // CELL, _cell_bytes(case))


def _gather_values(case, cells):
    """cells uint8 [..., bytes of a cell] -> K, V float32 [..., 16, D]"""
    d = case["d"]
    n = CELL * d // 2
    k, v = cells[..., :n].unflatten(-1, (CELL, d // 2)), cells[..., n:2 * n].unflatten(-1, (CELL, d // 2))
    p = cells[..., 2 * n:].contiguous().view(torch.bfloat16).float().unflatten(-1, (2, CELL, 2))
    return (_unpack(k) * p[..., 0, :, 0:1] + p[..., 0, :, 1:2],
            _unpack(v) * p[..., 1, :, 0:1] + p[..., 1, :, 1:2])


# ------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------
def _angles(case, positions):
    d = case["d"]
    f = 500000.0 ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float32) / d)
    a = torch.arange(positions, device="cuda", dtype=torch.float32)[:, None] * f
    return torch.cat([a.cos(), a.sin()], -1).contiguous()


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    hq, hkv, d, P = case["hq"], case["hkv"], case["d"], case["page"]
    lens = _lengths(case)
    R, T = len(lens), sum(q for _, q in lens)
    i32 = dict(dtype=torch.int32, device=dev)
    kv_len, q_len = torch.tensor([kv for kv, _ in lens], **i32), torch.tensor([q for _, q in lens], **i32)
    before = [-(-kv // P) for kv, _ in lens]
    after = [-(-(kv + q) // P) for kv, q in lens]
    cap = max(after) + 1
    pages = sum(after) + 7
    order = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
    # pages already taken, request after request; the rest is the free stack
    table = torch.full((R, cap), -1, **i32)
    held = torch.arange(cap, device=dev)[None] < torch.tensor(before, device=dev)[:, None]
    table[held] = order[: sum(before)]
    free = torch.zeros(pages, **i32)
    free[: pages - sum(before)] = order[sum(before):]
    s = {"case": case, "lens": lens, "R": R, "T": T, "kv_len": kv_len, "q_len": q_len, "table": table,
         "free": free, "free_count": torch.tensor([pages - sum(before)], **i32), "pages": pages, "cap": cap,
         "max_q": max(q for _, q in lens), "max_pos": max(kv + q for kv, q in lens)}
    op = case["op"]
    # the fused projection's output: one row a token, query heads, then key heads, then value heads
    if op in ("norm_rope", "append"):
        s["qkv"] = torch.randn(T, (hq + 2 * hkv) * d, generator=g, device=dev).mul_(
            torch.rand((hq + 2 * hkv) * d, generator=g, device=dev) + 0.5).bfloat16()
        s["qw"] = (1 + 0.3 * torch.randn(d, generator=g, device=dev)).bfloat16()
        s["kw"] = (1 + 0.3 * torch.randn(d, generator=g, device=dev)).bfloat16()
        s["angles"] = _angles(case, s["max_pos"])
        s["positions"] = torch.cat([torch.arange(kv, kv + q, **i32) for kv, q in lens])
        s["q_out"] = torch.empty(T, hq * d, dtype=torch.bfloat16, device=dev)
        s["k_out"] = torch.empty(T, hkv * d, dtype=torch.bfloat16, device=dev)
        s["v_out"] = torch.empty(T, hkv * d, dtype=torch.bfloat16, device=dev)
    if op in ("append", "attention"):
        # memory that was never written: every scale and low is no number
        s["cache"] = torch.full((pages * hkv * (P // CELL) * _cell_bytes(case),), 255, dtype=torch.uint8, device=dev)
        taken = sum(after) - sum(before)
        new = torch.arange(cap, device=dev)[None] < torch.tensor(after, device=dev)[:, None]
        s["full_table"] = table.clone()
        s["full_table"][new & ~held] = free[: pages - sum(before)].flip(0)[:taken]
        s["slots"] = torch.cat([s["full_table"][r, torch.arange(kv, kv + q, device=dev) // P] * P
                                + torch.arange(kv, kv + q, **i32) % P for r, (kv, q) in enumerate(lens)])
    if op == "attention":
        s["scale"] = d ** -0.5
        # queries whose logits spread as a trained model's do; keys with unequal channels, values
        # with tokens of unequal size
        s["q"] = (torch.randn(T, hq * d, generator=g, device=dev) * 1.7).bfloat16()
        s["out"] = torch.empty_like(s["q"])
        gain = torch.exp(0.4 * torch.randn(hkv, d, generator=g, device=dev))
        cells = _cells(case, s["cache"])
        used = s["full_table"][s["full_table"] >= 0].long()
        step = max(1, (1 << 26) // (hkv * P * d))
        n = CELL * d // 2
        for a in range(0, used.numel(), step):
            at = used[a:a + step]
            shape = (at.numel(), hkv, P // CELL, CELL, d)
            kc, ks, kl = _quantise(torch.randn(shape, generator=g, device=dev) * gain[:, None, None])
            size = torch.exp(0.5 * torch.randn(shape[:-1], generator=g, device=dev))
            vc, vs, vl = _quantise(torch.randn(shape, generator=g, device=dev) * size[..., None])
            cells[at] = torch.cat([_pack(kc).flatten(-2), _pack(vc).flatten(-2),
                                   _params(ks, kl).flatten(-2), _params(vs, vl).flatten(-2)], -1)
            assert cells.shape[-1] == 2 * n + 8 * CELL
        # the last page of a request ends inside: what lies behind its tokens was never written
        for r, (kv, q) in enumerate(lens):
            end = kv + q
            if end % P:
                page = s["full_table"][r, end // P]
                tail = cells[page, :, (end % P) // CELL:]
                lo = (end % P) % CELL
                par = tail[:, 0, 2 * n:].view(hkv, 2, CELL, 4)
                par[:, :, lo:] = 255
                tail[:, 1:] = 255
        # decode requests and prompts are laid out apart: padding one to the other's length would be waste
        s["groups"] = [_group(s, 0, case["decode"]), _group(s, case["decode"], R)]
    if own:
        _attach(s)
    return s


def _group(s, r0, r1):
    """What the plain form needs of requests r0 .. r1 - 1, padded to the longest of them."""
    case, lens = s["case"], s["lens"]
    if r0 == r1:
        return None
    dev = "cuda"
    first = sum(q for _, q in lens[:r0])
    q_max, k_max = max(q for _, q in lens[r0:r1]), max(kv + q for kv, q in lens[r0:r1])
    q_len = torch.tensor([q for _, q in lens[r0:r1]], device=dev)
    kv = torch.tensor([kv for kv, _ in lens[r0:r1]], device=dev)
    start = first + torch.cumsum(q_len, 0) - q_len
    i = torch.arange(q_max, device=dev)
    return {"r0": r0, "r1": r1, "valid": i[None] < q_len[:, None], "token": (start[:, None] + i).clamp(max=s["T"] - 1),
            "limit": kv[:, None] + i + 1, "end": (kv + q_len)[:, None], "blocks": -(-k_max // case["page"])}


# ------------------------------------------------------------------------------------------
# plain forms
# ------------------------------------------------------------------------------------------
def _pair_sum(x):
    """The sum over the last dimension, neighbours first (its order is part of the operator)."""
    return x[..., 0] if x.shape[-1] == 1 else _pair_sum(x[..., 0::2] + x[..., 1::2])


def _norm_rotate(x, w, angles, eps):
    """float32 [T, heads, D]"""
    h = x.shape[-1] // 2
    sq = x * x
    ms = _pair_sum(sq[..., :h] + sq[..., h:]) / x.shape[-1]
    y = x * (1.0 / torch.sqrt(ms + eps))[..., None] * w
    a, b = y[..., :h], y[..., h:]
    c, s = angles[:, None, :h], angles[:, None, h:]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def _plain_qk(s):
    c = s["case"]
    T, hq, hkv, d = s["T"], c["hq"], c["hkv"], c["d"]
    x = s["qkv"].float().view(T, hq + 2 * hkv, d)
    at = s["angles"][s["positions"].long()]
    q = _norm_rotate(x[:, :hq], s["qw"].float(), at, 1e-6)
    k = _norm_rotate(x[:, hq:hq + hkv], s["kw"].float(), at, 1e-6)
    return q, k, x[:, hq + hkv:]


def _plain_norm_rope(s):
    q, k, _ = _plain_qk(s)
    return {"q": q.bfloat16().flatten(1), "k": k.bfloat16().flatten(1)}


def _plain_append(s):
    c = s["case"]
    d, P = c["d"], c["page"]
    n = CELL * d // 2
    q, k, v = _plain_qk(s)
    cells = _cells(c, s["cache"])
    slots = s["slots"].long()
    page, cell, row = slots // P, slots % P // CELL, slots % CELL
    (kc, ks, kl), (vc, vs, vl) = _quantise(k), _quantise(v)
    heads = torch.arange(c["hkv"], device="cuda")
    at = (page[:, None], heads[None], cell[:, None], row[:, None])
    codes = cells[..., :2 * n].unflatten(-1, (2, CELL, d // 2))
    params = cells[..., 2 * n:].unflatten(-1, (2, CELL, 4))
    codes[at[:3] + (0,) + at[3:]], codes[at[:3] + (1,) + at[3:]] = _pack(kc), _pack(vc)
    params[at[:3] + (0,) + at[3:]], params[at[:3] + (1,) + at[3:]] = _params(ks, kl), _params(vs, vl)
    # the written rows as the values they stand for
    kb, vb = codes[at[:3] + (0,) + at[3:]], codes[at[:3] + (1,) + at[3:]]
    kp = params[at[:3] + (0,) + at[3:]].view(torch.bfloat16).float()
    vp = params[at[:3] + (1,) + at[3:]].view(torch.bfloat16).float()
    return {"q": q.bfloat16().flatten(1), "k": (_unpack(kb) * kp[..., 0:1] + kp[..., 1:2]).bfloat16().flatten(1),
            "v": (_unpack(vb) * vp[..., 0:1] + vp[..., 1:2]).bfloat16().flatten(1)}


def _plain_attention_group(s, g, out):
    c = s["case"]
    hq, hkv, d, P = c["hq"], c["hkv"], c["d"], c["page"]
    n = g["r1"] - g["r0"]
    table = s["full_table"][g["r0"]:g["r1"], :g["blocks"]].long().clamp(min=0)
    cells = _cells(c, s["cache"])[table]                                     # [n, blocks, hkv, cells, bytes]
    k, v = _gather_values(c, cells)
    k = k.permute(0, 2, 1, 3, 4, 5).reshape(n, hkv, -1, d)
    v = v.permute(0, 2, 1, 3, 4, 5).reshape(n, hkv, -1, d)
    q = s["q"][g["token"]].float().view(n, -1, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(n, hkv, -1, d)
    t = torch.arange(k.shape[2], device="cuda")
    seen = t < g["limit"][..., None]
    if c["window"]:
        seen &= t >= g["limit"][..., None] - c["window"]
    seen = seen[:, None, None]                                               # [n, 1, 1, queries, keys]
    some = (t < g["end"])[:, None, :, None]                                  # what is behind was never written
    x = torch.matmul(q, k.transpose(-1, -2)).mul_(s["scale"]).unflatten(2, (hq // hkv, -1))
    x = x.masked_fill_(~seen, -math.inf)
    x = x.sub_(x.amax(-1, keepdim=True)).exp_()
    total = x.sum(-1)
    o = torch.matmul(x.flatten(2, 3), v.masked_fill_(~some, 0.0)).unflatten(2, (hq // hkv, -1)) / total[..., None]
    o = o.permute(0, 3, 1, 2, 4).reshape(n, -1, hq * d).bfloat16()
    out[g["token"][g["valid"]]] = o[g["valid"]]


def _plain_attention(s):
    out = torch.empty_like(s["q"])
    if s["groups"][0]:
        _plain_attention_group(s, s["groups"][0], out)
    if s["groups"][1]:
        _plain_attention_group(s, s["groups"][1], out)
    return {"out": out}


def _plain_tables(s):
    P, R, T = s["case"]["page"], s["R"], s["T"]
    kv, q, table, count = s["kv_len"].long(), s["q_len"].long(), s["table"], s["free_count"].long()
    end = torch.cumsum(q, 0)
    start = end - q
    have, want = (kv + P - 1) // P, (kv + q + P - 1) // P
    fits = (want <= s["cap"]) & (end <= T)
    need = torch.where(fits, want - have, 0)
    upto = torch.cumsum(need, 0)
    ok = fits & ((upto <= count) | (need == 0))
    taken = torch.where(ok, upto, 0).amax().clamp(min=0)
    # the new pages, in request order, from the top of the stack
    col = torch.arange(s["cap"], device="cuda")[None]
    new = (col >= have[:, None]) & (col < want[:, None]) & ok[:, None]
    k = (upto - need)[:, None] + col - have[:, None]
    page = s["free"][(count - 1 - k).clamp(0, s["pages"] - 1)]
    table = torch.where(new, page, table)
    t = torch.arange(T, device="cuda")
    r = torch.searchsorted(end, t, right=True).clamp(max=R - 1)
    pos = kv[r] + t - start[r]
    slot = table[r, (pos // P).clamp(max=s["cap"] - 1)].long() * P + pos % P
    slot = torch.where(ok[r] & (slot >= 0), slot, -1)
    zero = torch.zeros(1, dtype=torch.int64, device="cuda")
    return {"starts": torch.cat([zero, end]).int(), "kv_len": torch.where(ok, kv + q, kv).int(), "positions": pos.int(),
            "slots": slot.int(), "table": table, "free_count": (count - taken).int()}


# ------------------------------------------------------------------------------------------
# through the library
# ------------------------------------------------------------------------------------------
def _attach(s):
    """The handle, tables and workspace that a server keeps."""
    from paper_2602_24044_b200 import binding as lb
    from paper_2602_24044_b200.harness import KVCache
    c = s["case"]
    dev = torch.cuda.current_device()
    s["lb"] = lb
    heads = dict(num_q_heads=c["hq"], num_kv_heads=c["hkv"], head_dim=c["d"])
    s["kv"] = kv = KVCache(num_layers=1, num_pages=s["pages"], page_size=c["page"], device=dev, **heads)
    if c["op"] in ("append", "attention"):
        kv.layer(0).copy_(s["cache"])
    kv.reserve(s["R"], s["T"])
    if c["op"] == "tables":
        s["table_own"], s["kv_out"] = s["table"].clone(), torch.empty_like(s["kv_len"])
        s["count_out"] = torch.empty_like(s["free_count"])
    if c["op"] == "attention":
        # the pages are the same as those of full_table: the stack and the order of requests are
        kv.build_tables(s["kv_len"], s["q_len"], s["T"], s["free"], s["free_count"].clone(), s["table"].clone(),
                        max_q=s["max_q"], window=c["window"],
                        kv_len_out=torch.empty_like(s["kv_len"]))
    if c["op"] in ("norm_rope", "append"):
        T, hq, hkv, d = s["T"], c["hq"], c["hkv"], c["d"]
        qkv = s["qkv"]
        s["args"] = lb.qk_args(q=qkv, k=qkv[:, hq * d:], v=qkv[:, (hq + hkv) * d:], ldq=qkv.stride(0),
                               ldk=qkv.stride(0), ldv=qkv.stride(0), q_weight=s["qw"], k_weight=s["kw"], eps=1e-6,
                               cos_sin=s["angles"], positions=s["positions"], q_out=s["q_out"],
                               k_out=s["k_out"] if c["op"] == "norm_rope" else None, device=dev, **heads)


def _own_tables(s):
    kv = s["kv"]
    kv.build_tables(s["kv_len"], s["q_len"], s["T"], s["free"], s["free_count"], s["table_own"],
                    max_q=s["max_q"], stream=torch.cuda.current_stream(), kv_len_out=s["kv_out"], free_count_out=s["count_out"])
    return {"starts": kv.starts, "kv_len": s["kv_out"], "positions": kv.positions, "slots": kv.slots,
            "table": s["table_own"], "free_count": s["count_out"]}


def _own_norm_rope(s):
    s["lb"].qk_norm_rope(s["args"], s["T"], stream=torch.cuda.current_stream())
    return {"q": s["q_out"], "k": s["k_out"]}


def _own_append(s):
    kv, stream = s["kv"], torch.cuda.current_stream()
    kv.append(0, s["args"], s["slots"], s["T"], stream=stream)
    kv.read(0, s["slots"], s["k_out"], s["v_out"], stream=stream)
    return {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}


def _own_attention(s):
    s["kv"].attention(0, s["q"], s["out"], scale=s["scale"], stream=torch.cuda.current_stream())
    return {"out": s["out"]}


def run(state):
    op = state["case"]["op"]
    if own:
        return {"tables": _own_tables, "norm_rope": _own_norm_rope, "append": _own_append,
                "attention": _own_attention}[op](state)
    return {"tables": _plain_tables, "norm_rope": _plain_norm_rope, "append": _plain_append,
            "attention": _plain_attention}[op](state)


# ------------------------------------------------------------------------------------------
# the definition in 64 bits
# ------------------------------------------------------------------------------------------
def _exact_norm(x, w, pos, d, eps=1e-6):
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w
    out = torch.empty_like(y)
    for i in range(d // 2):
        # the angle table is an input in 32 bits
        f = torch.tensor(500000.0, device="cuda") ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float32)[i] / d)
        a = pos.float() * f
        c, s = a.cos().double()[:, None], a.sin().double()[:, None]
        out[..., i] = y[..., i] * c - y[..., i + d // 2] * s
        out[..., i + d // 2] = y[..., i + d // 2] * c + y[..., i] * s
    return out


def exact(case, seed):
    op = case["op"]
    if op == "tables":
        return None
    s = prepare(case, seed)
    T, hq, hkv, d, P = s["T"], case["hq"], case["hkv"], case["d"], case["page"]
    if op in ("norm_rope", "append"):
        x = s["qkv"].double().view(T, hq + 2 * hkv, d)
        q = _exact_norm(x[:, :hq], s["qw"].double(), s["positions"], d)
        k = _exact_norm(x[:, hq:hq + hkv], s["kw"].double(), s["positions"], d)
        if op == "norm_rope":
            return {"q": q.flatten(1), "k": k.flatten(1)}
        # what 4 bits leave of a row has no value in 64 bits apart from the rounding that the format makes
        return {"q": q.flatten(1), "k": None, "v": None}
    out = torch.zeros(T, hkv, hq // hkv, d, dtype=torch.float64, device="cuda")
    n = CELL * d // 2
    words = [NIBBLE.index(i) for i in range(8)]
    cells = _cells(case, s["cache"])
    t0 = 0
    for r, (kv, q) in enumerate(s["lens"]):
        end = kv + q
        pages = s["full_table"][r, :-(-end // P)].long()
        for h in range(hkv):
            b = cells[pages, h].reshape(-1, cells.shape[-1])
            par = b[:, 2 * n:].contiguous().view(torch.bfloat16).double().view(-1, 2, CELL, 2)
            val = []
            for j in (0, 1):
                byte = b[:, j * n:(j + 1) * n].reshape(-1, CELL, d // 8, 4).int()
                nib = torch.stack([byte & 15, byte >> 4], -1).reshape(-1, CELL, d // 8, 8)[..., words]
                y = nib.reshape(-1, CELL, d).double() * par[:, j, :, 0:1] + par[:, j, :, 1:2]
                val.append(y.reshape(-1, d)[:end])
            qr = s["q"][t0:t0 + q].view(q, hkv, hq // hkv, d)[:, h].double()
            x = torch.einsum("qgd,kd->qgk", qr, val[0]) * s["scale"]
            at = torch.arange(end, device="cuda")[None]
            limit = kv + torch.arange(q, device="cuda")[:, None] + 1
            seen = at < limit
            if case["window"]:
                seen &= at >= limit - case["window"]
            p = torch.softmax(x.masked_fill(~seen[:, None], -math.inf), -1)
            out[t0:t0 + q, h] = torch.einsum("qgk,kd->qgd", p, val[1])
        t0 += q
    return {"out": out.view(T, hq * d)}
