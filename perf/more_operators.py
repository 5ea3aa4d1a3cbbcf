"""The measured cases of the row operators before, inside and after a served attention layer: residual
addition with the root-mean-square norm (bf16 rows for the adapters, e4m3 rows with scales for a projection
in 8 bits), positions of image and video tokens on three axes, rotation of queries and keys by several axes
(alone, and with the 4-bit cache write), and sampling of the next tokens.  Each is given in its plain form
(elementary torch operations) and through the library.

Sizes follow the repository's workloads: rows of 4096 and 14336, 32 query heads and 8 key/value heads of 128
(the fused QKV projection 4096 -> 6144), 16 / 256 / 512 decode tokens, 32 prompts of 32..2048 tokens.
Vocabularies are generic.
"""
import math
import random

import torch

own = False

CELL = 16
TIME, HEIGHT, WIDTH = 0, 1, 2


# ------------------------------------------------------------------------------------------
# cases
# ------------------------------------------------------------------------------------------
def _norm(name, **kw):
    c = {"name": name, "op": "norm", "tokens": 1, "width": 4096, "residual": True, "rows": True, "group": 0}
    c.update(kw)
    return c


def _batch(name, op, **kw):
    c = {"name": name, "op": op, "hq": 32, "hkv": 8, "d": 128, "rot": 128, "pairs": False, "page": 16, "striped": False,
         "lens": 1, "decode": 0, "ctx_lo": 1, "ctx_hi": 1, "prompts": 0, "q_lo": 0, "q_hi": 0, "media": 4}
    c.update(kw)
    return c


def _sample(name, **kw):
    c = {"name": name, "op": "sample", "requests": 1, "vocab": 32000, "bf16": False, "filters": "mixed", "masked": 0.1}
    c.update(kw)
    return c


def listed():
    return [
        # the smallest decode batch between two projections: the time is launch latency
        _norm("norm_decode", tokens=16),
        # a prefill step of 32 prompts
        _norm("norm_prompts", tokens=12937),
        # the same for a base projection in 8 bits (a scale for each 128 values) with adapters on bf16 rows
        _norm("norm_prompts_8bit", tokens=12937, group=128),
        # one decode step of a busy server whose requests hold images and videos
        _batch("positions_decode", "positions", decode=256, ctx_lo=1, ctx_hi=8192),
        # 32 prompts with images in them
        _batch("positions_prompts", "positions", prompts=32, q_lo=32, q_hi=2048, media=12),
        # queries and keys of a handful of decode tokens, channels of the axes in sections
        _batch("rotate_decode", "rotate", decode=16, ctx_lo=1, ctx_hi=2048),
        # queries and keys of 32 prompts, channels of the axes in turn
        _batch("rotate_prompts", "rotate", prompts=32, q_lo=32, q_hi=2048, striped=True),
        # cache write of one decode step
        _batch("append_decode", "append", decode=256, ctx_lo=1, ctx_hi=2048, striped=True),
        # cache write of 32 prompts on pages of 64 tokens
        _batch("append_prompts", "append", prompts=32, q_lo=32, q_hi=2048, page=64),
        # the next tokens of a handful of requests
        _sample("sample_few", requests=4, bf16=True),
        # a busy server's step, every request with parameters of its own
        _sample("sample_batch", requests=256, vocab=128000),
        # samples for training: temperature alone, the whole vocabulary counts
        _sample("sample_whole", requests=512, vocab=150001, bf16=True, filters="none", masked=0.0),
    ]


def _log_uniform(rng, lo, hi):
    if hi <= lo:
        return lo
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(max(lo, 1)), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm", "positions", "rotate", "append", "sample", "sample"])
    if op == "norm":
        group = rng.choice([0, 1, 32, 128])
        unit = max(8, group)
        width = unit * _log_uniform(rng, max(1, 64 // unit), 16384 // unit)
        c = _norm("", tokens=_log_uniform(rng, 1, min(20000, 12937 * 4096 // width)), width=width, group=group,
                  residual=rng.random() < 0.7, rows=group == 0 or rng.random() < 0.5)
    elif op == "sample":
        vocab = _log_uniform(rng, 100, 200000)
        c = _sample("", vocab=vocab, requests=_log_uniform(rng, 1, min(512, 512 * 150001 // (2 * vocab))),
                    bf16=rng.random() < 0.5, filters=rng.choice(["mixed", "mixed", "none", "greedy", "wide"]),
                    masked=rng.choice([0.0, 0.1, 0.5]))
    else:
        d = rng.choice([64, 128])
        hkv = rng.choice([1, 2, 4, 8])
        kw = dict(hq=hkv * rng.choice([1, 2, 4, 5, 7] if hkv < 8 else [1, 2, 4]), hkv=hkv, d=d,
                  rot=rng.choice([d, d, d // 2]), pairs=rng.random() < 0.3, page=rng.choice([16, 32, 64, 128]),
                  striped=rng.random() < 0.5, lens=rng.randrange(1 << 20), media=_log_uniform(rng, 1, 20))
        kind = rng.choice(["decode", "prompts", "mixed"])
        if kind != "prompts":
            kw.update(decode=_log_uniform(rng, 1, 512), ctx_lo=rng.choice([0, 1, 100]), ctx_hi=_log_uniform(rng, 128, 8192))
        if kind == "prompts":
            kw.update(prompts=_log_uniform(rng, 1, 24), q_lo=_log_uniform(rng, 1, 64), q_hi=_log_uniform(rng, 65, 2000))
        if kind == "mixed":
            kw.update(prompts=rng.randint(1, 4), q_lo=33, q_hi=_log_uniform(rng, 64, 700))
        c = _batch("", op, **kw)
    del c["name"]
    return c


def _lengths(case):
    """[(keys already cached, new tokens)] of the batch: decode requests first, then prompts."""
    rng = random.Random(case["lens"])
    out = [(_log_uniform(rng, case["ctx_lo"], case["ctx_hi"]), 1) for _ in range(case["decode"])]
    return out + [(0, _log_uniform(rng, case["q_lo"], case["q_hi"])) for _ in range(case["prompts"])]


def _spans(case, lens, seed):
    """Images and videos of each request, [(first token, frames, rows, columns, position of the first, step of a
    frame)]: text between them counts one by one, what follows one goes on behind its largest position."""
    rng = random.Random(seed * 7919 + case["lens"])
    out = []
    for kv, q in lens:
        # decode requests have theirs behind them; a few end inside one that is still to come in full
        at, base, mine = 0, 0, []
        for _ in range(rng.randint(0, case["media"])):
            text = rng.randint(0, 40)
            t, h, w, step = rng.choice([1, 1, 1, rng.randint(2, 6)]), rng.randint(2, 24), rng.randint(2, 24), rng.randint(1, 4)
            if at + text >= kv + q:
                break
            at, base = at + text, base + text
            mine.append((at, t, h, w, base, step))
            at, base = at + t * h * w, base + max((t - 1) * step + 1, h, w)
        out.append(mine)
    return out


def work(case):
    if case["op"] == "norm":
        T, n, g = case["tokens"], case["width"], case["group"]
        size = 2 * T * n * (1 + 2 * case["residual"] + case["rows"]) + 2 * n
        if g:
            size += T * n + (T * 4 if g == 1 else T * n // g * (1 if g == 32 else 4))
        return {"bytes": size, "flops": 5 * T * n}
    if case["op"] == "sample":
        R, V = case["requests"], case["vocab"]
        return {"bytes": R * V * (2 if case["bf16"] else 4) + 28 * R, "flops": 4 * R * V}
    hq, hkv, d, rot = case["hq"], case["hkv"], case["d"], case["rot"]
    lens = _lengths(case)
    R, T = len(lens), sum(q for _, q in lens)
    if case["op"] == "positions":   # starts, positions and spans in; three positions a token out
        return {"bytes": 4 * (2 * R + 2 + T) + 32 * sum(len(m) for m in _spans(case, lens, 1)) + 12 * T, "flops": 0}
    angles = 12 * T + 4 * T * rot   # three positions and a cosine and a sine for each pair
    if case["op"] == "rotate":
        return {"bytes": 4 * T * (hq + hkv) * d + angles, "flops": 8 * T * (hq + hkv) * d}
    # q, k, v in; q and the cache rows out; the rows back in and out as bf16
    return {"bytes": 4 * T * hq * d + 4 * T * hkv * d + 2 * T * hkv * (d + 8) + 4 * T * hkv * d + 4 * T + angles,
            "flops": 8 * T * (hq + 3 * hkv) * d}


# ------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------
def _axis_of_pair(case):
    """Which axis turns each rotation pair: a quarter, three eighths and three eighths of the pairs in sections,
    or time, height and width in turn with what is left over for time."""
    half = case["rot"] // 2
    if case["striped"]:
        each = 3 * half // 8
        return [p % 3 if p < 3 * each else TIME for p in range(half)]
    return [TIME] * (half // 4) + [HEIGHT] * (3 * half // 8) + [WIDTH] * (half - half // 4 - 3 * half // 8)


def _positions_on_host(lens, spans):
    """[(time, height, width)] of every new token, one request after the other."""
    out = []
    for (kv, q), mine in zip(lens, spans):
        for p in range(kv, kv + q):
            here = [m for m in mine if m[0] <= p]
            if not here:
                out.append((p, p, p))
                continue
            first, t, h, w, base, step = here[-1]
            k = p - first
            if k < t * h * w:
                out.append((base + k // (h * w) * step, base + k // w % h, base + k % w))
            else:
                out.append((k - t * h * w + base + max((t - 1) * step + 1, h, w),) * 3)
    return out


def _prepare_norm(case, g):
    T, n = case["tokens"], case["width"]
    bf = dict(generator=g, device="cuda")
    s = {"x": (torch.randn(T, n, **bf) * 0.5).bfloat16(), "w": (1 + 0.2 * torch.randn(n, **bf)).bfloat16(), "eps": 1e-6,
         "y": torch.empty(T, n, dtype=torch.bfloat16, device="cuda") if case["rows"] else None, "r": None, "r_out": None}
    if case["residual"]:
        # the stream of a deep layer: a few channels much larger than the others
        gain = torch.exp(0.8 * torch.randn(n, **bf))
        s["r"] = (2 * torch.randn(T, n, **bf) * gain).bfloat16()
        s["r_out"] = torch.empty_like(s["r"])
    if case["group"]:
        s["codes"] = torch.empty(T, n, dtype=torch.float8_e4m3fn, device="cuda")
        groups = 1 if case["group"] == 1 else n // case["group"]
        s["scales"] = torch.empty(T, groups, dtype=torch.uint8 if case["group"] == 32 else torch.float32, device="cuda")
    return s


def _prepare_sample(case, g):
    R, V = case["requests"], case["vocab"]
    kw = dict(generator=g, device="cuda")
    # a model's logits: a broad field with a few that stand out
    x = torch.randn(R, V, **kw) * 2.2
    stand_out = torch.randint(0, V, (R, 64), **kw)
    x.scatter_add_(1, stand_out, -2.5 * torch.log(torch.rand(R, 64, **kw)) + 6 * torch.rand(R, 1, **kw))
    # requests whose grammar leaves a few tokens
    few = torch.rand(R, 1, **kw) < case["masked"]
    x.masked_fill_(few & (torch.rand(R, V, **kw) < 0.99), -math.inf)
    s = {"logits": x.bfloat16() if case["bf16"] else x, "uniform": torch.rand(R, **kw), "top_k": None, "top_p": None,
         "min_p": None, "token": torch.empty(R, dtype=torch.int32, device="cuda"),
         "logprob": torch.empty(R, dtype=torch.float32, device="cuda")}

    def one_of(values, dtype):
        at = torch.randint(0, len(values), (R,), **kw)
        return torch.tensor(values, dtype=dtype, device="cuda")[at]

    if case["filters"] == "greedy":
        s["temperature"] = torch.zeros(R, device="cuda")
    elif case["filters"] == "none":
        s["temperature"] = 0.7 + 0.5 * torch.rand(R, **kw)
    elif case["filters"] == "wide":
        s["temperature"] = one_of([0.8, 1.0, 1.5], torch.float32)
        s["top_k"] = one_of([0, 1000, 5000], torch.int32)
        s["top_p"] = one_of([0.9, 0.98, 0.999], torch.float32)
    else:
        s["temperature"] = one_of([0.0, 0.6, 0.8, 1.0, 1.0, 1.3], torch.float32)
        s["top_k"] = one_of([0, 0, 1, 20, 50, 200], torch.int32)
        s["top_p"] = one_of([1.0, 0.5, 0.9, 0.95], torch.float32)
        s["min_p"] = one_of([0.0, 0.0, 0.02, 0.1], torch.float32)
    return s


def _prepare_batch(case, g, seed):
    dev = "cuda"
    i32 = dict(dtype=torch.int32, device=dev)
    hq, hkv, d, P, rot = case["hq"], case["hkv"], case["d"], case["page"], case["rot"]
    lens = _lengths(case)
    spans = _spans(case, lens, seed)
    R, T = len(lens), sum(q for _, q in lens)
    s = {"lens": lens, "R": R, "T": T, "kv_len": torch.tensor([kv for kv, _ in lens], **i32),
         "q_len": torch.tensor([q for _, q in lens], **i32)}
    flat = [(*m, 0, 0) for mine in spans for m in mine]
    s["spans"] = torch.tensor(flat or [(0,) * 8], **i32)
    begin = [0]
    for mine in spans:
        begin.append(begin[-1] + len(mine))
    s["begin"] = torch.tensor(begin, **i32)
    s["starts"] = torch.cumsum(torch.tensor([0] + [q for _, q in lens], device=dev), 0).int()
    s["at"] = torch.cat([torch.arange(kv, kv + q, **i32) for kv, q in lens])
    on_host = _positions_on_host(lens, spans)
    s["positions"] = torch.tensor(on_host, **i32).t().contiguous()
    s["positions_out"] = torch.empty_like(s["positions"])
    before, after = [-(-kv // P) for kv, _ in lens], [-(-(kv + q) // P) for kv, q in lens]
    s["cap"], s["pages"] = max(after) + 1, sum(after) + 7
    order = torch.randperm(s["pages"], generator=g, device=dev).to(torch.int32)
    table = torch.full((R, s["cap"]), -1, **i32)
    col = torch.arange(s["cap"], device=dev)[None]
    held = col < torch.tensor(before, device=dev)[:, None]
    table[held] = order[: sum(before)]
    s["table"], s["free"] = table, order[sum(before):].contiguous()
    s["count"] = torch.tensor([s["pages"] - sum(before)], **i32)
    if case["op"] == "positions":
        return s
    # the fused projection's output: one row a token, query heads, then key heads, then value heads
    s["qkv"] = torch.randn(T, (hq + 2 * hkv) * d, generator=g, device=dev).mul_(
        torch.rand((hq + 2 * hkv) * d, generator=g, device=dev) + 0.5).bfloat16()
    s["qw"] = (1 + 0.3 * torch.randn(d, generator=g, device=dev)).bfloat16()
    s["kw"] = (1 + 0.3 * torch.randn(d, generator=g, device=dev)).bfloat16()
    f = 500000.0 ** (-torch.arange(0, rot, 2, device=dev, dtype=torch.float32) / rot)
    a = torch.arange(max(max(p) for p in on_host) + 1, device=dev, dtype=torch.float32)[:, None] * f
    s["angles"] = torch.cat([a.cos(), a.sin()], -1).contiguous()
    s["axis"] = _axis_of_pair(case)
    s["axis_dev"] = torch.tensor(s["axis"], device=dev)
    s["q_out"] = torch.empty(T, hq * d, dtype=torch.bfloat16, device=dev)
    s["k_out"] = torch.empty(T, hkv * d, dtype=torch.bfloat16, device=dev)
    s["v_out"] = torch.empty(T, hkv * d, dtype=torch.bfloat16, device=dev)
    if case["op"] == "append":
        s["cache"] = torch.full((s["pages"] * hkv * P * (d + 8),), 255, dtype=torch.uint8, device=dev)
        full = table.clone()
        new = col < torch.tensor(after, device=dev)[:, None]
        full[new & ~held] = s["free"].flip(0)[: sum(after) - sum(before)]
        r = torch.repeat_interleave(torch.arange(R, device=dev), s["q_len"].long())
        at = s["at"].long()
        s["slots"] = (full[r, at // P] * P + at % P).int()
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] == "norm":
        s = _prepare_norm(case, g)
    elif case["op"] == "sample":
        s = _prepare_sample(case, g)
    else:
        s = _prepare_batch(case, g, seed)
    s["case"] = case
    if own:
        _attach(s)
    return s


# ------------------------------------------------------------------------------------------
# plain forms
# ------------------------------------------------------------------------------------------
def _pair_sum(x):
    """The sum over the last dimension, neighbours first (its order is part of the operator)."""
    return x[..., 0] if x.shape[-1] == 1 else _pair_sum(x[..., 0::2] + x[..., 1::2])


def _plain_norm(s):
    c = s["case"]
    T, n, g = c["tokens"], c["width"], c["group"]
    x = s["x"].float()
    out = {}
    if c["residual"]:
        x = x + s["r"].float()
        out["residual"] = x.bfloat16()
    # squares of eight neighbours in 32 bits, the sum of these in 64: so its order does not matter
    total = _pair_sum((x * x).unflatten(-1, (n // 8, 8))).double().sum(-1).float()
    y = x * (1.0 / torch.sqrt(total * (1.0 / n) + s["eps"]))[:, None] * s["w"].float()
    if c["rows"]:
        out["rows"] = y.bfloat16()
    if g:
        y = y.unflatten(-1, (-1, n if g == 1 else g))
        top = y.abs().amax(-1)
        bad = ~torch.isfinite(top)
        if g == 32:
            # the smallest power of two that brings the group to 448 or less
            m, e = torch.frexp(top)
            e = (e - 9 + (m > 0.875)).clamp(-127, 127)
            scales = torch.where(top == 0, 0, e + 127).masked_fill(bad, 255).to(torch.uint8)
            inv = torch.ldexp(torch.ones_like(top), torch.where(top == 0, 0, -e))
        else:
            scales = top * (1.0 / 448.0)
            scales = torch.where(scales < 1.17549435e-38, torch.zeros_like(scales), scales).masked_fill(bad, math.nan)
            inv = torch.where(scales == 0, torch.zeros_like(scales), 1.0 / scales)
        codes = (y * inv[..., None]).masked_fill(bad[..., None], 0.0)
        out["codes"], out["scales"] = codes.flatten(1).to(torch.float8_e4m3fn), scales
    return out


def _plain_positions(s):
    T, R, S = s["T"], s["R"], s["spans"].shape[0]
    t = torch.arange(T, device="cuda")
    starts, begin, spans = s["starts"].long(), s["begin"].long(), s["spans"].long()
    r = torch.searchsorted(starts[1:].contiguous(), t, right=True).clamp(max=R - 1)
    p = s["at"].long()
    # the last span of the token's request that begins at or before it
    of = torch.searchsorted(begin[1:].contiguous(), torch.arange(S, device="cuda"), right=True)
    key = of * (1 << 32) + spans[:, 0]
    i = torch.searchsorted(key, r * (1 << 32) + p, right=True) - 1
    some = i >= begin[r]
    first, f, h, w, base, step = (spans[i.clamp(min=0)][:, j] for j in range(6))
    k, size = p - first, f * h * w
    inside = k < size
    hw, w1 = (h * w).clamp(min=1), w.clamp(min=1)
    behind = k - size + base + torch.maximum(torch.maximum((f - 1) * step + 1, h), w)
    axes = torch.stack([base + k // hw * step, base + k % hw // w1, base + k % w1])
    axes = torch.where(inside, axes, behind)
    return {"positions": torch.where(some, axes, p).int()}


def _plain_turn(x, c, s, pairs):
    """float32 [T, heads, rot] by the cosines and sines [T, rot / 2]"""
    c, s = c[:, None], s[:, None]
    if pairs:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    a, b = x.chunk(2, -1)
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def _plain_head_norm(x, w, eps):
    h = x.shape[-1] // 2
    sq = x * x
    ms = _pair_sum(sq[..., :h] + sq[..., h:]) / x.shape[-1]
    return x * (1.0 / torch.sqrt(ms + eps))[..., None] * w


def _plain_qkv(s):
    c = s["case"]
    T, hq, hkv, d, rot = s["T"], c["hq"], c["hkv"], c["d"], c["rot"]
    x = s["qkv"].float().view(T, hq + 2 * hkv, d)
    p = torch.arange(rot // 2, device="cuda")
    row = s["positions"].long()[s["axis_dev"]].t()                       # [T, rot / 2]: each pair's row of the table
    cos, sin = s["angles"][row, p], s["angles"][row, p + rot // 2]
    q = _plain_head_norm(x[:, :hq], s["qw"].float(), 1e-6)
    k = _plain_head_norm(x[:, hq:hq + hkv], s["kw"].float(), 1e-6)
    q = torch.cat([_plain_turn(q[..., :rot], cos, sin, c["pairs"]), q[..., rot:]], -1)
    k = torch.cat([_plain_turn(k[..., :rot], cos, sin, c["pairs"]), k[..., rot:]], -1)
    return q, k, x[:, hq + hkv:]


def _plain_rotate(s):
    q, k, _ = _plain_qkv(s)
    return {"q": q.bfloat16().flatten(1), "k": k.bfloat16().flatten(1)}


#: nibble n of a 32-bit word of the cache holds element NIBBLE[n] of its eight
NIBBLE = (0, 2, 4, 6, 1, 3, 5, 7)
ELEMENT = tuple(NIBBLE.index(i) for i in range(8))


def _quantise(x):
    """float32 [..., D] -> codes (float32, whole numbers 0..15), scale and low (bfloat16 [...])."""
    low = x.amin(-1).bfloat16()
    scale = ((x.amax(-1) - low.float()) * (1.0 / 15.0)).bfloat16()
    inv = torch.where(scale == 0, torch.zeros_like(scale, dtype=torch.float32), 1.0 / scale.float())
    return torch.round((x - low.float()[..., None]) * inv[..., None]).clamp(0.0, 15.0), scale, low


def _pack(codes):
    n = codes.to(torch.uint8).unflatten(-1, (-1, 8))[..., list(NIBBLE)]
    return (n[..., 0::2] | (n[..., 1::2] << 4)).flatten(-2)


def _unpack(b):
    n = torch.stack([b & 15, b >> 4], -1).unflatten(-2, (-1, 4)).flatten(-2)
    return n[..., list(ELEMENT)].flatten(-2).float()


def _plain_append(s):
    c = s["case"]
    d, P, hkv = c["d"], c["page"], c["hkv"]
    n = CELL * d // 2
    q, k, v = _plain_qkv(s)
    cells = s["cache"].view(-1, hkv, P // CELL, CELL * (d + 8))
    slots = s["slots"].long()
    at = ((slots // P)[:, None], torch.arange(hkv, device="cuda")[None], (slots % P // CELL)[:, None])
    row = (slots % CELL)[:, None]
    codes = cells[..., :2 * n].unflatten(-1, (2, CELL, d // 2))
    params = cells[..., 2 * n:].unflatten(-1, (2, CELL, 4))
    (kc, ks, kl), (vc, vs, vl) = _quantise(k), _quantise(v)
    codes[at + (0, row)], codes[at + (1, row)] = _pack(kc), _pack(vc)
    params[at + (0, row)] = torch.stack([ks, kl], -1).view(torch.uint8)
    params[at + (1, row)] = torch.stack([vs, vl], -1).view(torch.uint8)
    # the written rows as the values they stand for
    kp = params[at + (0, row)].view(torch.bfloat16).float()
    vp = params[at + (1, row)].view(torch.bfloat16).float()
    k_back = _unpack(codes[at + (0, row)]) * kp[..., 0:1] + kp[..., 1:2]
    v_back = _unpack(codes[at + (1, row)]) * vp[..., 0:1] + vp[..., 1:2]
    return {"q": q.bfloat16().flatten(1), "k": k_back.bfloat16().flatten(1), "v": v_back.bfloat16().flatten(1)}


def _plain_sample(s):
    x, u = s["logits"].float(), s["uniform"].double()
    R, V = x.shape
    top = x.amax(-1, keepdim=True)
    tau = s["temperature"].double()[:, None]
    greedy = ~(tau > 0)
    # in 64 bits: whether a token is kept, and which one u falls on, is decided next to borders
    e = (x.double() - top.double()) / torch.where(greedy, 1.0, tau)
    e = torch.where(x == top, 0.0, e)
    w = torch.where((x == -math.inf) | (e < -46 * math.log(2.0)), 0.0, torch.exp(e))
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices      # ties: the lowest index first
    ws = w.gather(1, order)
    rank = torch.arange(V, device="cuda")[None]
    keep = torch.ones_like(ws, dtype=torch.bool)
    if s["top_k"] is not None:
        k = s["top_k"].long()[:, None]
        keep &= (rank < k) | (k <= 0)
    if s["min_p"] is not None:
        p = s["min_p"].double()[:, None].clamp(max=1.0)
        keep &= (e.gather(1, order) >= torch.log(p)) | ~(p > 0)
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        cum = torch.cumsum(torch.where(keep, ws, 0.0), -1)
        keep &= (cum - ws < p * cum[:, -1:]) | ~(p < 1) | (rank == 0)
    kept = torch.zeros_like(w).scatter_(1, order, torch.where(keep, ws, 0.0))
    cum = torch.cumsum(kept, -1)
    total = cum[:, -1:]
    at = torch.searchsorted(cum, u[:, None] * total, right=True).clamp(max=V - 1)
    at = torch.where(greedy, order[:, :1], at)
    logprob = torch.where(greedy, 0.0, torch.log(kept.gather(1, at) / total))
    return {"token": at[:, 0].int(), "logprob": logprob[:, 0].float()}


# ------------------------------------------------------------------------------------------
# through the library
# ------------------------------------------------------------------------------------------
def _attach(s):
    """The argument blocks, handle and tables that a server keeps."""
    from paper_2602_24044_b200 import binding as lb
    from paper_2602_24044_b200.harness import KVCache
    c = s["case"]
    dev = torch.cuda.current_device()
    s["lb"] = lb
    if c["op"] == "norm":
        s["args"] = lb.norm_args(x=s["x"], weight=s["w"], eps=s["eps"], residual=s["r"], residual_out=s["r_out"],
                                 out=s["y"], codes=s.get("codes"), scales=s.get("scales"),
                                 group={0: 0, 1: c["width"]}.get(c["group"], c["group"]), device=dev)
        return
    if c["op"] == "sample":
        s["args"] = lb.sample_args(logits=s["logits"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                                   min_p=s["min_p"], uniform=s["uniform"], token=s["token"], logprob=s["logprob"],
                                   device=dev)
        return
    heads = dict(num_q_heads=c["hq"], num_kv_heads=c["hkv"], head_dim=c["d"])
    if c["op"] != "rotate":
        s["kv"] = kv = KVCache(num_layers=1, num_pages=s["pages"], page_size=c["page"], device=dev, **heads)
        if c["op"] == "append":
            kv.layer(0).copy_(s["cache"])
        else:
            kv.build_tables(s["kv_len"], s["q_len"], s["T"], s["free"], s["count"].clone(), s["table"].clone(),
                            kv_len_out=torch.empty_like(s["kv_len"]), stream=torch.cuda.current_stream())
            return
    hq, hkv, d, qkv = c["hq"], c["hkv"], c["d"], s["qkv"]
    s["args"] = lb.qk_args(q=qkv, k=qkv[:, hq * d:], v=qkv[:, (hq + hkv) * d:], ldq=qkv.stride(0), ldk=qkv.stride(0),
                           ldv=qkv.stride(0), q_weight=s["qw"], k_weight=s["kw"], eps=1e-6, cos_sin=s["angles"],
                           interleaved=c["pairs"], positions=s["positions"], axis_of_pair=s["axis"], q_out=s["q_out"],
                           k_out=s["k_out"] if c["op"] == "rotate" else None, device=dev, **heads)


def _own_norm(s):
    s["lb"].add_norm(s["args"], s["case"]["tokens"], stream=torch.cuda.current_stream())
    out = {} if s["r"] is None else {"residual": s["r_out"]}
    if s["y"] is not None:
        out["rows"] = s["y"]
    if s["case"]["group"]:
        out["codes"], out["scales"] = s["codes"], s["scales"]
    return out


def _own_positions(s):
    s["kv"].axis_positions(s["spans"], s["begin"], s["positions_out"], stream=torch.cuda.current_stream())
    return {"positions": s["positions_out"]}


def _own_rotate(s):
    s["lb"].qk_norm_rope(s["args"], s["T"], stream=torch.cuda.current_stream())
    return {"q": s["q_out"], "k": s["k_out"]}


def _own_append(s):
    kv, stream = s["kv"], torch.cuda.current_stream()
    kv.append(0, s["args"], s["slots"], s["T"], stream=stream)
    kv.read(0, s["slots"], s["k_out"], s["v_out"], stream=stream)
    return {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}


def _own_sample(s):
    s["lb"].sample(s["args"], s["case"]["requests"], stream=torch.cuda.current_stream())
    return {"token": s["token"], "logprob": s["logprob"]}


def run(state):
    op = state["case"]["op"]
    if own:
        return {"norm": _own_norm, "positions": _own_positions, "rotate": _own_rotate, "append": _own_append,
                "sample": _own_sample}[op](state)
    return {"norm": _plain_norm, "positions": _plain_positions, "rotate": _plain_rotate, "append": _plain_append,
            "sample": _plain_sample}[op](state)


# ------------------------------------------------------------------------------------------
# the definition in 64 bits
# ------------------------------------------------------------------------------------------
def _exact_norm(case, s):
    n, g = case["width"], case["group"]
    x = s["x"].double()
    out = {}
    if case["residual"]:
        x = x + s["r"].double()
        out["residual"] = x
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * s["w"].double()
    if case["rows"]:
        out["rows"] = y
    if g:
        z = y.view(y.shape[0], -1, n if g == 1 else g)
        top = z.abs().amax(-1)
        # the codes' values before their rounding; the power of two of a group of 32 is a whole number
        scale = torch.exp2(torch.ceil(torch.log2(top / 448.0))) if g == 32 else top / 448.0
        out["codes"] = (z / scale[..., None]).flatten(1)
        out["scales"] = None if g == 32 else scale
    return out


def _exact_qk(case, s):
    T, hq, hkv, d, half = s["T"], case["hq"], case["hkv"], case["d"], case["rot"] // 2
    x = s["qkv"].double().view(T, hq + 2 * hkv, d)
    pos = s["positions"].long()
    out = []
    for part, w in ((x[:, :hq], s["qw"]), (x[:, hq:hq + hkv], s["kw"])):
        y = part / torch.sqrt((part * part).mean(-1, keepdim=True) + 1e-6) * w.double()
        z = y.clone()
        for p in range(half):
            i, j = (2 * p, 2 * p + 1) if case["pairs"] else (p, p + half)
            row = s["angles"][pos[s["axis"][p]]].double()       # the angle table is an input in 32 bits
            c, n = row[:, None, p], row[:, None, half + p]
            z[..., i] = y[..., i] * c - y[..., j] * n
            z[..., j] = y[..., j] * c + y[..., i] * n
        out.append(z.flatten(1))
    return out


def _exact_sample(s):
    R, V = s["logits"].shape
    token, logprob = [], []
    for r in range(R):
        x, tau = s["logits"][r].double(), float(s["temperature"][r])
        by_size = torch.argsort(x, descending=True, stable=True)
        if not tau > 0:
            token.append(int(by_size[0]))
            logprob.append(0.0)
            continue
        p = torch.softmax(x[by_size] / tau, -1)
        n = V if s["top_k"] is None or int(s["top_k"][r]) <= 0 else min(V, int(s["top_k"][r]))
        if s["min_p"] is not None:
            n = min(n, max(1, int((p >= float(s["min_p"][r]) * p[0]).sum())))
        if s["top_p"] is not None and float(s["top_p"][r]) < 1:
            before = torch.cumsum(p[:n], 0) - p[:n]
            n = max(1, int((before < float(s["top_p"][r]) * p[:n].sum()).sum()))
        mine = torch.sort(by_size[:n]).values
        q = torch.softmax(x[mine] / tau, -1)
        i = min(int((torch.cumsum(q, 0) <= float(s["uniform"][r])).sum()), n - 1)
        token.append(int(mine[i]))
        logprob.append(float(torch.log(q[i])))
    return {"token": torch.tensor(token, dtype=torch.int32), "logprob": torch.tensor(logprob, dtype=torch.float64)}


def exact(case, seed):
    if case["op"] == "positions":
        return None
    s = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(case, s)
    if case["op"] == "sample":
        return _exact_sample(s)
    q, k = _exact_qk(case, s)
    if case["op"] == "rotate":
        return {"q": q, "k": k}
    # what 4 bits leave of a row has no value in 64 bits apart from the rounding that the format makes
    return {"q": q, "k": None, "v": None}
