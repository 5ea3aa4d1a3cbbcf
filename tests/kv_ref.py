"""Plain definitions of the cache operators for the tests: loops and float64, or float32 step by step
where the operator's result is defined bit for bit.  numpy only; nothing of the library."""
import numpy as np

NIBBLE = (0, 2, 4, 6, 1, 3, 5, 7)      # nibble n of a word holds element NIBBLE[n] of its eight
CELL = 16


def bf16(x):
    """float32 -> nearest bfloat16 (ties to even), as float32; NaN stays NaN."""
    x = np.asarray(x, np.float32)
    u = x.view(np.uint32)
    r = ((u >> np.uint32(16)) & np.uint32(1)) + np.uint32(0x7FFF)
    out = ((u + r) & np.uint32(0xFFFF0000)).view(np.float32)
    return np.where(np.isnan(x), np.float32(np.nan), out)


# -- tables ---------------------------------------------------------------------------------
def tables(kv_len, q_len, T, P, free, count, table, num_pages, max_q=0):
    R, cap = table.shape
    table = table.copy()
    max_q = T if max_q == 0 or max_q > T else max_q
    kv = [max(int(k), 0) for k in kv_len]
    q = [max(int(x), 0) for x in q_len]
    count = min(max(int(count), 0), num_pages)
    start, after, pos, slot = [0], [], [0] * T, [-1] * T
    end, upto, taken, n_failed = 0, 0, 0, 0
    for r in range(R):
        first = min(end, T)
        end += q[r]
        ok = end <= T and q[r] <= max_q and -(-(kv[r] + q[r]) // P) <= cap
        need = -(-(kv[r] + q[r]) // P) - -(-kv[r] // P) if ok else 0
        upto += need
        if need and upto > count:
            ok = False
        if ok:
            old = -(-kv[r] // P)
            for i in range(need):
                table[r, old + i] = free[count - 1 - (upto - need + i)]
            if need:
                taken = upto
        n_failed += not ok
        for t in range(first, min(end, T)):
            pos[t] = kv[r] + t - first
            if ok:
                page = int(table[r, pos[t] // P])
                slot[t] = page * P + pos[t] % P if 0 <= page < num_pages else -1
        start.append(min(end, T))
        after.append(kv[r] + q[r] if ok else kv[r])
    neg = sum(int(a) < 0 or int(b) < 0 for a, b in zip(kv_len, q_len))
    return {"header": [R, T, end, n_failed, neg, taken], "start": start, "kv_len": after, "position": pos,
            "slot": slot, "table": table, "free_count": count - taken}


# -- rows -----------------------------------------------------------------------------------
def norm32(x, w, eps):
    """float32 [n, D], every operation rounded by itself, the sum of squares as the documented tree."""
    D = x.shape[-1]
    sq = x * x
    s = sq[:, : D // 2] + sq[:, D // 2:]
    while s.shape[-1] > 1:
        s = s[:, 0::2] + s[:, 1::2]
    r = np.float32(1) / np.sqrt(s * np.float32(1.0 / D) + np.float32(eps))
    return (x * r) * w


def rotate(x, cos_sin, rot, interleaved):
    """[n, D] of float32 (each operation rounded) or float64; cos_sin [n, rot]."""
    y, h = x.copy(), rot // 2
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, h), slice(h, rot))
    c, s = cos_sin[:, :h], cos_sin[:, h:]
    y[:, a] = x[:, a] * c - x[:, b] * s
    y[:, b] = x[:, b] * c + x[:, a] * s
    return y


def quantise(x):
    """float32 [n, D] -> codes uint8 [n, D], scale and low float32 (bf16 values) [n]."""
    with np.errstate(all="ignore"):
        low = bf16(x.min(-1))
        scale = bf16((x.max(-1) - low) * np.float32(1.0 / 15.0))
        scale = np.where(scale < np.float32(1.17549435e-38), np.float32(0), scale)
        bad = ~(np.isfinite(scale) & np.isfinite(low) & np.isfinite(x).all(-1))
        inv = np.where(scale == 0, np.float32(0), np.float32(1) / np.where(scale == 0, np.float32(1), scale))
        c = np.clip(np.rint((x - low[:, None]) * inv[:, None].astype(np.float32)), 0, 15)
    c = np.where(bad[:, None], 0, c)
    nan = np.float32(np.nan)
    return c.astype(np.uint8), np.where(bad, nan, scale), np.where(bad, nan, low)


def dequantise32(c, scale, low):
    return c.astype(np.float32) * scale[:, None] + low[:, None]


def _bits(x):
    return (np.asarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16)


def pack_layer(K, V, num_pages, P, hkv, D):
    """K, V: (codes [slots, hkv, D], scale, low [slots, hkv]) with slots = num_pages * P -> bytes of a layer."""
    n = num_pages * (P // CELL)
    out = np.empty((num_pages, hkv, P // CELL, CELL * (D + 8)), np.uint8)
    part = CELL * D // 2
    for j, (c, s, l) in enumerate((K, V)):
        w = c.reshape(num_pages, P // CELL, CELL, hkv, D // 8, 8)[..., list(NIBBLE)]
        b = (w[..., 0::2] | (w[..., 1::2] << 4)).reshape(num_pages, P // CELL, CELL, hkv, D // 2)
        out[..., j * part:(j + 1) * part] = b.transpose(0, 3, 1, 2, 4).reshape(num_pages, hkv, P // CELL, part)
        p = np.stack([_bits(s), _bits(l)], -1).reshape(num_pages, P // CELL, CELL, hkv, 2)
        pb = np.ascontiguousarray(p.transpose(0, 3, 1, 2, 4)).view(np.uint8)
        at = 2 * part + j * CELL * 4
        out[..., at:at + CELL * 4] = pb.reshape(num_pages, hkv, P // CELL, CELL * 4)
    assert n * hkv * CELL * (D + 8) == out.size
    return out.reshape(-1)


# -- attention ------------------------------------------------------------------------------
def attention(q, K, V, table, P, num_pages, start, base, scale, window=0):
    """q float64 [T, hq, D]; K, V float64 [slots, hkv, D]; base[r]: keys before request r's tokens, or
    None for a failed request.  Returns out, lse and sum_j p_j |v_j| (for the tolerance), float64."""
    T, hq, D = q.shape
    hkv = K.shape[1]
    out, mag = np.zeros((T, hq, D)), np.zeros((T, hq, D))
    lse = np.full((T, hq), -np.inf)
    for r in range(len(start) - 1):
        if base[r] is None:
            continue
        for t in range(start[r], start[r + 1]):
            end = base[r] + t - start[r] + 1
            keys = np.arange(max(0, end - window) if window else 0, end)
            page = table[r][keys // P]
            ok = (page >= 0) & (page < num_pages)
            at = page[ok].astype(np.int64) * P + keys[ok] % P
            if at.size == 0:
                continue
            for h in range(hq):
                x = K[at, h // (hq // hkv)] @ q[t, h] * scale
                m = x.max()
                p = np.exp(x - m)
                out[t, h] = p @ V[at, h // (hq // hkv)] / p.sum()
                mag[t, h] = p @ np.abs(V[at, h // (hq // hkv)]) / p.sum()
                lse[t, h] = m + np.log(p.sum())
    return out, lse, mag
