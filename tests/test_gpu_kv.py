"""The paged 4-bit cache on the GPU: tables, rows in and out, attention, against plain definitions."""
import numpy as np
import pytest

import kv_ref as ref
from gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def _dev(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a))
    return t.to("cuda") if dtype is None else t.to("cuda").to(dtype)


def _i32(a):
    return _dev(np.asarray(a, np.int32))


def _np(t):
    import torch
    torch.cuda.synchronize()
    return t.float().cpu().numpy() if t.dtype == torch.bfloat16 else t.cpu().numpy()


def _cache(**kw):
    from paper_2602_24044_b200.harness import KVCache
    a = dict(num_layers=1, num_pages=64, page_size=16, num_q_heads=8, num_kv_heads=2, head_dim=128)
    a.update(kw)
    return KVCache(**a)


# -- tables ---------------------------------------------------------------------------------
def _table_case(rng, R, P, num_pages, cap, kv_hi, q_hi, count=None):
    kv = rng.integers(0, kv_hi + 1, R)
    q = rng.integers(0, q_hi + 1, R)
    order = rng.permutation(num_pages).astype(np.int32)
    table = np.full((R, cap), -1, np.int32)
    at = 0
    for r in range(R):
        n = min(-(-int(kv[r]) // P), cap)
        table[r, :n] = order[(at + np.arange(n)) % num_pages]
        at += n
    free = np.zeros(num_pages, np.int32)
    left = order[min(at, num_pages):]
    free[: left.size] = left
    return kv.astype(np.int32), q.astype(np.int32), table, free, left.size if count is None else count


@pytest.mark.parametrize("R,P,kv_hi,q_hi,max_q,short", [
    (1, 16, 0, 1, 0, 0), (1, 16, 40, 1, 1, 0), (3, 16, 33, 0, 0, 0), (16, 16, 200, 1, 1, 0), (37, 32, 300, 5, 0, 0),
    (64, 64, 500, 70, 0, 40), (200, 16, 100, 3, 2, 60), (516, 16, 600, 9, 0, 0), (1025, 128, 300, 1, 0, 0),
    (7, 16, 100, 3000, 0, 0), (4096, 16, 20, 2, 0, 100)])
@pytest.mark.parametrize("in_place", [False, True])
def test_tables_match_the_definition(R, P, kv_hi, q_hi, max_q, short, in_place):
    """short: how many pages the stack lacks, so that requests fail."""
    require_gpu()
    rng = np.random.default_rng(R * 1000 + P + q_hi)
    num_pages = sum(-(-(kv_hi + q_hi) // P) for _ in range(R)) + 5
    cap = -(-(kv_hi + q_hi) // P) + 1
    kv, q, table, free, count = _table_case(rng, R, P, num_pages, cap, kv_hi, q_hi)
    if short:
        need = sum(max(0, -(-(int(a) + int(b)) // P) - -(-int(a) // P)) for a, b in zip(kv, q))
        drop = count - max(0, need - short)
        free, count = free[: count], count - drop
        free = np.concatenate([free[:count], np.zeros(num_pages - count, np.int32)])
    T = int(q.sum())
    want = ref.tables(kv, q, T, P, free, count, table, num_pages, max_q)
    with _cache(num_pages=num_pages, page_size=P) as c:
        kv_d, q_d, free_d, cnt_d, tab_d = _i32(kv), _i32(q), _i32(free), _i32([count]), _i32(table)
        kv_o, cnt_o = (kv_d, cnt_d) if in_place else (_i32(kv * 0 - 9), _i32([-9]))
        c.reserve(R, T)
        c.tables.fill_(-77)
        c.build_tables(kv_d, q_d, T, free_d, cnt_d, tab_d, max_q=max_q, kv_len_out=kv_o, free_count_out=cnt_o)
        assert _np(c.header)[:6].tolist() == want["header"]
        assert _np(c.starts).tolist() == want["start"]
        assert _np(c.positions).tolist() == want["position"]
        assert _np(c.slots).tolist() == want["slot"]
        assert _np(c.lengths).tolist() == want["kv_len"] == _np(kv_o).tolist()
        assert np.array_equal(_np(tab_d), want["table"])
        assert _np(cnt_o)[0] == want["free_count"]
        if short:
            assert want["header"][3] > 0        # the case reaches what it is for
        if not in_place:
            assert np.array_equal(_np(kv_d), kv) and _np(cnt_d)[0] == count


@pytest.mark.parametrize("kv,q,T,max_q,cap", [
    ([5, -3, 7], [1, 2, -4], 3, 0, 4),           # negative lengths count as 0
    ([0, 0, 0], [4, 4, 4], 8, 0, 4),             # the last request's tokens pass T
    ([0, 60, 0], [1, 10, 1], 12, 0, 4),          # more pages than the table has
    ([0, 3, 0], [1, 9, 2], 12, 2, 4),            # more tokens than max_q
    ([0, 0], [3, 2], 9, 0, 4),                   # fewer tokens than T
    ([0, 0], [2000000000, 2], 9, 0, 4), ([2147483600, 1], [1, 1], 2, 0, 4),
    ([0], [0], 0, 0, 4), ([], [], 0, 0, 4), ([], [], 5, 0, 4)])
def test_tables_of_odd_batches(kv, q, T, max_q, cap):
    require_gpu()
    R, P, n = len(kv), 16, 40
    table = np.full((R, cap), -1, np.int32)
    for r in range(R):
        table[r, :min(cap, -(-max(kv[r], 0) // P))] = 39 - r
    free = np.arange(n, dtype=np.int32)
    want = ref.tables(kv, q, T, P, free, 30, table, n, max_q)
    with _cache(num_pages=n) as c:
        kv_d, cnt, tab = _i32(np.asarray(kv, np.int64).astype(np.int32)), _i32([30]), _i32(table)
        c.reserve(R, T)
        c.tables.fill_(-77)
        c.build_tables(kv_d, _i32(q), T, _i32(free), cnt, tab, max_q=max_q)
        h = _np(c.header)[:6].tolist()
        assert [h[i] for i in (0, 1, 3, 4, 5)] == [want["header"][i] for i in (0, 1, 3, 4, 5)]
        if sum(max(x, 0) for x in q) <= T:
            assert h[2] == want["header"][2]
        else:
            assert h[2] > T
        assert _np(c.starts).tolist() == want["start"] and _np(c.slots).tolist() == want["slot"]
        assert _np(c.positions).tolist() == want["position"] and _np(kv_d).tolist() == want["kv_len"]
        assert np.array_equal(_np(tab), want["table"]) and _np(cnt)[0] == want["free_count"]


def test_tables_keep_a_slot_out_of_pages_that_do_not_exist():
    require_gpu()
    table = np.array([[999, -1], [3, -1]], np.int32)      # request 0's old page is outside the cache
    with _cache(num_pages=8) as c:
        c.build_tables(_i32([5, 5]), _i32([1, 1]), 2, _i32(np.arange(8)), _i32([2]), _i32(table))
        assert _np(c.slots).tolist() == [-1, 3 * 16 + 5]


@pytest.mark.parametrize("ids", [[2, 0], [1], [0, 1, 2, 3], [3, 3, 9, -1, 1], []])
def test_release_gives_pages_back_in_order(ids):
    require_gpu()
    P, n, lens = 16, 64, [40, 16, 0, 33]
    table = np.full((4, 5), -1, np.int32)
    at = 10
    for r, k in enumerate(lens):
        m = -(-k // P)
        table[r, :m] = np.arange(at, at + m)
        at += m
    free = np.zeros(n, np.int32)
    free[:4] = [50, 51, 52, 53]
    stack, kv, tab, seen = [50, 51, 52, 53], list(lens), table.copy(), set()
    for i in ids:
        if 0 <= i < 4 and i not in seen:
            seen.add(i)
            stack += [int(p) for p in tab[i, : -(-kv[i] // P)]]
            tab[i, : -(-kv[i] // P)] = -1
            kv[i] = 0
    with _cache(num_pages=n) as c:
        kv_d, tab_d, free_d, cnt = _i32(lens), _i32(table), _i32(free), _i32([4])
        c.release(_i32(ids), kv_d, tab_d, free_d, cnt)
        assert _np(cnt)[0] == len(stack) and _np(free_d)[: len(stack)].tolist() == stack
        assert _np(kv_d).tolist() == kv and np.array_equal(_np(tab_d), tab)
        assert c.status()[0] == 0


def test_release_does_not_write_past_the_stack():
    require_gpu()
    table = np.array([[0, 1, 2]], np.int32)
    with _cache(num_pages=8) as c:
        free, cnt = _i32(np.arange(8)), _i32([7])
        c.release(_i32([0]), _i32([48]), _i32(table), free, cnt)
        assert _np(cnt)[0] == 8 and _np(free).tolist() == [0, 1, 2, 3, 4, 5, 6, 0] and c.status()[0] == 2


# -- rows -----------------------------------------------------------------------------------
def _rows(rng, T, n, D, spread=1.0):
    x = rng.standard_normal((T, n * D)) * np.exp(spread * rng.standard_normal((1, n * D)))
    return ref.bf16(x.astype(np.float32))


def _angles(n, rot, theta=10000.0):
    f = theta ** (-np.arange(0, rot, 2) / rot)
    a = np.arange(n)[:, None] * f
    return np.concatenate([np.cos(a), np.sin(a)], -1).astype(np.float32)


def _want_rows(x, D, w, eps, cs, pos, rot, inter, npos):
    """float32 [T, n * D] after norm and rotation, bit for bit."""
    T = x.shape[0]
    y = x.reshape(-1, D)
    if w is not None:
        y = ref.norm32(y, w, eps)
    if cs is not None:
        n = y.shape[0] // T
        ok = np.repeat((pos >= 0) & (pos < npos), n)
        at = np.repeat(np.where((pos >= 0) & (pos < npos), pos, 0), n)
        y = np.where(ok[:, None], ref.rotate(y, cs[at], rot, inter), y)
    return y.reshape(T, -1)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rot,inter", [(0, False), (1, False), (1, True), (16, False), (32, False), (48, False),
                                       (32, True), (48, True)])
@pytest.mark.parametrize("T,hq,hk,norm", [(1, 1, 1, True), (5, 7, 3, True), (33, 32, 8, True), (3, 4, 0, True),
                                          (3, 0, 2, False), (4, 5, 5, False)])
def test_norm_rope_bits(D, rot, inter, T, hq, hk, norm):
    """rot 1: the whole head.  Queries and keys are parts of one fused row, outputs lie in wider rows."""
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    rot = D if rot == 1 else rot
    rng = np.random.default_rng(T * 100 + hq + rot)
    x = _rows(rng, T, hq + 2 * hk, D)
    qw, kw = (ref.bf16(1 + 0.3 * rng.standard_normal(D).astype(np.float32)) for _ in (0, 1))
    pos = rng.integers(0, 50, T).astype(np.int32)
    if T > 2:
        pos[1], pos[2] = 50, -1                     # outside the table: not rotated
    cs = _angles(50, rot) if rot else None
    xd = _dev(x, torch.bfloat16)
    q_out = torch.full((T, hq * D + 24), 7.0, dtype=torch.bfloat16, device="cuda")
    k_out = torch.full((T, hk * D + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    a = lb.qk_args(num_q_heads=hq, num_kv_heads=hk, head_dim=D, q=xd, ldq=x.shape[1], k=xd[:, hq * D:] if hk else None,
                   ldk=x.shape[1], q_weight=_dev(qw, torch.bfloat16) if norm else None,
                   k_weight=_dev(kw, torch.bfloat16) if norm else None, eps=1e-5,
                   cos_sin=_dev(cs) if rot else None, positions=_i32(pos), interleaved=inter,
                   q_out=q_out if hq else None, k_out=k_out if hk else None)
    lb.qk_norm_rope(a, T)
    got_q, got_k = _np(q_out), _np(k_out)
    wq = _want_rows(x[:, :hq * D], D, qw if norm else None, 1e-5, cs, pos, rot, inter, 50)
    wk = _want_rows(x[:, hq * D:(hq + hk) * D], D, kw if norm else None, 1e-5, cs, pos, rot, inter, 50)
    assert np.array_equal(got_q[:, :hq * D], ref.bf16(wq)) and np.array_equal(got_k[:, :hk * D], ref.bf16(wk))
    assert (got_q[:, hq * D:] == 7).all() and (got_k[:, hk * D:] == 7).all()
    # and the definition in 64 bits: half a unit in the last place of the output, and fp32 noise of a
    # handful of operations (2^-20 of the row's largest value)
    y = x[:, :hq * D].astype(np.float64).reshape(-1, D)
    if norm and hq:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + 1e-5) * qw
    if rot and hq:
        ok = np.repeat((pos >= 0) & (pos < 50), hq)
        y = np.where(ok[:, None], ref.rotate(y, cs.astype(np.float64)[np.repeat(pos * ((pos >= 0) & (pos < 50)), hq)], rot, inter), y)
    err = np.abs(got_q[:, :hq * D].reshape(-1, D) - y)
    assert (err <= 2.0 ** -8 * np.abs(y) + 2.0 ** -20 * np.abs(y).max(-1, keepdims=True, initial=0)).all()


def test_norm_rope_in_place_and_special_values():
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    rng = np.random.default_rng(5)
    T, hq, hk, D = 9, 4, 2, 128
    x = _rows(rng, T, hq + 2 * hk, D)
    x[0, :D] = 0                                     # a zero row stays zero
    x[1, 3] = np.inf
    x[2, 5] = np.nan
    x[3, :D] = 3e38                                  # the sum of squares overflows: the row becomes zero
    w = ref.bf16(np.linspace(0.5, 2, D).astype(np.float32))
    pos = np.arange(T, dtype=np.int32)
    cs = _angles(T, D)
    with np.errstate(all="ignore"):
        wq = ref.bf16(_want_rows(x[:, :hq * D], D, w, 1e-6, cs, pos, D, False, T))
        wk = ref.bf16(_want_rows(x[:, hq * D:(hq + hk) * D], D, None, 1e-6, cs, pos, D, False, T))
    xd = _dev(x, torch.bfloat16)
    k = xd[:, hq * D:]
    a = lb.qk_args(num_q_heads=hq, num_kv_heads=hk, head_dim=D, q=xd, ldq=x.shape[1], k=k, ldk=x.shape[1],
                   q_weight=_dev(w, torch.bfloat16), eps=1e-6, cos_sin=_dev(cs), positions=_i32(pos), q_out=xd,
                   ldqo=x.shape[1], k_out=k, ldko=x.shape[1])
    lb.qk_norm_rope(a, T)
    got = _np(xd)
    assert np.array_equal(got[:, :hq * D], wq, equal_nan=True)
    assert np.array_equal(got[:, hq * D:(hq + hk) * D], wk, equal_nan=True)
    assert np.array_equal(got[:, (hq + hk) * D:], x[:, (hq + hk) * D:])


@pytest.mark.parametrize("D,P,hq,hk", [(128, 16, 8, 2), (64, 64, 7, 1), (128, 128, 3, 3), (64, 32, 40, 8)])
@pytest.mark.parametrize("norm,rot", [(True, True), (False, False), (True, False)])
def test_append_and_read_bits(D, P, hq, hk, norm, rot):
    """Codes, scales and lows bit for bit (through the layer's bytes), the rows read back, rows not named
    left alone."""
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    rng = np.random.default_rng(D + P + hq)
    T, n = 45, 6
    x = _rows(rng, T, hq + 2 * hk, D, 0.3)
    vs = (hq + hk) * D
    x[3, vs:vs + D] = 1.5                            # a constant row: scale 0
    x[4, vs:vs + D] = 0
    x[5, vs + 3] = np.inf                            # not finite: the row reads back as NaN
    x[6, vs + 3] = np.nan
    x[7, vs:vs + D] = ref.bf16(np.linspace(-3.3e38, 3.3e38, D).astype(np.float32))   # its range is not finite
    x[8, vs:vs + D] = ref.bf16((rng.standard_normal(D) * 1e-39).astype(np.float32))  # its scale is not normal
    w = ref.bf16(1 + 0.3 * rng.standard_normal(D).astype(np.float32)) if norm else None
    pos = rng.integers(0, 300, T).astype(np.int32)
    cs = _angles(300, D) if rot else None
    slots = rng.permutation(n * P)[:T].astype(np.int32)
    slots[9], slots[10] = -1, n * P                  # not stored; outside the cache
    with np.errstate(all="ignore"):
        k32 = _want_rows(x[:, hq * D:vs], D, w, 1e-6, cs, pos, D, False, 300)
    K = [np.zeros((n * P, hk, D), np.uint8), np.zeros((n * P, hk), np.float32), np.zeros((n * P, hk), np.float32)]
    V = [a.copy() for a in K]
    wk, wv = np.zeros((T, hk * D), np.float32), np.zeros((T, hk * D), np.float32)
    for dst, src, back in ((K, k32, wk), (V, x[:, vs:], wv)):
        c, s, l = ref.quantise(src.reshape(-1, D))
        vals = ref.bf16(ref.dequantise32(c, s, l)).reshape(T, -1)
        for t in range(T):
            if 0 <= slots[t] < n * P:
                for a, b in zip(dst, (c.reshape(T, hk, D), s.reshape(T, hk), l.reshape(T, hk))):
                    a[slots[t]] = b[t]
                back[t] = vals[t]
    want = ref.pack_layer(K, V, n, P, hk, D)
    with _cache(num_layers=2, num_pages=n, page_size=P, num_q_heads=hq if hq % hk == 0 else hk, num_kv_heads=hk,
                head_dim=D) as c:
        c.mem[256:].zero_()
        xd = _dev(x, torch.bfloat16)
        wd = _dev(w, torch.bfloat16) if norm else None
        q_out = torch.empty((T, hq * D), dtype=torch.bfloat16, device="cuda")
        a = lb.qk_args(num_q_heads=hq, num_kv_heads=hk, head_dim=D, q=xd, ldq=x.shape[1], k=xd[:, hq * D:],
                       ldk=x.shape[1], v=xd[:, vs:], ldv=x.shape[1], q_weight=wd, k_weight=wd, eps=1e-6,
                       cos_sin=_dev(cs) if rot else None, positions=_i32(pos), q_out=q_out)
        c.append(1, a, _i32(slots), T)
        assert np.array_equal(_np(c.layer(1)), want)
        assert (_np(c.layer(0)) == 0).all()
        with np.errstate(all="ignore"):
            wq = _want_rows(x[:, :hq * D], D, w, 1e-6, cs, pos, D, False, 300)
        assert np.array_equal(_np(q_out), ref.bf16(wq), equal_nan=True)
        k_out = torch.full((T, hk * D + 8), 7.0, dtype=torch.bfloat16, device="cuda")
        v_out = torch.full((T, hk * D), 7.0, dtype=torch.bfloat16, device="cuda")
        c.read(1, _i32(slots), k_out, v_out)
        assert np.array_equal(_np(k_out)[:, :hk * D], wk, equal_nan=True) and (_np(k_out)[:, hk * D:] == 7).all()
        assert np.array_equal(_np(v_out), wv, equal_nan=True)
        assert c.status()[0] == 1
        # queries left out: the cache is the same
        c.mem[256:].zero_()
        b = lb.qk_args(num_q_heads=0, num_kv_heads=hk, head_dim=D, k=xd[:, hq * D:], ldk=x.shape[1], v=xd[:, vs:],
                       ldv=x.shape[1], k_weight=wd, eps=1e-6, cos_sin=_dev(cs) if rot else None, positions=_i32(pos))
        c.append(1, b, _i32(slots), T)
        assert np.array_equal(_np(c.layer(1)), want)


# -- attention ------------------------------------------------------------------------------
class Batch:
    """A cache filled with random rows and a batch over it, with the definition's answer."""

    def __init__(self, lens, hq, hkv, D, P=16, window=0, seed=0, max_q=0, q_scale=1.0, v_spread=0.5, fail=(),
                 scale=None, pad_tokens=0):
        import torch
        rng = np.random.default_rng(seed)
        self.P, self.D, self.hq, self.hkv, self.window = P, D, hq, hkv, window
        R, T = len(lens), sum(q for _, q in lens) + pad_tokens
        cap = max(-(-(k + q) // P) for k, q in lens) + 1
        n = sum(-(-(k + q) // P) for k, q in lens) + 2
        self.scale = D ** -0.5 if scale is None else scale
        slots = n * P
        k32 = (rng.standard_normal((slots * hkv, D)) * np.exp(0.4 * rng.standard_normal(D))).astype(np.float32)
        v32 = (rng.standard_normal((slots * hkv, D)) *
               np.exp(v_spread * rng.standard_normal((slots * hkv, 1)))).astype(np.float32)
        self.Kq = [a.reshape((slots, hkv) + a.shape[1:]) for a in ref.quantise(k32)]
        self.Vq = [a.reshape((slots, hkv) + a.shape[1:]) for a in ref.quantise(v32)]
        order = rng.permutation(n).astype(np.int32)
        table, at = np.full((R, cap), -1, np.int32), 0
        for r, (k, q) in enumerate(lens):
            m = -(-k // P)
            table[r, :m] = order[at:at + m]
            at += m
        free = np.zeros(n, np.int32)
        free[: n - at] = order[at:]
        kv, q = [k for k, _ in lens], [q for _, q in lens]
        self.want_tables = ref.tables(kv, q, T, P, free, n - at, table, n, max_q)
        self.base = [k if a == k + q else None for (k, q), a in zip(lens, self.want_tables["kv_len"])]
        # rows that no visible token owns were never written
        used = np.zeros(slots, bool)
        for r, end in enumerate(self.want_tables["kv_len"]):
            for j in range(end if self.base[r] is not None else 0):
                used[self.want_tables["table"][r, j // P] * P + j % P] = True
        for a in (self.Kq, self.Vq):
            a[1][~used], a[2][~used] = np.nan, np.nan
            a[0][~used] = 15
        self.q = ref.bf16((q_scale * rng.standard_normal((T, hq * D))).astype(np.float32))
        from paper_2602_24044_b200.harness import KVCache
        self.c = KVCache(1, n, P, hq, hkv, D)
        self.n, self.T = n, T
        self.store()
        self.c.build_tables(_i32(kv), _i32(q), T, _i32(free), _i32([n - at]), _i32(table), max_q=max_q, window=window)
        self.qd = _dev(self.q, torch.bfloat16)

    def store(self):
        self.c.layer(0).copy_(_dev(ref.pack_layer(self.Kq, self.Vq, self.n, self.P, self.hkv, self.D)))

    def values(self):
        out = []
        for c, s, l in (self.Kq, self.Vq):
            out.append(c.astype(np.float64) * s[..., None] + l[..., None])
        return out

    def run(self, stream=None):
        import torch
        out = torch.full((self.T, self.hq * self.D), 777.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((self.T, self.hq), 777.0, dtype=torch.float32, device="cuda")
        torch.cuda.synchronize()
        self.c.attention(0, self.qd, out, scale=self.scale, lse=lse, stream=stream)
        assert self.c.status(stream)[1] == 0
        return _np(out).reshape(self.T, self.hq, self.D), _np(lse)

    def check(self, got=None):
        """Half a unit in the last place of the bf16 output; 2^-11 a probability (fp16) and 2^-12 for the
        exponential and the scores' fp32 sums, on the sum of p |v|; probabilities below fp16's normal range
        are off by 2^-25 of the largest value, one for each key."""
        out, lse = self.run() if got is None else got
        K, V = self.values()
        w = self.want_tables
        want, want_lse, mag = ref.attention(self.q.astype(np.float64).reshape(self.T, self.hq, self.D), K, V, w["table"],
                                            self.P, self.n, w["start"], self.base, self.scale, self.window)
        most = np.nanmax(np.abs(V)) * max([k for k in w["kv_len"]] + [0])
        bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2.0 ** -12) * mag + 2.0 ** -25 * most
        err = np.abs(out - want)
        assert np.isfinite(out).all() and (err <= bound).all(), \
            "worst %.3g times the bound" % np.nanmax(err / np.maximum(bound, 1e-30))
        some = np.isfinite(want_lse)
        assert np.array_equal(np.isneginf(lse), ~some)
        # the scores' fp32 sums: 2^-20 of a score; the sum of probabilities: 2^-20
        assert (np.abs(lse[some] - want_lse[some]) <= 2.0 ** -19 * (np.abs(want_lse[some]) + 8)).all()
        return want


@pytest.mark.parametrize("hq,hkv,D", [(4, 4, 64), (8, 2, 128), (7, 1, 128), (16, 1, 64), (24, 1, 128), (10, 2, 64)])
@pytest.mark.parametrize("P,window", [(16, 0), (64, 0), (32, 20)])
def test_attention_of_single_tokens(hq, hkv, D, P, window):
    require_gpu()
    lens = [(k, 1) for k in (0, 1, 14, 15, 16, 17, 30, 31, 32, 33, 63, 64, 127, 128, 129, 255, 300, 700)]
    Batch(lens, hq, hkv, D, P, window, seed=hq + P, max_q=1).check()


@pytest.mark.parametrize("hq,hkv,D", [(4, 4, 64), (8, 2, 128), (7, 1, 128)])
@pytest.mark.parametrize("P,window", [(16, 0), (128, 0), (32, 50)])
def test_attention_of_mixed_batches(hq, hkv, D, P, window):
    """Prompts with and without a cached part, single tokens, a few tokens at once, idle requests."""
    require_gpu()
    lens = [(0, 1), (5, 0), (40, 3), (0, 70), (100, 33), (0, 257), (77, 1), (300, 128), (31, 2), (0, 16), (250, 65)]
    Batch(lens, hq, hkv, D, P, window, seed=hq + P).check()


@pytest.mark.parametrize("lens", [[(3000, 1)], [(3000, 1), (1, 1), (2500, 1)], [(2000, 300)], [(0, 900)], [(0, 1)]])
@pytest.mark.parametrize("hq,hkv,D", [(2, 1, 128), (4, 1, 64)])
def test_attention_split_along_the_keys(lens, hq, hkv, D):
    require_gpu()
    Batch(lens, hq, hkv, D, 16, seed=len(lens), max_q=max(q for _, q in lens)).check()


@pytest.mark.parametrize("max_q", [0, 2])
def test_failed_requests_and_spare_tokens_give_zeros(max_q):
    """max_q 2: the request of 40 tokens fails; two tokens past the last request."""
    require_gpu()
    b = Batch([(20, 2), (10, 40), (33, 1)], 8, 2, 128, max_q=max_q, pad_tokens=2, seed=3)
    want = b.check()
    assert (want[-2:] == 0).all() and ((want[2:42] == 0).all() == (max_q == 2))


@pytest.mark.parametrize("lens", [[(900, 1), (40, 1)], [(100, 200)]])
def test_values_of_very_different_sizes(lens):
    """Scales of the value rows from 2^-20 to 2^20: what a probability loses below fp16's range is small
    beside the largest value it is added to."""
    require_gpu()
    Batch(lens, 4, 1, 128, v_spread=4.0, seed=9).check()


@pytest.mark.parametrize("lens", [[(500, 1)], [(100, 200)]])
def test_peaked_scores(lens):
    require_gpu()
    Batch(lens, 4, 1, 128, q_scale=12.0, seed=10).check()


@pytest.mark.parametrize("lens,q_scale", [([(300, 1)], 1.0), ([(64, 150)], 1.0)])
def test_huge_and_tiny_values_keep_their_range(lens, q_scale):
    """Values far outside fp16's range: 2^60 and 2^-60 times the usual ones."""
    require_gpu()
    for f in (2.0 ** 60, 2.0 ** -60):
        b = Batch(lens, 4, 1, 128, seed=11)
        want, _ = b.run()
        b.Vq[1], b.Vq[2] = (b.Vq[1] * np.float32(f)).astype(np.float32), (b.Vq[2] * np.float32(f)).astype(np.float32)
        b.store()
        got, _ = b.run()
        assert np.array_equal(got, want * np.float32(f))


@pytest.mark.parametrize("lens", [[(200, 1), (60, 1)], [(64, 150), (0, 90)]])
def test_a_bad_row_reaches_only_those_who_see_it(lens):
    """A key row of NaN, a value row of NaN: the outputs that see it are NaN, the others keep their bits."""
    require_gpu()
    b = Batch(lens, 4, 2, 128, window=40, seed=12)
    want, _ = b.run()
    t = b.want_tables["table"]
    k0, q0 = lens[0]
    for j, kind in ((k0 - 10, b.Kq), (k0 + q0 - 1, b.Vq)):
        slot = t[0, j // 16] * 16 + j % 16
        keep = kind[1][slot, 0], kind[2][slot, 0]
        kind[1][slot, 0] = kind[2][slot, 0] = np.nan
        b.store()
        got, _ = b.run()
        pos = np.array(b.want_tables["position"])
        sees = np.zeros((b.T, 4), bool)
        sees[:q0, :2] = ((pos[:q0] >= j) & (pos[:q0] - 40 < j))[:, None]
        assert np.isnan(got[sees]).all() and sees.any()
        assert np.array_equal(got[~sees], want[~sees])
        kind[1][slot, 0], kind[2][slot, 0] = keep
    b.store()


def test_pages_outside_the_cache_are_not_seen():
    require_gpu()
    for lens in ([(100, 1)], [(50, 130)]):
        b = Batch(lens, 4, 1, 64, seed=13)
        b.c.block_table[0, 1] = 10 ** 6
        b.c.block_table[0, 2] = -5
        b.want_tables["table"][0, 1:3] = -1
        b.check()


def test_attention_bits_repeat_and_do_not_depend_on_the_stream():
    require_gpu()
    import torch
    b = Batch([(700, 1), (0, 300), (3, 1), (1500, 1)], 8, 2, 128, seed=14)
    want, lse = b.run()
    for stream in (None, torch.cuda.Stream(), torch.cuda.Stream()):
        got, l2 = b.run(stream)
        assert np.array_equal(got, want) and np.array_equal(l2, lse)


def test_query_and_output_rows_may_be_parts_of_wider_ones():
    require_gpu()
    import torch
    b = Batch([(70, 1), (0, 200)], 4, 2, 128, seed=15)
    want, _ = b.run()
    wide = torch.full((b.T, 4 * 128 + 2 * 2 * 128), 3.0, dtype=torch.bfloat16, device="cuda")
    wide[:, :512] = b.qd
    out = torch.full((b.T, 512 + 40), 5.0, dtype=torch.bfloat16, device="cuda")
    b.c.attention(0, wide[:, :512], out[:, :512], scale=b.scale)
    got = _np(out)
    assert np.array_equal(got[:, :512].reshape(want.shape), want) and (got[:, 512:] == 5).all()


def test_attention_in_a_graph_follows_the_lengths():
    """The step is captured once; the lengths it works on are read from the device at every replay."""
    require_gpu()
    import torch
    b = Batch([(100, 1), (31, 1), (5, 1)], 4, 1, 128, seed=16, max_q=1)
    kv = _i32([100, 31, 5])
    out = torch.zeros((3, 512), dtype=torch.bfloat16, device="cuda")
    table, free, cnt = b.c.block_table.clone(), _i32([0]), _i32([0])
    s = torch.cuda.Stream()

    def step():
        b.c.build_tables(kv, _i_one, 3, free, cnt, table, max_q=1, kv_len_out=scratch, stream=s)
        b.c.attention(0, b.qd, out, scale=b.scale, stream=s)

    _i_one, scratch = _i32([1, 1, 1]), _i32([0, 0, 0])
    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    want = _np(out).copy()
    assert np.array_equal(want.reshape(3, 4, 128), b.run()[0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        step()
    kv.copy_(_i32([40, 20, 5]))
    g.replay()
    torch.cuda.synchronize()
    shorter = _np(out).copy()
    assert not np.array_equal(shorter[:2], want[:2]) and np.array_equal(shorter[2], want[2])
    kv.copy_(_i32([100, 31, 5]))
    g.replay()
    assert np.array_equal(_np(out), want)


def test_refusals_leave_everything_alone():
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    b = Batch([(20, 1), (3, 2)], 4, 2, 128, seed=17)
    c, q = b.c, b.qd
    out = torch.zeros_like(q)
    before = lb.launch_count()

    def att(**kw):
        a = dict(kv=c.kv, layer=0, q=q, ldq=512, out=out, ldo=512, lse=None, scale=1.0, tables=c.tables, R=2, T=3,
                 block_table=c.block_table, ld_table=c.ld_table, workspace=c.workspace)
        a.update(kw)
        lb.kv_attention(**a)

    for status, kw in [(3, dict(layer=1)), (3, dict(layer=-1)), (1, dict(q=None)), (1, dict(out=None)),
                       (1, dict(tables=None)), (1, dict(block_table=None)), (2, dict(ldq=504)), (2, dict(ldo=516)),
                       (1, dict(q=q.data_ptr() + 2)), (1, dict(out=q)), (1, dict(R=3)), (1, dict(T=2)),
                       (1, dict(workspace=None)), (7, dict(workspace_bytes_=16)), (2, dict(T=-1))]:
        with pytest.raises(lb.LoraError) as e:
            att(**kw)
        assert e.value.status == status, kw
    kv, ql, free, cnt = _i32([20, 3]), _i32([1, 2]), _i32([0, 1]), _i32([2])
    for status, kw in [(7, dict(tables_bytes=64)), (2, dict(R=5000)), (2, dict(T=-1)), (2, dict(window=-1)),
                       (2, dict(max_q=-1)), (1, dict(kv_len=None)), (1, dict(free_pages=None)),
                       (1, dict(block_table=None)), (1, dict(tables=c.tables.data_ptr() + 4, tables_bytes=1 << 20))]:
        a = dict(kv=c.kv, kv_len=kv, q_len=ql, R=2, T=3, free_pages=free, free_count=cnt, block_table=c.block_table,
                 ld_table=c.ld_table, tables=c.tables)
        a.update(kw)
        with pytest.raises(lb.LoraError) as e:
            lb.kv_build_tables(**a)
        assert e.value.status == status, kw
    ok = dict(num_q_heads=4, num_kv_heads=2, head_dim=128, q=q, ldq=512, k=q, ldk=512, v=q, ldv=512, q_out=out)
    for status, layer, kw in [(3, 1, {}), (2, 0, dict(num_kv_heads=1)), (2, 0, dict(num_q_heads=2)),
                              (1, 0, dict(v=None)), (1, 0, dict(q_out=q[:, 8:], ldqo=512)), (1, 0, dict(k_out=out, ldko=512))]:
        with pytest.raises(lb.LoraError) as e:
            lb.kv_append(c.kv, layer, lb.qk_args(**{**ok, **kw}), c.slots, 3)
        assert e.value.status == status, kw
    with pytest.raises(lb.LoraError) as e:
        lb.kv_read(c.kv, 0, c.slots, 3, out, 100, None, 0)
    assert e.value.status == 2
    with pytest.raises(lb.LoraError) as e:
        lb.kv_release(c.kv, kv, 5000, 2, kv, c.block_table, c.ld_table, free, cnt)
    assert e.value.status == 2
    assert lb.launch_count() == before and (_np(out) == 0).all()
    lb.kv_append(c.kv, 0, lb.qk_args(**ok), c.slots, 0)       # nothing to do
    lb.kv_read(c.kv, 0, c.slots, 0, out, 512, None, 0)
    assert lb.launch_count() == before


def test_layer_of_a_served_batch():
    """The example's layer: prompts, then a mixed step, then single tokens; its attention against the definition
    on the rows that its QKV projection (adapters included) gave."""
    require_gpu()
    import sys
    import torch
    import os
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    from attention_step import AttentionLayer
    hq, hkv, d = 8, 2, 128
    layer = AttentionLayer(pages=64, max_positions=256)
    layer.admit(3, 200)
    g = torch.Generator(device="cuda").manual_seed(3)
    owner = torch.tensor([0, 2, -1], dtype=torch.int32, device="cuda")
    K, V = [np.zeros((0, hkv, d)) for _ in range(3)], [np.zeros((0, hkv, d)) for _ in range(3)]
    qw, kw = _np(layer.q_weight), _np(layer.k_weight)
    cs = _np(layer.angles)
    used = 0
    for q_len in ([40, 70, 1], [1, 33, 5], [1, 1, 1], [1, 1, 1]):
        T = sum(q_len)
        x = torch.randn(T, 1024, generator=g, device="cuda").bfloat16()
        ids = torch.repeat_interleave(owner, torch.tensor(q_len, device="cuda"))
        out, attn, qkv = layer.step(x, q_len, ids.contiguous())
        assert torch.isfinite(out).all()
        rows, got = _np(qkv), _np(attn).reshape(T, hq, d)
        t0 = 0
        for r, n in enumerate(q_len):
            pos = np.arange(len(K[r]), len(K[r]) + n)
            part = rows[t0:t0 + n].reshape(n, hq + 2 * hkv, d)
            at = lambda h: cs[np.repeat(pos, h)]      # noqa: E731
            q = ref.bf16(ref.rotate(ref.norm32(part[:, :hq].reshape(-1, d), qw, 1e-6), at(hq), d, False))
            k = ref.rotate(ref.norm32(part[:, hq:hq + hkv].reshape(-1, d), kw, 1e-6), at(hkv), d, False)
            for store, val in ((K, k), (V, part[:, hq + hkv:].reshape(-1, d))):
                c, s, low = ref.quantise(val)
                store[r] = np.concatenate([store[r], (c.astype(np.float64) * s[:, None] + low[:, None]).reshape(n, hkv, d)])
            L = len(K[r])
            want, _, mag = ref.attention(q.astype(np.float64).reshape(n, hq, d), K[r], V[r], np.arange(-(-L // 16))[None],
                                         16, 1 << 20, [0, n], [L - n], d ** -0.5)
            bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2.0 ** -12) * mag + 2.0 ** -25 * np.abs(V[r]).max() * L
            assert (np.abs(got[t0:t0 + n] - want) <= bound).all()
            t0 += n
    used = sum(-(-len(k) // 16) for k in K)
    assert int(layer.free_count) == 64 - used
    layer.release([0, 1, 2])
    assert int(layer.free_count) == 64 and sorted(_np(layer.free).tolist()) == list(range(64))
    assert layer.kv.status()[:2] == [0, 0]
    layer.close()


def test_pages_beyond_four_gigabytes():
    """Byte offsets of pages pass 32 bits: a cache of 4.6 GB of which the last pages are used."""
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    n, P, hkv, D, T = 33000, 128, 8, 128, 300
    rng = np.random.default_rng(21)
    with _cache(num_pages=n, page_size=P, num_q_heads=hkv, num_kv_heads=hkv, head_dim=D) as c:
        assert c.mem.numel() > 1 << 32
        x = ref.bf16(rng.standard_normal((T, 3 * hkv * D)).astype(np.float32))
        xd = _dev(x, torch.bfloat16)
        free, cnt = _i32(np.arange(n)), _i32([n])                     # the stack's top is the last page
        kv, table = _i32([0, 0]), _i32(np.full((2, 4), -1))
        c.build_tables(kv, _i32([T - 1, 1]), T, free, cnt, table)
        assert _np(table)[0, 0] == n - 1 and _np(c.slots).max() == n * P - 1
        q = torch.empty((T, hkv * D), dtype=torch.bfloat16, device="cuda")
        w = 3 * hkv * D
        c.append(0, lb.qk_args(num_q_heads=hkv, num_kv_heads=hkv, head_dim=D, q=xd, ldq=w, k=xd[:, hkv * D:], ldk=w,
                               v=xd[:, 2 * hkv * D:], ldv=w, q_out=q))
        out = torch.empty_like(q)
        c.attention(0, q, out, scale=D ** -0.5)
        got = _np(out).reshape(T, hkv, D)
        vals = []
        for part in (x[:, hkv * D:2 * hkv * D], x[:, 2 * hkv * D:]):
            code, s, low = ref.quantise(part.reshape(-1, D))
            vals.append((code.astype(np.float64) * s[:, None] + low[:, None]).reshape(T, hkv, D))
        back = torch.empty_like(q)
        c.read(0, c.slots, None, back)
        assert np.array_equal(_np(back), ref.bf16(vals[1].astype(np.float32)).reshape(T, -1))
        want, _, mag = ref.attention(x[:, :hkv * D].astype(np.float64).reshape(T, hkv, D), vals[0], vals[1],
                                     np.arange(3)[None], P, 1 << 20, [0, T - 1], [0], D ** -0.5)
        bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2.0 ** -12) * mag + 2.0 ** -25 * np.abs(vals[1]).max() * T
        assert (np.abs(got - want)[:T - 1] <= bound[:T - 1]).all()
        # the request of one token sees itself alone
        assert (np.abs(got[T - 1] - vals[1][T - 1]) <= 2.0 ** -8 * np.abs(vals[1][T - 1]) + 2.0 ** -10 * np.abs(vals[1][T - 1])).all()
        assert c.status()[:2] == [0, 0]


@pytest.mark.parametrize("lens,hq,hkv,P", [
    ([(20000, 1)], 1, 1, 128),                                        # one pair, hundreds of pieces
    ([(9000, 1), (3, 1)], 3, 1, 16),
    ([(k % 37, 1) for k in range(700)], 4, 4, 16),                    # more pairs than warps
    ([(k % 5, 17 + k % 3) for k in range(60)], 4, 2, 16),             # many prompts of one chunk
    ([(0, 0), (0, 0), (5000, 80)], 2, 1, 64), ([(6, 33), (0, 1500)], 1, 1, 32)])
def test_walks_of_every_shape(lens, hq, hkv, P):
    require_gpu()
    Batch(lens, hq, hkv, 64, P, seed=len(lens), max_q=max(q for _, q in lens)).check()


def test_scale_zero_and_negative():
    """scale 0: the mean of the values; a negative scale turns the scores."""
    require_gpu()
    for lens in ([(70, 1)], [(10, 90)]):
        Batch(lens, 4, 2, 128, seed=30, scale=0.0).check()
        Batch(lens, 4, 2, 128, seed=31, scale=-0.1).check()


def test_pieces_behind_a_failed_request_are_joined():
    """A request of 60 tokens fails (max_q 1) and leaves more items than there are requests; the long one behind
    it is cut into pieces all the same."""
    require_gpu()
    Batch([(3, 60), (3000, 1)], 8, 1, 128, max_q=1, seed=40).check()
