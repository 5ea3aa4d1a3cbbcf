"""The paged 4-bit cache on the GPU at its edges: several handles at once, tables in turn, streams, probabilities
far below the largest, bad pages and scales, groups of every size, batches of many rows."""
import numpy as np
import pytest

import kv_ref as ref
from gpu_util import require_gpu
from test_gpu_kv import Batch, _angles, _cache, _dev, _i32, _np

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("large,small", [(2000, 3), (100, 16)])
def test_two_caches_build_tables_in_turn(large, small):
    """A cache that has built small tables does not take from another what its large ones need."""
    require_gpu()

    def build(c, R):
        kv, q = np.arange(R) % 31, np.ones(R, int)
        table = np.zeros((R, 3), np.int32)
        c.build_tables(_i32(kv), _i32(q), R, _i32(np.arange(64)), _i32([0]), _i32(table))
        return _np(c.slots).tolist(), ref.tables(kv, q, R, 16, np.arange(64), 0, table, 64)["slot"]

    with _cache() as a, _cache() as b:
        for c, R in ((a, large), (b, small), (a, large), (b, large), (a, small), (b, large)):
            got, want = build(c, R)
            assert got == want, (R, c is a)


def test_an_error_is_reported_once():
    """A call that the CUDA runtime refused does not leave its error for the next call, which has nothing to do
    with it."""
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    x = torch.ones((3, 128), dtype=torch.bfloat16, device="cuda")
    out = torch.zeros_like(x)
    kw = dict(num_q_heads=2, num_kv_heads=0, head_dim=64, q=x, ldq=128, q_out=out, eps=1e-6)
    buf = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    shape = dict(num_layers=1, num_pages=4, page_size=16, num_q_heads=2, num_kv_heads=2, head_dim=64)
    for _ in range(2):
        with pytest.raises(lb.LoraError) as e:
            lb.kv_create(**shape, device_buf=buf, device=99)
        assert e.value.status == 9
        lb.qk_norm_rope(lb.qk_args(**kw), 3)
    assert torch.equal(out, x)


def test_a_device_that_is_not_there_runs_nothing():
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    x = torch.ones((3, 128), dtype=torch.bfloat16, device="cuda")
    out = torch.zeros_like(x)
    before = lb.launch_count()
    args = lb.qk_args(num_q_heads=2, num_kv_heads=0, head_dim=64, q=x, ldq=128, q_out=out)
    args.device = 99
    with pytest.raises(lb.LoraError) as e:
        lb.qk_norm_rope(args, 3)
    assert e.value.status == 9 and lb.launch_count() == before and (_np(out) == 0).all()


def _sink(hq, hkv, D, R, kv, q_len, bits, seed, mean=0.5):
    """R requests that share one cached prefix of kv keys (the last page of each is its own), whose first key, with
    a value of zero, has a score `bits` binades above the others.  So long a walk that a span holds whole requests.
    Returns outputs, the definition's in 64 bits, sum_j p_j |v_j|, and the largest scale and value."""
    import torch
    rng = np.random.default_rng(seed)
    P = 16
    shared = kv // P
    own = -(-(kv + q_len) // P) - shared
    n = shared + R * own
    slots = n * P
    k32 = rng.standard_normal((slots, hkv, D)).astype(np.float32)
    v32 = (mean + rng.standard_normal((slots, hkv, D)) * np.exp(0.5 * rng.standard_normal((slots, hkv, 1)))).astype(np.float32)
    k32[..., 0] = 0
    k32[0] = 0
    k32[0, :, 0] = bits * np.log(2.0) * D ** 0.5 / 4
    v32[0] = 0
    Kq, Vq = ([a.reshape((slots, hkv) + a.shape[1:]) for a in ref.quantise(x.reshape(-1, D))] for x in (k32, v32))
    table = np.concatenate([np.tile(np.arange(shared), (R, 1)), shared + np.arange(R * own).reshape(R, own)], 1).astype(np.int32)
    T = R * q_len
    q = (0.3 * rng.standard_normal((T, hq, D))).astype(np.float32)
    q[..., 0] = 4
    q = ref.bf16(q)
    with _cache(num_pages=n, num_q_heads=hq, num_kv_heads=hkv, head_dim=D) as c:
        c.layer(0).copy_(_dev(ref.pack_layer(Kq, Vq, n, P, hkv, D)))
        # the table holds its last pages already: the stack hands out the same ones
        have = _i32(np.full(R, kv))
        full = _i32(table)
        new = table[:, shared + (kv % P > 0):].reshape(-1)
        free, cnt = _i32(np.append(new[::-1], 0)), _i32([new.size])
        c.build_tables(have, _i32(np.full(R, q_len)), T, free, cnt, full, max_q=q_len)
        assert np.array_equal(_np(full), table)
        qd = _dev(q.reshape(T, hq * D), torch.bfloat16)
        out = torch.empty_like(qd)
        c.attention(0, qd, out, scale=D ** -0.5)
        assert c.status()[1] == 0
        got = out.double().view(R, q_len, hkv, hq // hkv, D)
    K, V = (_dev(a.astype(np.float64) * s[..., None].astype(np.float64) + l[..., None].astype(np.float64)) for a, s, l in (Kq, Vq))
    want, mag = torch.empty_like(got), torch.empty_like(got)
    limit = kv + torch.arange(q_len, device="cuda") + 1
    for r in range(R):
        at = (full[r].long()[:, None] * P + torch.arange(P, device="cuda")).view(-1)[: kv + q_len]
        x = torch.einsum("qhgd,khd->qhgk", qd.double().view(R, q_len, hkv, hq // hkv, D)[r], K[at]) * D ** -0.5
        x.masked_fill_((torch.arange(kv + q_len, device="cuda") >= limit[:, None])[:, None, None], -float("inf"))
        p = torch.softmax(x, -1)
        want[r], mag[r] = torch.einsum("qhgk,khd->qhgd", p, V[at]), torch.einsum("qhgk,khd->qhgd", p, V[at].abs())
    return got, want, mag, float(np.max(Vq[1])), float(V.abs().max())


@pytest.mark.parametrize("D,hq,hkv", [(64, 8, 8), (128, 64, 4)])
def test_single_tokens_beside_a_key_far_above_the_others(D, hq, hkv):
    """p s is rounded to 11 bits, or to 2^-33 of the largest p times the largest s where that is more (half of it off
    at most); a value is at most 24 times its row's scale here (low between -24 and 8 scales).  With the output's own
    rounding and 2^-12 for exponentials and sums."""
    require_gpu()
    kv = 8191
    got, want, mag, s_max, _ = _sink(hq, hkv, D, 300 * 8 // hkv, kv, 1, 22, D)
    bound = 2.0 ** -8 * want.abs() + (2.0 ** -11 + 2.0 ** -12) * mag + (kv + 1) * 2.0 ** -34 * s_max * 24
    worst = float(((got - want).abs() / bound).max())
    assert worst <= 1, "worst %.3g times the bound" % worst


@pytest.mark.parametrize("D,hq,hkv", [(64, 4, 4), (128, 8, 2)])
def test_prompts_beside_a_key_far_above_the_others(D, hq, hkv):
    """Probabilities are rounded to 11 bits, or to 2^-33 of the largest where that is more (half of it off at most);
    values to 11 bits."""
    require_gpu()
    kv = 8190
    got, want, mag, _, v_max = _sink(hq, hkv, D, 160 // hkv, kv, 70, 25.5, D + 1)
    bound = 2.0 ** -8 * want.abs() + (2.0 ** -11 + 2.0 ** -12) * mag + (kv + 70) * 2.0 ** -34 * v_max
    worst = float(((got - want).abs() / bound).max())
    assert worst <= 1, "worst %.3g times the bound" % worst


@pytest.mark.parametrize("D", [64, 128])
def test_prompt_values_keep_eleven_bits_when_small_beside_their_scale(D):
    """Rows whose low value is a small fraction of the scale: their smallest elements are rounded as such and not
    as parts of the row's middle, which is hundreds of times larger."""
    require_gpu()
    b = Batch([(0, 90), (3, 70)], 2, 1, D, seed=50)
    rng = np.random.default_rng(51)
    written = np.isfinite(b.Vq[1])
    b.Vq[1] = np.where(written, np.float32(1), b.Vq[1])
    b.Vq[2] = np.where(written, ref.bf16(rng.uniform(0.005, 0.06, b.Vq[2].shape).astype(np.float32)), b.Vq[2])
    b.store()
    got = b.run()
    b.check(got)
    # the first token of a prompt sees itself alone: its values, rounded to 11 bits and then to 8
    t = b.want_tables["slot"][0]
    v = b.values()[1][t, 0]
    assert (b.Vq[0][t, 0] == 0).any()
    assert (np.abs(got[0][0] - v) <= (2.0 ** -11 + 2.0 ** -8) * 1.001 * np.abs(v)).all()


def test_memory_that_a_side_stream_still_reads_is_not_handed_out():
    """Work on a side stream is pending when the tables grow, and when the cache goes: what is allocated next does
    not get their memory."""
    require_gpu()
    import torch
    side, inputs = torch.cuda.Stream(), []
    c = _cache()

    def build(R):
        a = [_i32(v) for v in (np.zeros(R), np.ones(R), np.arange(64), [64], np.full((R, 1), -1))]
        inputs.append(a)
        c.build_tables(a[0], a[1], R, a[2], a[3], a[4], max_q=1, stream=side)

    def place(t):
        return t.data_ptr(), t.numel(), t.dtype

    def handed_out(at, n, dtype):
        return any(t.data_ptr() == at for t in [torch.empty(n, dtype=dtype, device="cuda") for _ in range(4)])

    c.reserve(1, 1)
    build(1)
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)       # about 0.2 s
    old = place(c.tables)
    build(60)
    reused = [handed_out(*old)]
    old = place(c.buf), place(c.workspace)
    del c
    reused += [handed_out(*p) for p in old]
    pending = not side.query()
    torch.cuda.synchronize()
    assert pending and not any(reused)


def test_tokens_whose_page_is_outside_the_cache_are_counted():
    """Word 0 of the status tells of a page that a block table or the stack should not hold, where a new token
    goes: once a token, and not for tokens that fail."""
    require_gpu()
    table = np.array([[999, -1], [3, -1], [-7, -1], [998, -1]], np.int32)
    with _cache(num_pages=8) as c:
        c.build_tables(_i32([5, 5, 14, 9]), _i32([1, 1, 2, 9]), 13, _i32([4, 5, 6, 7]), _i32([4]), _i32(table), max_q=4)
        assert c.status()[0] == 1 + 2
        c.build_tables(_i32([16]), _i32([3]), 3, _i32([77]), _i32([1]), _i32([[2, -1]]))
        assert c.status()[0] == 3 + 3


def test_pages_that_no_query_sees_are_not_counted():
    """Behind the window, past the end and of failed requests: pages that are not there are nobody's mistake."""
    require_gpu()
    for lens, window in (([(200, 1)], 20), ([(300, 70)], 33)):
        b = Batch(lens, 4, 1, 64, window=window, seed=14)
        want, _ = b.run()
        first = (lens[0][0] + 1 - window) // 16
        b.c.block_table[0, :first] = -1
        b.want_tables["table"][0, :first] = -1
        assert np.array_equal(b.check(), b.check()) and np.array_equal(b.run()[0], want)
        assert b.c.status()[0] == 0
    b = Batch([(20, 2), (10, 40), (33, 1)], 8, 2, 128, max_q=2, pad_tokens=2, seed=15)
    b.check()
    assert b.c.status()[0] == 0


def test_tables_written_again_are_not_the_oldest():
    """A handle knows the last 256 buffers that it wrote tables to: one that was written first, and again just
    now, is among them when the 257th comes."""
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    with _cache(num_pages=4, num_q_heads=1, num_kv_heads=1, head_dim=64) as c:
        c.mem[256:].zero_()
        n = lb.kv_tables_bytes(c.kv, 1, 1)
        bufs = torch.zeros((257, (n + 15) // 16 * 4), dtype=torch.int32, device="cuda")
        kv, q, free, cnt, table = _i32([3]), _i32([1]), _i32([0]), _i32([0]), _i32([[0]])

        def build(i):
            lb.kv_build_tables(c.kv, kv, q, 1, 1, free, cnt, table, 1, bufs[i], max_q=1)

        x = torch.zeros((1, 64), dtype=torch.bfloat16, device="cuda")
        out = torch.empty_like(x)

        def attend(i):
            lb.kv_attention(c.kv, 0, x, 64, out, 64, None, 1.0, bufs[i], 1, 1, table, 1, c.workspace)

        for i in range(256):
            build(i)
        build(0)
        build(256)
        attend(0)
        attend(256)
        with pytest.raises(lb.LoraError) as e:       # the oldest now
            attend(1)
        assert e.value.status == 1
        attend(2)


def test_a_scale_that_is_no_number_is_refused():
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    b = Batch([(20, 1)], 4, 2, 128, seed=17)
    out = torch.zeros_like(b.qd)
    before = lb.launch_count()
    for scale in (float("nan"), float("inf"), -float("inf"), 3e38):
        with pytest.raises(lb.LoraError) as e:
            b.c.attention(0, b.qd, out, scale=scale)
        assert e.value.status == 1
    assert lb.launch_count() == before and (_np(out) == 0).all()


@pytest.mark.parametrize("lens", [[(70, 1)], [(10, 90)]])
def test_scale_zero_with_huge_keys(lens):
    """scale 0 is the mean of the values, however large the keys are."""
    require_gpu()
    b = Batch(lens, 4, 2, 128, seed=18, scale=0.0)
    for i in (1, 2):
        b.Kq[i] = (b.Kq[i] * np.float32(2.0 ** 110)).astype(np.float32)
    b.store()
    b.check()


def test_queries_and_outputs_may_be_parts_of_the_same_rows():
    """Rows of one pitch that lie beside each other do not overlap; those that do are refused."""
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    b = Batch([(70, 1), (0, 200)], 4, 2, 128, seed=19)
    want, _ = b.run()
    wide = torch.full((b.T, 2 * 512 + 24), 3.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 16:528] = b.qd
    b.c.attention(0, wide[:, 16:528], wide[:, 528:1040], scale=b.scale)
    got = _np(wide)
    assert np.array_equal(got[:, 528:1040].reshape(want.shape), want)
    assert np.array_equal(got[:, 16:528], b.q) and (got[:, :16] == 3).all() and (got[:, 1040:] == 3).all()
    for q, out in ((wide[:, :512], wide[:, 504:1016]), (wide[:, 512:1024], wide[:, 8:520]), (wide[:, 8:520], wide[:, 8:520])):
        with pytest.raises(lb.LoraError) as e:
            b.c.attention(0, q, out, scale=b.scale)
        assert e.value.status == 1


@pytest.mark.parametrize("hq,hkv,D", [(16, 1, 128), (24, 2, 64), (20, 1, 64), (128, 1, 64)])
@pytest.mark.parametrize("P,window", [(16, 0), (32, 21)])
def test_attention_of_mixed_batches_in_wide_groups(hq, hkv, D, P, window):
    """More than eight query heads share keys: items of sixteen rows that span tokens, and prompts."""
    require_gpu()
    lens = [(0, 1), (5, 0), (40, 3), (0, 19), (100, 5), (0, 41), (77, 1), (130, 2), (31, 4), (60, 1)]
    Batch(lens, hq, hkv, D, P, window, seed=hq + P).check()


@pytest.mark.parametrize("hq,hkv,D", [(72, 1, 128), (130, 2, 64), (128, 1, 64), (9, 1, 128)])
def test_attention_of_single_tokens_in_wide_groups(hq, hkv, D):
    """Above 64 query heads a key/value head one token alone is a prompt's tile."""
    require_gpu()
    lens = [(k, 1) for k in (0, 1, 15, 16, 31, 33, 127, 128, 129, 300)]
    Batch(lens, hq, hkv, D, seed=hq, max_q=1).check()


@pytest.mark.parametrize("hq", [16, 72])
@pytest.mark.parametrize("max_q", [0, 2])
def test_failed_requests_and_spare_tokens_in_wide_groups(hq, max_q):
    require_gpu()
    b = Batch([(20, 2), (10, 40), (33, 1)], hq, 1, 64, max_q=max_q, pad_tokens=3, seed=4)
    want = b.check()
    assert (want[-3:] == 0).all() and ((want[2:42] == 0).all() == (max_q == 2))


@pytest.mark.parametrize("D,hq,hk", [(128, 30, 5), (64, 45, 9)])
@pytest.mark.parametrize("rot,inter", [(0, False), (1, False), (32, False), (48, True)])
def test_many_rows_are_the_same_as_few(D, hq, hk, rot, inter):
    """Batches that are large enough for a warp to take several passes of heads: bit for bit what calls of 250
    tokens give, and a sample of rows against the definition; with and without the cache."""
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    rot = D if rot == 1 else rot
    per = 512 // D
    T = 32768 // -(-(hq + hk) // per) + 7          # the first count, with a margin, at which passes are put together
    rng = np.random.default_rng(D + rot)
    n_pages = -(-T // 16) + 1
    g = torch.Generator(device="cuda").manual_seed(D + rot)
    x = torch.randn(T, (hq + 2 * hk) * D, generator=g, device="cuda").mul_(
        torch.rand((hq + 2 * hk) * D, generator=g, device="cuda") + 0.5).bfloat16()
    w = ref.bf16(1 + 0.3 * rng.standard_normal(D).astype(np.float32))
    wd = _dev(w, torch.bfloat16)
    pos = rng.integers(-1, 301, T).astype(np.int32)       # -1 and 300 are outside the table
    slots = rng.permutation(n_pages * 16)[:T].astype(np.int32)
    pos_d, slots_d, cs = _i32(pos), _i32(slots), _angles(300, rot) if rot else None
    cs_d = _dev(cs) if rot else None
    ld = x.stride(0)

    def args(a, b, q_out, k_out):
        return lb.qk_args(num_q_heads=hq, num_kv_heads=hk, head_dim=D, q=x[a:b], ldq=ld, k=x[a:b, hq * D:], ldk=ld,
                          v=x[a:b, (hq + hk) * D:], ldv=ld, q_weight=wd, k_weight=wd, eps=1e-6, cos_sin=cs_d,
                          positions=pos_d[a:b], interleaved=inter, q_out=q_out[a:b], k_out=k_out[a:b])

    def outputs():
        return (torch.full((T, hq * D + 8), 7.0, dtype=torch.bfloat16, device="cuda"),
                torch.full((T, hk * D), 7.0, dtype=torch.bfloat16, device="cuda"))

    pieces = [(a, min(a + 250, T)) for a in range(0, T, 250)]
    one, few = outputs(), outputs()
    lb.qk_norm_rope(args(0, T, *one), T)
    for a, b in pieces:
        lb.qk_norm_rope(args(a, b, *few), b - a)
    assert all(torch.equal(p, q) for p, q in zip(one, few))
    sample = np.unique(np.concatenate([np.arange(0, T, 61), [T - 1]]))
    rows = _np(x[_dev(sample)])

    def want(part):
        y = ref.norm32(part.reshape(-1, D), w, 1e-6)
        if rot:
            p = np.repeat(pos[sample], y.shape[0] // sample.size)
            ok = (p >= 0) & (p < 300)
            y = np.where(ok[:, None], ref.rotate(y, cs[np.where(ok, p, 0)], rot, inter), y)
        return y.reshape(sample.size, -1)

    wq, wk = want(rows[:, :hq * D]), want(rows[:, hq * D:(hq + hk) * D])
    assert np.array_equal(_np(one[0])[sample, :hq * D], ref.bf16(wq)) and (_np(one[0])[:, hq * D:] == 7).all()
    assert np.array_equal(_np(one[1])[sample], ref.bf16(wk))
    with _cache(num_pages=n_pages, num_q_heads=hq, num_kv_heads=hk, head_dim=D) as c:
        bytes_ = []
        for calls in ([(0, T)], pieces):
            c.mem[256:].zero_()
            out = outputs()
            for a, b in calls:
                lb.kv_append(c.kv, 0, args(a, b, *out), slots_d[a:b], b - a)
            assert all(torch.equal(p, q) for p, q in zip(one, out))
            bytes_.append(c.layer(0).clone())
        assert torch.equal(*bytes_)
        back = torch.empty((2, sample.size, hk * D), dtype=torch.bfloat16, device="cuda")
        c.read(0, _i32(slots[sample]), back[0], back[1])
        for got, val in zip(_np(back), (wk, rows[:, (hq + hk) * D:])):
            assert np.array_equal(got, ref.bf16(ref.dequantise32(*ref.quantise(val.reshape(-1, D)))).reshape(got.shape))
        if rot:
            assert c.status()[0] == 2 * int(((pos < 0) | (pos >= 300)).sum())


@pytest.mark.parametrize("D,hq,hkv,kv,q_len,R", [
    (64, 8, 8, 16383, 1, 600), (128, 16, 4, 16383, 1, 1200), (64, 8, 8, 131071, 1, 256), (64, 4, 4, 16382, 70, 160)])
def test_long_flat_sums_are_as_exact_as_their_rounding(D, hq, hkv, kv, q_len, R):
    """Tens of thousands of keys of about the same weight in one span, values around zero: the error is that of
    rounding the output to bf16.  (Probabilities of 11 bits, 2^-12 off as a rule, and fp32 sums are less than a third
    of that each; a tenth is added for both.)"""
    require_gpu()
    got, want, _, _, _ = _sink(hq, hkv, D, R, kv, q_len, 0, 7 + D, mean=0.0)
    rounding = want.bfloat16().double() - want
    ratio = float((got - want).norm() / rounding.norm())
    assert ratio <= 1.1, "%.3g times the rounding alone" % ratio
