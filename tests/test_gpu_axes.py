"""Positions on several axes, and rotation by them: against plain loops, bit for bit."""
import numpy as np
import pytest

import kv_ref as ref
from gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def _dev(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).to("cuda")
    return t if dtype is None else t.to(dtype)


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


# -- positions ------------------------------------------------------------------------------
def _by_hand(mine, p):
    """A request's media [(first, frames, rows, columns, step)], token p: walked through one by one."""
    at = end = 0
    for first, f, h, w, step in mine:
        if p < first:
            break
        at += first - end
        k = p - first
        if k < f * h * w:
            return at + k // (h * w) * step, at + k // w % h, at + k % w
        end = first + f * h * w
        at += max((f - 1) * step + 1, h, w)
    return (at + p - end,) * 3


def _media(rng, tokens, most):
    out, at = [], 0
    for _ in range(int(rng.integers(0, most + 1))):
        at += int(rng.integers(0, 9))
        f, h, w, step = (int(v) for v in (rng.integers(1, 4), rng.integers(1, 6), rng.integers(1, 6), rng.integers(0, 4)))
        if at > tokens:
            break
        out.append((at, f, h, w, step))
        at += f * h * w
    return out


@pytest.mark.parametrize("R,kv_hi,q_hi,most,spare", [
    (1, 0, 1, 0, 0), (1, 0, 40, 3, 0), (3, 60, 1, 4, 2), (17, 100, 30, 6, 0), (300, 50, 1, 3, 0), (9, 0, 700, 60, 5),
    (5, 200, 0, 4, 3), (1100, 30, 2, 2, 1), (4096, 20, 1, 1, 0)])
def test_positions(R, kv_hi, q_hi, most, spare):
    require_gpu()
    import torch
    from paper_2602_24044_b200.harness import media_spans
    rng = np.random.default_rng(R + q_hi)
    kv, q = rng.integers(0, kv_hi + 1, R), rng.integers(0 if R > 1 else q_hi, q_hi + 1, R)
    media = [_media(rng, int(a + b), most) for a, b in zip(kv, q)]
    T = int(q.sum()) + spare
    spans, begin = media_spans(media)
    pages = int(sum(-(-(a + b) // 16) for a, b in zip(kv, q))) + 4
    with _cache(num_pages=pages) as c:
        out = torch.full((4, T + 5), -77, dtype=torch.int32, device="cuda")
        if T:
            c.build_tables(_i32(kv), _i32(q), T, _i32(np.arange(pages)), _i32([pages]),
                           _i32(np.zeros((R, (kv_hi + q_hi) // 16 + 1))))
            c.axis_positions(_i32(spans), _i32(begin), out[:, :T])
        got = _np(out)
    want = [_by_hand(m, int(a) + i) for m, a, n in zip(media, kv, q) for i in range(n)] + [(0, 0, 0)] * spare
    assert got[:3, :T].T.tolist() == [list(w) for w in want]
    assert (got[3] == -77).all() and (got[:, T:] == -77).all()


def test_positions_of_failed_requests_odd_spans_and_offsets():
    """Requests without pages still have positions; spans without tokens, far positions; offsets that lie
    outside the spans are taken to their ends."""
    require_gpu()
    import torch
    kv, q = [0, 2_000_000_000, 5], [3, 4, 1000]
    spans = np.array([(1, 0, 0, 0, 50, 1, 0, 0), (1_999_999_000, 1, 100, 100, 7, 1, 0, 0),
                      (2_000_000_001, 3, 1, 1, 9, 1_000_000, 0, 0), (0, 2, 50_000, 60_000, 0, 3, 0, 0)], np.int32)
    T = sum(q)
    with _cache(num_pages=8) as c:
        c.build_tables(_i32(kv), _i32(q), T, _i32(np.arange(8)), _i32([8]), _i32(np.zeros((3, 4))))
        out = torch.zeros((3, T), dtype=torch.int32, device="cuda")
        c.axis_positions(_i32(spans), _i32([-5, 1, 3, 99]), out)
        got = _np(out)
        assert _np(c.header)[3] >= 2
    assert got[:, 0].tolist() == [0, 0, 0] and got[:, 1:3].tolist() == [[50, 51]] * 3
    assert got[:, 3].tolist() == [7, 7 + 10, 7 + 0]                     # token 1000 of a grid of 100 x 100
    assert got[:, 4:7].tolist() == [[9, 1_000_009, 2_000_009], [9, 9, 9], [9, 9, 9]]
    p = np.arange(5, 1005)                                             # a grid with more cells than 32 bits count
    assert np.array_equal(got[:, 7:], np.stack([p * 0, p * 0, p]))


def test_positions_refusals_leave_everything_alone():
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    out = torch.full((3, 8), -7, dtype=torch.int32, device="cuda")
    spans, begin = _i32(np.zeros((2, 8))), _i32([0, 1, 2])
    with _cache(num_pages=8) as c:
        with pytest.raises(ValueError):
            c.axis_positions(spans, begin, out)                         # no tables yet
        c.build_tables(_i32([0, 0]), _i32([3, 5]), 8, _i32(np.arange(8)), _i32([8]), _i32(np.zeros((2, 1))))
        before = lb.launch_count()
        for bad in (dict(out=out[:2]), dict(out=out[:, :7]), dict(out=out[:1].expand(3, 8)), dict(out=out.t()), dict(out=out[0]),
                    dict(out=out.float()), dict(spans=spans[:, :7]), dict(spans=spans.long()), dict(spans=spans.view(-1)),
                    dict(begin=begin[:2]), dict(begin=begin.float())):
            a = dict(dict(spans=spans, begin=begin, out=out), **bad)
            with pytest.raises(ValueError):
                c.axis_positions(a["spans"], a["begin"], a["out"])
        for (tables, R, T, sp, be, n, to, ld), status in (
                ((c.tables, 2, 7, spans, begin, 2, out, 8), 1), ((c.tables, 3, 8, spans, begin, 2, out, 8), 1),
                ((out, 2, 8, spans, begin, 2, out, 8), 1), ((c.tables, 2, 8, spans, None, 2, out, 8), 1),
                ((c.tables, 2, 8, None, begin, 2, out, 8), 1), ((c.tables, 2, 8, spans, begin, 2, None, 8), 1),
                ((c.tables, 2, 8, spans, begin, 2, out, 7), 2), ((c.tables, 2, 8, spans, begin, -1, out, 8), 2),
                ((c.tables, 2, -1, spans, begin, 2, out, 8), 2),
                ((c.tables, 2, 8, spans.data_ptr() + 4, begin, 1, out, 8), 1)):
            with pytest.raises(lb.LoraError) as e:
                lb.kv_axis_positions(c.kv, tables, R, T, sp, be, n, to, ld)
            assert e.value.status == status
        assert lb.launch_count() == before and (out == -7).all()
        c.axis_positions(spans[:0], _i32([0, 0, 0]), out)               # no media at all
        assert _np(out).tolist() == [[0, 1, 2, 0, 1, 2, 3, 4]] * 3


def test_positions_feed_a_captured_step():
    require_gpu()
    import torch
    from paper_2602_24044_b200.harness import media_spans
    media = [[(2, 1, 3, 4, 1)], [], [(0, 2, 2, 2, 2), (20, 1, 5, 5, 1)]]
    spans, begin = (_i32(a) for a in media_spans(media))
    kv, one = _i32([5, 0, 18]), _i32([1, 1, 1])
    with _cache(num_pages=32) as c:
        c.reserve(3, 3)
        free, count, table = _i32(np.arange(32)), _i32([32]), _i32(np.zeros((3, 8)))
        out = torch.zeros((3, 3), dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s = torch.cuda.current_stream()
            c.build_tables(kv, one, 3, free, count, table, max_q=1, stream=s)
            c.axis_positions(spans, begin, out, stream=s)
        for i in range(6):
            graph.replay()
            want = [_by_hand(m, a + i) for m, a in zip(media, (5, 0, 18))]
            assert _np(out).T.tolist() == [list(w) for w in want]


# -- rotation -------------------------------------------------------------------------------
def _angles(n, rot, theta=10000.0):
    f = theta ** (-np.arange(0, rot, 2) / rot)
    a = np.arange(n)[:, None] * f
    return np.concatenate([np.cos(a), np.sin(a)], -1).astype(np.float32)


def _turned_by(cs, axis, pos):
    """[T, rot]: each pair's cosine and sine from its axis' row."""
    half = cs.shape[1] // 2
    rows = cs[pos]                                                     # [axes, T, rot]
    p = np.arange(half)
    return np.concatenate([rows[axis, :, p].T, rows[axis, :, half + p].T], -1)


@pytest.mark.parametrize("D,rot,inter", [(128, 128, False), (128, 128, True), (128, 64, False), (128, 16, False),
                                         (128, 48, True), (64, 64, False), (64, 64, True), (64, 32, False)])
@pytest.mark.parametrize("T,hq,hk,axes,norm", [(1, 1, 1, 3, True), (5, 7, 3, 2, True), (33, 32, 8, 3, True),
                                               (4, 40, 2, 4, False), (3, 4, 0, 3, True), (3, 0, 5, 1, True),
                                               (1700, 32, 8, 3, True), (2100, 28, 4, 4, False)])
def test_rotation_bits(D, rot, inter, T, hq, hk, axes, norm):
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    rng = np.random.default_rng(T + D + rot + axes)
    x = ref.bf16(rng.standard_normal((T, (hq + hk) * D)).astype(np.float32))
    w = [ref.bf16((1 + 0.3 * rng.standard_normal(D)).astype(np.float32)) for _ in range(2)]
    npos = 61
    cs, axis = _angles(npos, rot), rng.integers(0, axes, rot // 2)
    pos = rng.integers(0, npos, (axes, T)).astype(np.int32)
    if T > 2:
        pos[axes - 1, 1], pos[0, 2] = -1, npos                          # tokens that are not rotated
    xd, posd = _dev(x, torch.bfloat16), torch.zeros((axes, T + 3), dtype=torch.int32, device="cuda")
    posd[:, :T] = _i32(pos)
    q_out = torch.full((T, max(hq, 1) * D), 3e38, dtype=torch.bfloat16, device="cuda")
    k_out = torch.full((T, max(hk, 1) * D), 3e38, dtype=torch.bfloat16, device="cuda")
    wd = [_dev(v, torch.bfloat16) if norm else None for v in w]
    args = lb.qk_args(num_q_heads=hq, num_kv_heads=hk, head_dim=D, q=xd, ldq=x.shape[1], k=xd[:, hq * D:], ldk=x.shape[1],
                      q_weight=wd[0], k_weight=wd[1], eps=1e-6, cos_sin=_dev(cs), interleaved=inter, positions=posd[:, :T],
                      axis_of_pair=axis, q_out=q_out, k_out=k_out)
    lb.qk_norm_rope(args, T)
    turn = ((pos >= 0) & (pos < npos)).all(0)
    row = _turned_by(cs, axis, np.where(turn, pos, 0))
    for out, first, n, wt in ((q_out, 0, hq, w[0]), (k_out, hq, hk, w[1])):
        if not n:
            continue
        v = x[:, first * D:(first + n) * D].reshape(-1, D)
        y = ref.norm32(v, wt, 1e-6) if norm else v
        y = np.where(np.repeat(turn, n)[:, None], ref.rotate(y, np.repeat(row, n, 0), rot, inter), y)
        assert np.array_equal(_np(out).reshape(-1, D), ref.bf16(y))


@pytest.mark.parametrize("D,rot,inter", [(128, 128, False), (64, 32, False), (64, 64, True)])
@pytest.mark.parametrize("T", [3, 2000])
def test_equal_positions_are_one_position(D, rot, inter, T):
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    rng = np.random.default_rng(T)
    hq, hk = 32, 8
    x = _dev(rng.standard_normal((T, (hq + hk) * D)).astype(np.float32), torch.bfloat16)
    cs, one = _dev(_angles(50, rot)), _i32(rng.integers(0, 50, T))
    outs = []
    for positions, axis in ((one, None), (one.repeat(3, 1), rng.integers(0, 3, rot // 2))):
        q, k = (torch.empty((T, n * D), dtype=torch.bfloat16, device="cuda") for n in (hq, hk))
        lb.qk_norm_rope(lb.qk_args(num_q_heads=hq, num_kv_heads=hk, head_dim=D, q=x, ldq=x.stride(0), k=x[:, hq * D:],
                                   ldk=x.stride(0), cos_sin=cs, interleaved=inter, positions=positions, axis_of_pair=axis,
                                   q_out=q, k_out=k), T)
        outs.append((q, k))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


@pytest.mark.parametrize("D,P,hq,hk,T", [(128, 16, 8, 2, 7), (64, 64, 7, 1, 40), (128, 32, 32, 8, 1500)])
@pytest.mark.parametrize("inter", [False, True])
def test_append_bits(D, P, hq, hk, T, inter):
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    rng = np.random.default_rng(T + D)
    pages = -(-T // P) + 2
    width = (hq + 2 * hk) * D
    x = ref.bf16(rng.standard_normal((T, width)).astype(np.float32))
    kw = ref.bf16((1 + 0.3 * rng.standard_normal(D)).astype(np.float32))
    cs, axis = _angles(40, D), rng.integers(0, 3, D // 2)
    pos = rng.integers(0, 40, (3, T)).astype(np.int32)
    pos[2, T // 2] = 40                                                 # not rotated, and counted
    slots = rng.permutation(pages * P)[:T].astype(np.int32)
    slots[0] = -1
    xd = _dev(x, torch.bfloat16)
    with _cache(num_pages=pages, page_size=P, num_q_heads=hq, num_kv_heads=hk, head_dim=D) as c:
        c.mem.fill_(0)
        q_out = torch.empty((T, hq * D), dtype=torch.bfloat16, device="cuda")
        args = lb.qk_args(num_q_heads=hq, num_kv_heads=hk, head_dim=D, q=xd, ldq=width, k=xd[:, hq * D:], ldk=width,
                          v=xd[:, (hq + hk) * D:], ldv=width, k_weight=_dev(kw, torch.bfloat16), eps=1e-6,
                          cos_sin=_dev(cs), interleaved=inter, positions=_i32(pos), axis_of_pair=axis, q_out=q_out)
        c.append(0, args, _i32(slots), T)
        turn = (pos < 40).all(0)
        row = _turned_by(cs, axis, np.where(turn, pos, 0))

        def rotated(y, n):
            return np.where(np.repeat(turn, n)[:, None], ref.rotate(y, np.repeat(row, n, 0), D, inter), y)

        qv = x[:, :hq * D].reshape(-1, D)
        assert np.array_equal(_np(q_out).reshape(-1, D), ref.bf16(rotated(qv, hq)))
        k = rotated(ref.norm32(x[:, hq * D:(hq + hk) * D].reshape(-1, D), kw, 1e-6), hk)
        v = x[:, (hq + hk) * D:].reshape(-1, D)
        stored = []
        for val in (k, v):
            code, s, low = ref.quantise(val)
            all_c, all_s, all_l = np.zeros((pages * P, hk, D), np.uint8), np.zeros((pages * P, hk), np.float32), np.zeros((pages * P, hk), np.float32)
            all_c[slots[1:]], all_s[slots[1:]], all_l[slots[1:]] = (a.reshape(T, hk, *a.shape[1:])[1:] for a in (code, s, low))
            stored.append((all_c, all_s, all_l))
        assert np.array_equal(_np(c.layer(0)), ref.pack_layer(stored[0], stored[1], pages, P, hk, D))
        assert c.status()[0] == 1


@pytest.mark.parametrize("D,P,hq,hk,T,rot", [(128, 16, 8, 2, 7, 64), (128, 32, 32, 8, 1500, 32), (64, 64, 7, 1, 40, 16),
                                             (64, 16, 48, 16, 900, 32), (128, 16, 1, 1, 3, 112)])
@pytest.mark.parametrize("inter", [False, True])
def test_append_of_heads_rotated_in_part(D, P, hq, hk, T, rot, inter):
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    rng = np.random.default_rng(T + D + rot)
    pages = -(-T // P) + 2
    width = (hq + 2 * hk) * D
    x = ref.bf16(rng.standard_normal((T, width)).astype(np.float32))
    w = [ref.bf16((1 + 0.3 * rng.standard_normal(D)).astype(np.float32)) for _ in range(2)]
    cs, axis = _angles(40, rot), rng.integers(0, 3, rot // 2)
    pos = rng.integers(0, 40, (3, T)).astype(np.int32)
    pos[1, T // 2] = -1                                                 # not rotated, and counted
    slots = rng.permutation(pages * P)[:T].astype(np.int32)
    xd = _dev(x, torch.bfloat16)
    with _cache(num_pages=pages, page_size=P, num_q_heads=hq, num_kv_heads=hk, head_dim=D) as c:
        q_out, k_out, k_back, v_back = (torch.empty((T, n * D), dtype=torch.bfloat16, device="cuda") for n in (hq, hk, hk, hk))
        args = lb.qk_args(num_q_heads=hq, num_kv_heads=hk, head_dim=D, q=xd, ldq=width, k=xd[:, hq * D:], ldk=width,
                          v=xd[:, (hq + hk) * D:], ldv=width, q_weight=_dev(w[0], torch.bfloat16),
                          k_weight=_dev(w[1], torch.bfloat16), eps=1e-6, cos_sin=_dev(cs), interleaved=inter,
                          positions=_i32(pos), axis_of_pair=axis, q_out=q_out, k_out=k_out)
        c.append(0, args, _i32(slots), T)
        lb.kv_read(c.kv, 0, _i32(slots), T, k_back, hk * D, v_back, hk * D)
        turn = (pos >= 0).all(0)
        row = _turned_by(cs, axis, np.where(turn, pos, 0))
        k = None
        for out, first, n, wt in ((q_out, 0, hq, w[0]), (k_out, hq, hk, w[1])):
            y = ref.norm32(x[:, first * D:(first + n) * D].reshape(-1, D), wt, 1e-6)
            k = np.where(np.repeat(turn, n)[:, None], ref.rotate(y, np.repeat(row, n, 0), rot, inter), y)
            assert np.array_equal(_np(out).reshape(-1, D), ref.bf16(k))
        for back, val in ((k_back, k), (v_back, x[:, (hq + hk) * D:].reshape(-1, D))):
            code, scale, low = ref.quantise(val)
            want = ref.bf16(np.float32(low)[:, None] + np.float32(scale)[:, None] * code.astype(np.float32))
            assert np.array_equal(_np(back).reshape(-1, D), want)
        assert c.status()[0] == 1


def test_rotation_in_place_and_on_another_stream():
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    rng = np.random.default_rng(2)
    T, hq, hk, D = 64, 8, 2, 128
    x = _dev(rng.standard_normal((T, (hq + hk) * D)).astype(np.float32), torch.bfloat16)
    pos, cs, axis = _i32(rng.integers(0, 30, (3, T))), _dev(_angles(30, D)), [0, 1, 2, 1] * 16
    kw = dict(num_q_heads=hq, num_kv_heads=hk, head_dim=D, cos_sin=cs, positions=pos, axis_of_pair=axis)
    q, k = (torch.empty((T, n * D), dtype=torch.bfloat16, device="cuda") for n in (hq, hk))
    lb.qk_norm_rope(lb.qk_args(q=x, ldq=x.stride(0), k=x[:, hq * D:], ldk=x.stride(0), q_out=q, k_out=k, **kw), T)
    want = torch.cat([q, k], 1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    args = lb.qk_args(q=x, ldq=x.stride(0), k=x[:, hq * D:], ldk=x.stride(0), q_out=x, ldqo=x.stride(0), k_out=x[:, hq * D:],
                      ldko=x.stride(0), **kw)
    lb.qk_norm_rope(args, T, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(x, want)
