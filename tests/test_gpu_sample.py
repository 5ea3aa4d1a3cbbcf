"""Sampling of the next tokens against the definition in 64 bits, row by row."""
import numpy as np
import pytest

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def _reference(x, tau, k, p, mp, u):
    """One row: (token, logprob, distance of u from the nearest border of the kept tokens' sums)."""
    x = np.asarray(x, np.float64)
    if np.isnan(x).any() or not (x > -np.inf).any():
        return -1, np.nan, 1.0
    m = x.max()
    if not tau > 0:
        return int(np.argmax(x)), 0.0, 1.0
    with np.errstate(all="ignore"):
        e = np.where(x == m, 0.0, (x - m) / np.float64(tau))
    e = np.where(x == -np.inf, -np.inf, e)
    w = np.where(e < -46 * np.log(2), 0.0, np.exp(e))
    order = np.lexsort((np.arange(x.size), -x))
    keep = np.zeros(x.size, bool)
    keep[order[:k] if 0 < k < x.size else order] = True
    if mp > 0:
        keep &= e >= np.log(min(np.float64(mp), 1.0))
    if p < 1:
        o = order[keep[order]]
        cum = np.cumsum(w[o])
        n = max(1, int((cum - w[o] < max(np.float64(p), 0.0) * cum[-1]).sum()))
        keep[:] = False
        keep[o[:n]] = True
    w = np.where(keep, w, 0.0)
    cum = np.cumsum(w)
    u = 0.0 if np.isnan(u) else min(max(float(u), 0.0), 1.0)
    at = int(np.searchsorted(cum, u * cum[-1], side="right"))
    last = int(np.flatnonzero(w)[-1])
    at = min(at, last)
    return at, np.log(w[at] / cum[-1]), np.abs(cum / cum[-1] - u).min()


def _run(logits, tau, k=None, p=None, mp=None, u=None, stream=None, R=None):
    import torch
    from paper_2602_24044_b200 import binding as lb
    R = logits.shape[0] if R is None else R

    def dev(a, dtype):
        return None if a is None else torch.as_tensor(np.broadcast_to(np.asarray(a), (R,)).copy()).to(dtype).cuda()

    token = torch.full((R + 2,), -77, dtype=torch.int32, device="cuda")
    logprob = torch.full((R + 2,), 77.0, dtype=torch.float32, device="cuda")
    params = [dev(tau, torch.float32), dev(k, torch.int32), dev(p, torch.float32), dev(mp, torch.float32), dev(u, torch.float32)]
    lb.sample(lb.sample_args(logits=logits, temperature=params[0], top_k=params[1], top_p=params[2], min_p=params[3],
                             uniform=params[4], token=token[1:R + 1], logprob=logprob[1:R + 1]), R, stream=stream)
    torch.cuda.synchronize()
    assert token[0] == token[R + 1] == -77 and logprob[0] == logprob[R + 1] == 77.0
    return token[1:R + 1].cpu().numpy(), logprob[1:R + 1].cpu().numpy()


def _check(logits, tau, k=None, p=None, mp=None, u=None):
    R = logits.shape[0]
    got, lp = _run(logits, tau, k, p, mp, u)
    x = logits.float().cpu().numpy()

    def each(a, none, dtype):
        return np.full(R, none) if a is None else np.broadcast_to(np.asarray(a), (R,)).astype(dtype)

    tau, k, p, mp, u = (each(a, n, t) for a, n, t in ((tau, 1, np.float32), (k, 0, np.int32), (p, 1.0, np.float32),
                                                     (mp, 0.0, np.float32), (u, 0.0, np.float32)))
    for r in range(R):
        want, want_lp, _ = _reference(x[r], tau[r], int(k[r]), p[r], mp[r], u[r])
        assert got[r] == want, (r, got[r], want, tau[r], k[r], p[r], mp[r], u[r])
        # the weight and the sum to 1e-11 each, and one rounding to fp32
        assert (np.isnan(lp[r]) and np.isnan(want_lp)) or abs(lp[r] - want_lp) <= 4e-11 + 2.0 ** -24 * abs(want_lp), (r, lp[r], want_lp)
    return got


def _logits(R, V, seed, bf16=False, spread=2.5, peaks=True, masked=0.0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(R, V, generator=g, device="cuda") * spread
    if peaks:
        at = torch.randint(0, V, (R, min(V, 20)), generator=g, device="cuda")
        x.scatter_add_(1, at, 8 * torch.rand(at.shape, generator=g, device="cuda"))
    if masked:
        x.masked_fill_(torch.rand(R, V, generator=g, device="cuda") < masked, -float("inf"))
        x[:, seed % V] = 1.0
    return x.bfloat16() if bf16 else x


def _params(R, seed, ks, ps, mps):
    rng = np.random.default_rng(seed)
    return dict(tau=rng.choice([0.0, 0.5, 0.8, 1.0, 1.0, 1.7], R), k=rng.choice(ks, R), p=rng.choice(ps, R),
                mp=rng.choice(mps, R), u=rng.random(R).astype(np.float32))


SIZES = [1, 2, 7, 31, 100, 511, 512, 513, 1000, 1025, 4097, 8192, 20000, 32000, 50021, 131072, 200001]


@pytest.mark.parametrize("V", SIZES)
@pytest.mark.parametrize("bf16", [False, True])
def test_mixed_parameters(V, bf16):
    require_gpu()
    R = 40 if V < 10000 else 24
    x = _logits(R, V, V, bf16)
    _check(x, **_params(R, V, [0, 0, 1, 2, 5, 40, 200, 256, 257, 1000], [1.0, 1.0, 0.1, 0.5, 0.9, 0.95, 0.999],
                        [0.0, 0.0, 0.01, 0.2, 1.0]))


@pytest.mark.parametrize("V", SIZES)
@pytest.mark.parametrize("bf16", [False, True])
def test_whole_vocabulary(V, bf16):
    require_gpu()
    R = 30
    x = _logits(R, V, V + 1, bf16, peaks=False)
    rng = np.random.default_rng(V)
    _check(x, rng.choice([0.3, 1.0, 2.0, 30.0], R), u=rng.random(R).astype(np.float32))


@pytest.mark.parametrize("R,V", [(297, 3), (297, 5000), (400, 9001), (592, 2049), (700, 4097), (1300, 777), (300, 60001)])
@pytest.mark.parametrize("bf16", [False, True])
def test_many_rows_without_filters(R, V, bf16):
    """Temperatures of all kinds, and rows that need more than a sum."""
    require_gpu()
    x = _logits(R, V, R + V, bf16)
    inf = float("inf")
    x[0, V // 2], x[1], x[2, V - 1], x[3, 0] = float("nan"), -inf, inf, -inf
    x[4] = x[4] * 0 - 3.0                                    # all equal
    x[5, : V - 1] = -inf
    x[6, V // 3] = 3e38
    x[7] = x[7] * 1e30
    rng = np.random.default_rng(V)
    tau = rng.choice([0.0, 0.3, 1.0, 1.0, 1.0, 5.0], R).astype(np.float32)
    tau[8:14] = [inf, 1e-30, 3e38, float("nan"), -1.0, 1e-42]
    tau[[4, 5, 6, 7]] = [1.0, 0.0, 1.0, 1.0]
    u = rng.random(R).astype(np.float32)
    u[20:24] = [0.0, 1.0, float("nan"), 2.0 ** -40]
    _check(x, tau, u=u)


@pytest.mark.parametrize("R", [1, 2, 5, 37, 74, 75, 148, 149, 297, 600])
@pytest.mark.parametrize("bf16", [False, True])
def test_every_number_of_blocks_a_row(R, bf16):
    require_gpu()
    V = 9001
    x = _logits(R, V, R, bf16)
    _check(x, **_params(R, R, [0, 0, 3, 50, 700], [1.0, 0.9, 0.99], [0.0, 0.0, 0.05]))


@pytest.mark.parametrize("V,k,p,mp", [(50021, 300, 1.0, 0.0), (50021, 5000, 0.98, 0.0), (50021, 50020, 1.0, 0.0),
                                      (50021, 50021, 1.0, 0.0), (50021, 0, 0.999, 0.0), (50021, 0, 0.5, 0.0),
                                      (131072, 20000, 0.9, 1e-6), (131072, 0, 0.97, 1e-4), (3000, 2999, 0.9999, 1e-9),
                                      (600, 599, 1.0, 0.0), (50021, 257, 0.3, 0.0), (50021, 0, 1.0, 1e-5)])
@pytest.mark.parametrize("bf16", [False, True])
def test_what_no_list_holds(V, k, p, mp, bf16):
    require_gpu()
    R = 20
    x = _logits(R, V, V + k, bf16, peaks=False, spread=1.5)
    rng = np.random.default_rng(k)
    _check(x, rng.choice([0.7, 1.0, 2.0], R), k, p, mp, rng.random(R).astype(np.float32))


@pytest.mark.parametrize("R", [3, 700])
@pytest.mark.parametrize("k,p,mp", [(0, 1.0, 0.0), (1, 1.0, 0.0), (7, 1.0, 0.0), (250, 1.0, 0.0), (3000, 1.0, 0.0),
                                    (0, 0.3, 0.0), (40, 0.5, 0.0), (0, 1.0, 1.0), (0, 0.25, 0.5), (4000, 0.7, 0.9)])
@pytest.mark.parametrize("kind", ["equal", "two", "whole", "steps"])
def test_ties_go_to_the_lowest_index(R, k, p, mp, kind):
    """Weights that are exact (1, and 2^-n with the temperature 1 / ln 2 missed by a rounding): many equal values."""
    require_gpu()
    import torch
    V = 6001
    g = torch.Generator(device="cuda").manual_seed(k)
    if kind == "equal":
        x = torch.full((R, V), -3.25, device="cuda")
    elif kind == "two":
        x = torch.where(torch.rand(R, V, generator=g, device="cuda") < 0.4, 2.0, -1.0)
    elif kind == "whole":
        x = torch.randint(-6, 7, (R, V), generator=g, device="cuda").float()
    else:
        x = (torch.arange(V, device="cuda") // 100).float().expand(R, V).contiguous() * 0.25
    u = torch.rand(R, generator=g, device="cuda").cpu().numpy()
    _check(x if k % 2 else x.bfloat16(), 1.0, k, p, mp, u)
    _check(x, 0.0, k, p, mp, u)


@pytest.mark.parametrize("R", [4, 330])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("V,held", [(345, 2), (345, 4), (1024, 1024), (5000, 4096), (40000, 64), (40000, 32768)])
def test_borders_that_fall_together(R, bf16, V, held):
    """Equal logits, a power of two of them, and shares that are whole numbers of them: every sum in question is exact."""
    import torch
    at = np.sort(np.random.default_rng(V + held).permutation(V)[:held])
    x = np.full(V, -np.inf, np.float32)
    x[at] = -1.65625
    logits = torch.as_tensor(x)[None].expand(R, V).to(torch.bfloat16 if bf16 else torch.float32).contiguous().cuda()
    u = np.array([0.0, 0.25, 0.5, 0.75])[np.arange(R) % 4]
    tau = np.array([1.0, 0.7, 1.3])[np.arange(R) % 3]
    for p in (None, 0.5, np.where(np.arange(R) % 2, 0.5, 1.0)):
        kept = held if p is None else np.where(np.broadcast_to(p, R) < 1, held // 2, held)
        for k in (None, 0):
            got, lp = _run(logits, tau, k, p, None, u)
            np.testing.assert_array_equal(got, at[(u * kept).astype(int)])
            np.testing.assert_allclose(lp, np.broadcast_to(-np.log(kept), R), rtol=2.0 ** -24, atol=4e-11)


def test_zeros_of_both_signs_are_one_value():
    require_gpu()
    import torch
    x = torch.tensor([[-0.0, 0.0, -0.0, 0.0, -1.0, -0.0]] * 8, device="cuda")
    got = _check(x, 1.0, 3, 1.0, 0.0, np.linspace(0, 0.99, 8))
    assert set(got.tolist()) == {0, 1, 2}
    assert _check(x, 0.0, u=0.5).tolist() == [0] * 8


@pytest.mark.parametrize("V", [50, 3000, 40000])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("k,p,mp", [(0, 1.0, 0.0), (5, 1.0, 0.0), (0, 0.9, 0.0), (0, 1.0, 0.1), (1000, 0.8, 0.01)])
def test_values_that_are_not_finite(V, bf16, k, p, mp):
    require_gpu()
    import torch
    inf = float("inf")
    x = _logits(12, V, V, bf16)
    x[0, V // 2] = float("nan")
    x[1] = -inf
    x[2, :] = -inf
    x[2, V - 1] = -5.0                                     # one token is left
    x[3, V // 3] = inf
    x[4, [3, V // 2, V - 2]] = inf                         # three share the weight
    x[5, : V - 7] = -inf
    x[6, V // 5] = 3e38
    x[7] = -3e38
    x[8, ::2] = -inf
    x[9, 1] = -float("nan")
    x[10, 10:] = x[10, 10:] * 1e4
    x[11] = 1e-42
    for tau in (1.0, 0.0, 0.01, 50.0):
        _check(x, tau, k, p, mp, np.linspace(0.0, 0.999, 12).astype(np.float32))


@pytest.mark.parametrize("V", [100, 5000])
def test_odd_parameters(V):
    require_gpu()
    nan, inf = float("nan"), float("inf")
    for tau in (-1.0, nan, -inf, inf, 1e-30, 1e-42, 1e30, 3e38, 1e-3, 1e6):
        x = _logits(6, V, 3, masked=0.3)
        u = np.array([0.0, 0.3, 0.6, 0.9, 0.999, 0.5], np.float32)
        for k, p, mp in ((0, 1.0, 0.0), (4, 1.0, 0.0), (0, 0.7, 0.0), (0, 1.0, 0.3), (90, 0.5, 0.2)):
            _check(x, tau, k, p, mp, u)
    x = _logits(9, V, 4)
    one = np.nextafter(np.float32(1), np.float32(0))
    for u in (0.0, one, 1.0, 5.0, -1.0, nan, inf, 2.0 ** -40):
        for k, p, mp in ((0, 1.0, 0.0), (9, 1.0, 0.0), (0, 0.8, 0.0), (0, 1.0, 0.1), (400, 0.99, 0.0)):
            _check(x, 1.0, k, p, mp, u)
    for k in (-5, -2 ** 31, 2 ** 31 - 1, V - 1, V, V + 1):
        _check(x, 1.0, k, None, None, 0.4)
    for p in (0.0, -1.0, nan, 1.5, inf, one, 1e-30):
        _check(x, 1.0, None, p, None, 0.4)
    for mp in (-1.0, nan, 1.0, 2.0, inf, 1e-30, 1e-44):
        _check(x, 1.0, None, None, mp, 0.4)


@pytest.mark.parametrize("bf16", [False, True])
def test_masked_rows(bf16):
    require_gpu()
    for masked in (0.5, 0.99, 0.9999):
        x = _logits(24, 40007, 8, bf16, masked=masked)
        _check(x, **_params(24, 5, [0, 0, 1, 30, 256, 400], [1.0, 0.9, 0.5], [0.0, 0.05]))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("R", [6, 320])
@pytest.mark.parametrize("V", [2500, 4096, 6001, 10000, 33000])
def test_steps_without_a_value(R, V, bf16):
    """Rows that leave some of a block's warps nothing, by their length or by a mask of whole stretches."""
    import torch
    rng = np.random.default_rng(V + R + bf16)
    x = rng.normal(0, 2, (R, V)).astype(np.float32)
    for r in range(R):
        step = 1024 if bf16 else 512
        if r % 3 == 1:
            x[r, :step * (1 + r % 4)] = -np.inf
        elif r % 3 == 2:                               # every other stretch, from the second on
            x[r].reshape(-1)[np.arange(V) // step % 2 == 1] = -np.inf
    logits = torch.as_tensor(x).to(torch.bfloat16 if bf16 else torch.float32).cuda()
    tau = np.where(np.arange(R) % 5 == 0, 0.0, 0.8)
    k = np.array([0, 1, 50, 64, 130, 200, 256])[np.arange(R) % 7]
    p = np.where(np.arange(R) % 2 == 0, 1.0, 0.7)
    _check(logits, tau, k, p, 0.0, rng.random(R))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("V,more,at", [(1000, 24, 0), (1001, 0, 0), (1000, 1, 0), (999, 25, 3), (30001, 7, 1)])
def test_rows_of_any_stride_and_alignment(V, more, at, bf16):
    require_gpu()
    import torch
    wide = torch.full((9, V + more + 8), float("nan"), dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
    flat = wide.view(-1)
    x = _logits(9, V, V, bf16)
    rows = torch.as_strided(flat, (9, V), (V + more, 1), at)
    rows.copy_(x)
    if more:
        rows = torch.as_strided(flat, (9, V), (V + more, 1), at)
    _check(rows, **_params(9, 3, [0, 20, 300], [1.0, 0.9], [0.0, 0.1]))


@pytest.mark.parametrize("R,V,bf16", [(2, 1048568, False), (3, 1048568, True), (1, 700001, True), (300, 300000, True)])
def test_largest_vocabularies(R, V, bf16):
    require_gpu()
    import torch
    x = _logits(min(R, 5), V, R, bf16)
    n = x.shape[0]
    rng = np.random.default_rng(R)
    kw = dict(tau=rng.choice([0.6, 1.0, 1.4], n), k=rng.choice([0, 0, 50, 3000], n), p=rng.choice([1.0, 0.9], n),
              mp=rng.choice([0.0, 0.0, 0.01], n), u=rng.random(n).astype(np.float32))
    want = _check(x, **kw)
    if n < R:        # the same few rows over and over: many blocks' work, few references
        at = np.arange(R) % n
        got, _ = _run(x[torch.as_tensor(at, device="cuda")], **{key: v[at] for key, v in kw.items()})
        assert np.array_equal(got, want[at])


@pytest.mark.parametrize("with_workspace", [False, True])
def test_with_and_without_a_workspace(with_workspace):
    """Rows that no list holds, in a batch that fills the GPU: in one launch, or noted for a second one; twice, as the
    workspace has to be left as it was."""
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    R, V = 320, 20000
    x = _logits(R, V, 1, peaks=False)
    u = torch.rand(R, device="cuda")
    one = torch.ones(R, device="cuda")
    p = torch.where(torch.arange(R, device="cuda") % 3 == 0, 0.95, 1.0)
    token, lp = torch.empty(R, dtype=torch.int32, device="cuda"), torch.empty(R, device="cuda")
    args = lb.sample_args(logits=x, temperature=one, top_p=p, uniform=u, token=token, logprob=lp)
    assert args.workspace
    if not with_workspace:
        args.workspace = None
    before = lb.launch_count()
    for _ in range(2):
        token.fill_(-7)
        lb.sample(args, R, stream=torch.cuda.current_stream())
        torch.cuda.synchronize()
        xs, us, ps = x.cpu().numpy(), u.cpu().numpy(), p.cpu().numpy()
        assert token.tolist() == [_reference(xs[r], 1.0, 0, ps[r], 0.0, us[r])[0] for r in range(R)]
        if with_workspace:
            assert not args.own_workspace[:4].any()
        u.copy_(torch.rand(R, device="cuda"))
    assert lb.launch_count() == before + (4 if with_workspace else 2)


@pytest.mark.parametrize("R,V", [(150, 9001), (297, 20000), (700, 4097)])
def test_second_launch_over_and_over(R, V):
    """Every row is one for the second launch, call behind call with nothing between them: its clusters begin while those
    of the last call end."""
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    x = _logits(R, V, R, peaks=False, spread=0.5)
    tau, p = torch.ones(R, device="cuda"), torch.full((R,), 0.9, device="cuda")
    u = torch.rand(30, R, generator=torch.Generator(device="cuda").manual_seed(V), device="cuda")
    token = torch.full((30, R), -7, dtype=torch.int32, device="cuda")
    work = torch.zeros(lb.sample_workspace_bytes(R) // 4, dtype=torch.int32, device="cuda")
    blocks = [lb.sample_args(logits=x, temperature=tau, top_p=p, uniform=u[i], token=token[i], workspace=work)
              for i in range(30)]
    before = lb.launch_count()
    for b in blocks:
        lb.sample(b, R)
    torch.cuda.synchronize()
    assert lb.launch_count() == before + 60 and not work[:4].any()
    xs, us, got = x.cpu().numpy(), u.cpu().numpy(), token.cpu().numpy()
    for r in range(0, R, 7):
        for i in (0, 14, 29):
            assert got[i, r] == _reference(xs[r], 1.0, 0, np.float32(0.9), 0.0, us[i, r])[0], (i, r)
    assert ((got >= 0) & (got < V)).all()


@pytest.mark.parametrize("R", [20, 150, 290, 600])
@pytest.mark.parametrize("p", [None, 0.05])
@pytest.mark.parametrize("bf16", [False, True])
def test_rows_whose_values_rise(R, p, bf16):
    """What a block's sums are taken against comes from its first steps, and later ones hold far larger values: every row
    is the same one, so that each warp's view of it shows as a row that differs."""
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    V = 60001
    x = torch.linspace(-150, 3, V, device="cuda") + torch.rand(V, generator=torch.Generator(device="cuda").manual_seed(R), device="cuda")
    x = x.bfloat16() if bf16 else x
    want, want_lp, _ = _reference(x.float().cpu().numpy(), 1.0, 0, 1.0 if p is None else np.float32(p), 0.0, 0.375)
    rows, one = x.expand(R, V).contiguous(), torch.ones(R, device="cuda")
    u, share = torch.full((R,), 0.375, device="cuda"), None if p is None else torch.full((R,), p, device="cuda")
    token, lp = torch.empty(20, R, dtype=torch.int32, device="cuda"), torch.empty(20, R, device="cuda")
    for i in range(20):
        lb.sample(lb.sample_args(logits=rows, temperature=one, top_p=share, uniform=u, token=token[i], logprob=lp[i]), R,
                  stream=torch.cuda.current_stream())
    assert (token == want).all() and (lp == lp[0, 0]).all()
    assert abs(float(lp[0, 0]) - want_lp) <= 4e-11 + 2.0 ** -24 * abs(want_lp)


def _same_rows(x, R, tau, p, mp, us, workspace=True):
    """R copies of one row, with the numbers `us` in turn: every token and logprob against the definition."""
    import torch
    from paper_2602_24044_b200 import binding as lb
    rows = x.expand(R, x.shape[0]).contiguous()
    us = np.asarray(us, np.float32)
    u = torch.as_tensor(us[np.arange(R) % len(us)]).cuda()
    token, lp = torch.full((R,), -7, dtype=torch.int32, device="cuda"), torch.empty(R, device="cuda")

    def each(a):
        return None if a is None else torch.full((R,), a, device="cuda")

    args = lb.sample_args(logits=rows, temperature=each(tau), top_p=each(p), min_p=each(mp), uniform=u, token=token, logprob=lp)
    if not workspace:
        args.workspace = None
    lb.sample(args, R, stream=torch.cuda.current_stream())
    got, got_lp, host = token.cpu().numpy(), lp.cpu().numpy(), x.float().cpu().numpy()
    for i, v in enumerate(us):
        want, want_lp, _ = _reference(host, np.float32(tau), 0, 1.0 if p is None else np.float32(p),
                                      0.0 if mp is None else np.float32(mp), v)
        assert (got[i::len(us)] == want).all(), (tau, p, mp, v, got[i::len(us)][:4], want)
        assert (np.abs(got_lp[i::len(us)] - want_lp) <= 4e-11 + 2.0 ** -24 * abs(want_lp)).all(), (tau, p, mp, v)


@pytest.mark.parametrize("V", [262143, 262144, 262208, 300000, 1048568])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("R,workspace", [(1, True), (300, True), (300, False)])
def test_flat_rows_of_large_vocabularies(R, workspace, V, bf16):
    """Rows whose weights add up to 2^18 times the largest and more: equal logits, and ordinary ones at a temperature of 100."""
    require_gpu()
    import torch
    g = torch.Generator(device="cuda").manual_seed(V)
    for tau, x in ((1.0, torch.full((V,), -3.25, device="cuda")), (100.0, 2 * torch.randn(V, generator=g, device="cuda"))):
        for p, mp in ((0.5, None), (0.9, None), (0.9, 0.3)):
            _same_rows(x.bfloat16() if bf16 else x, R, tau, p, mp, [0.05, 0.317, 0.77][:R], workspace)


@pytest.mark.parametrize("bf16", [False, True])
def test_shares_of_many_small_weights(bf16):
    """One token with nearly all the weight, a million others with 10^-12 of it each: top_p ends among them.  A border may
    be taken 2^-34 of the sum too early (top_p) and too late (uniform), which is 50 of these tokens each."""
    require_gpu()
    import torch
    V = 1000003
    x = torch.full((V,), -27.5, device="cuda")
    x[777] = 0.0
    x = x.bfloat16() if bf16 else x
    p, u, w = 1 - 2.0 ** -21, 1 - 2.0 ** -24, np.exp(-27.5)
    kept = np.ceil((p * (1 + (V - 1) * w) - 1) / w)              # of the small ones, by hand: sums one by one would drift
    want = int((u * (1 + kept * w) - 1) / w) + 1
    want_lp = np.log(w / (1 + kept * w))
    got, lp = _run(x.expand(3, V).contiguous(), 1.0, None, p, None, u)
    most = 2 * 2.0 ** -34 / w
    assert (np.abs(got - want) <= most + 2).all(), (got, want, most)
    # the sum of what is kept is 1 and 10^-6 at most, so the tokens more or less do not show in its logarithm
    assert (np.abs(lp - want_lp) <= 2.0 ** -24 * abs(want_lp) + 2 ** -33).all()


@pytest.mark.parametrize("V", [345, 40000])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("R", [4, 320])
@pytest.mark.parametrize("top,ties", [(20.0, 1), (20.0, 3), (-20.0, 2), (1e4, 1), (1e4, 4), (-0.375, 3)])
def test_temperatures_next_to_nothing(R, bf16, V, top, ties):
    """Values next to each other are many powers of two apart: what is not among the largest has no weight."""
    require_gpu()
    import torch
    rng = np.random.default_rng(V + ties)
    x = torch.as_tensor((top - 0.5 - np.abs(rng.normal(0, 3, V))).astype(np.float32)).cuda()
    x = x.bfloat16() if bf16 else x
    x[torch.as_tensor(rng.permutation(V)[:ties]).cuda()] = top
    below = torch.full((), top, dtype=x.dtype).nextafter(torch.full((), -float("inf"), dtype=x.dtype))
    x[int(rng.integers(V // 2))] = float(below)
    for tau in (1e-5, 1e-6, 1e-7, 1e-8, 1e-9, 1e-10, 1e-11, 1e-12):
        for p in (None, 0.6):
            _same_rows(x, R, tau, p, None, [0.0, 0.2, 0.55, 0.9])


@pytest.mark.parametrize("bf16", [False, True])
def test_rows_noted_by_someone_else(bf16):
    """A workspace that was not zeroed names rows of its own, with largest values below theirs: those rows' tokens are
    anything, but tokens, and the other rows' are right."""
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    R, V, odd = 320, 20000, 6
    x = _logits(R, V, 1, bf16, peaks=False)
    one, u = torch.ones(R, device="cuda"), torch.rand(R, device="cuda")
    p = torch.where(torch.arange(R, device="cuda") % 3 == 0, 0.95, 1.0)
    words = np.zeros(lb.sample_workspace_bytes(R) // 4, np.int32)
    words[0] = odd
    noted = words[4:4 + 4 * odd].reshape(odd, 4)
    noted[:, 0] = [0, 1, 2, 3, -5, R]
    noted[:, 1] = np.array([-1000, -3e38, -1, -np.inf, 0, 0], np.float32).view(np.int32)
    noted[:, 2:] = np.array([1.0, np.nan, -5.0, np.inf, 0, 0]).view(np.int32).reshape(odd, 2)
    got = []
    for work in (None, torch.as_tensor(words).cuda()):
        token = torch.full((R,), 0, dtype=torch.int32, device="cuda")
        lb.sample(lb.sample_args(logits=x, temperature=one, top_p=p, uniform=u, token=token, workspace=work), R,
                  stream=torch.cuda.current_stream())
        got.append(token.cpu().numpy())
    assert np.array_equal(got[0][4:], got[1][4:])
    assert ((got[1] >= -1) & (got[1] < V)).all()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("R", [3, 40, 80, 150, 320])
@pytest.mark.parametrize("far", [-895.0, -850.0, -700.0, -300.0, 300.0, 850.0, 895.0, 905.0])
@pytest.mark.parametrize("p", [None, 0.05])
def test_first_steps_without_a_value_and_logits_far_from_zero(R, far, p, bf16):
    """A block's sums are then taken against 1, and the weights lie up to 2^900 below or above that."""
    import torch
    rng = np.random.default_rng(R)
    V, tau = 40000, np.float32(0.75)
    x = (far * np.log(2) * tau + rng.normal(0, 0.5, V)).astype(np.float32)
    x[:V // 2 + 700] = -np.inf
    logits = torch.as_tensor(x).to(torch.bfloat16 if bf16 else torch.float32).cuda()
    _same_rows(logits, R, tau, p, None, [0.03, 0.61, 0.93])


@pytest.mark.parametrize("V", [5470, 40000])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("R", [4, 320])
@pytest.mark.parametrize("k", [1, 2, 256, 257, 513, 3000])
def test_top_k_and_top_p_among_ties(R, bf16, V, k):
    """More equal values than a list holds: top_p cuts what top_k left of them, and leaves out what that did."""
    import torch
    rng = np.random.default_rng(V + k)
    x = np.where(rng.random(V) < 0.8, 2.0, rng.normal(0, 1, V)).astype(np.float32)
    two = np.where(np.arange(V) < 200, 3.0, x)            # a few in front of the ties
    p = np.array([0.5, 0.9, 0.99, 0.99999])[np.arange(R) % 4]
    for row in (x, two, np.full(V, -3.25, np.float32)):
        logits = torch.as_tensor(row.astype(np.float32)).expand(R, V).to(torch.bfloat16 if bf16 else torch.float32).contiguous().cuda()
        few = logits if R < 10 else logits[:20]
        want = _check(few, 0.7, k, p[:len(few)], 0.01, 0.77)
        got, _ = _run(logits, 0.7, k, p, 0.01, 0.77)
        assert np.array_equal(got, np.resize(want[:4], R))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("R", [1, 300])
def test_weights_that_count_as_nothing(R, bf16):
    """A million tokens below 2^-46 (2^-46.2) of one: none of them is ever the next, and what they add to the sum of all is
    no more than 2^-26 of it."""
    require_gpu()
    import torch
    V = 1048568
    x = torch.full((V,), -32.0, device="cuda")
    x[V // 3] = 0.0
    rows = (x.bfloat16() if bf16 else x).expand(R, V).contiguous()
    for p in (None, 0.9, 1 - 2.0 ** -24):
        for u in (0.0, 0.5, 1 - 2.0 ** -24, 1.0):
            got, lp = _run(rows, 1.0, None, p, None, u)
            assert (got == V // 3).all() and (lp <= 0).all() and (lp >= -2.0 ** -26).all(), (p, u, got[0], lp[0])


def test_a_block_made_in_a_capture():
    """Its workspace holds whatever was in that memory until the graph is replayed: calls outside of the graph, in another
    graph and on other streams are right before that too."""
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    R, V = 320, 20000
    x = _logits(R, V, 1, peaks=False)
    kw = dict(logits=x, temperature=torch.ones(R, device="cuda"), uniform=torch.rand(R, device="cuda"),
              top_p=torch.where(torch.arange(R, device="cuda") % 3 == 0, 0.95, 1.0))
    want, token = (torch.empty(R, dtype=torch.int32, device="cuda") for _ in range(2))
    lb.sample(lb.sample_args(token=want, **kw), R, stream=torch.cuda.current_stream())
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    with torch.cuda.graph(graphs[0]):
        args = lb.sample_args(token=token, **kw)
        lb.sample(args, R, stream=torch.cuda.current_stream())
    with torch.cuda.graph(graphs[1]):
        lb.sample(args, R, stream=torch.cuda.current_stream())
    side = torch.cuda.Stream()
    calls = [lambda: lb.sample(args, R), lambda: lb.sample(args, R, stream=torch.cuda.current_stream()),
             lambda: lb.sample(args, R, stream=side), lambda: lb.sample(args, R, stream=side.cuda_stream),
             lambda: lb.sample(args, R, stream=0), graphs[1].replay, graphs[0].replay, graphs[1].replay]
    for call in calls:
        args.own_workspace.fill_(1 << 20)
        token.fill_(-7)
        torch.cuda.synchronize()
        call()
        torch.cuda.synchronize()
        assert torch.equal(token, want)


def test_a_graph_follows_its_inputs():
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    R, V = 20, 12345
    x, u = _logits(R, V, 0), torch.rand(R, device="cuda")
    tau, k = torch.full((R,), 0.9, device="cuda"), torch.full((R,), 30, dtype=torch.int32, device="cuda")
    k[::3] = 0
    token, lp = torch.empty(R, dtype=torch.int32, device="cuda"), torch.empty(R, device="cuda")
    args = lb.sample_args(logits=x, temperature=tau, top_k=k, uniform=u, token=token, logprob=lp)
    lb.sample(args, R)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    before = lb.launch_count()
    with torch.cuda.graph(graph):
        lb.sample(args, R, stream=torch.cuda.current_stream())
    assert lb.launch_count() == before + 1
    for seed in range(3):
        x.copy_(_logits(R, V, seed))
        u.uniform_()
        graph.replay()
        torch.cuda.synchronize()
        xs, us, ks = x.cpu().numpy(), u.cpu().numpy(), k.cpu().numpy()
        assert token.tolist() == [_reference(xs[r], np.float32(0.9), int(ks[r]), 1.0, 0.0, us[r])[0] for r in range(R)]
    # on another stream, twice at once, without logprobs, and fewer rows than there are
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = [torch.full((R,), -77, dtype=torch.int32, device="cuda") for _ in side]
    torch.cuda.synchronize()
    for s, o in zip(side, outs):
        lb.sample(lb.sample_args(logits=x, temperature=tau, top_k=k, uniform=u, token=o), R - 1, stream=s)
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o[:-1], token[:-1]) and o[-1] == -77


def test_shares_of_the_tokens():
    """Ten thousand even numbers over one row: each token as often as its weight says, to one."""
    require_gpu()
    import torch
    R, V = 10000, 17
    x = torch.linspace(-2, 1, V, device="cuda").repeat(R, 1)
    u = (np.arange(R) + 0.5) / R
    got, _ = _run(x, 0.7, u=u)
    p = torch.softmax(x[0].double() / np.float32(0.7).astype(np.float64), 0).cpu().numpy()
    assert (np.abs(np.bincount(got, minlength=V) - p * R) <= 1).all()
