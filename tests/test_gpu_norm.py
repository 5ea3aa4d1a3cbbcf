"""Residual addition and norm of rows against the definition in 64 bits, codes against the same operations
on the host in 32 bits (they have to be equal)."""
import numpy as np
import pytest

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu

F32 = np.float32


def _tensors(T, n, residual, seed, ld_more=0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)

    def rows(scale):
        wide = torch.randn(T, n + ld_more, generator=g, device="cuda") * scale
        return wide.bfloat16()[:, :n]

    x = rows(0.5)
    r = rows(3.0) if residual else None
    w = (1 + 0.3 * torch.randn(n, generator=g, device="cuda")).bfloat16()
    return x, r, w


def _filled(shape, dtype):
    """Outputs start as bytes that no result has: a value left unwritten cannot pass."""
    import torch
    t = torch.empty(shape, dtype=dtype, device="cuda")
    t.view(torch.uint8).fill_(0x7D)
    return t


def _rows64(x, r, w, eps):
    s = x.double() if r is None else x.double() + r.double()
    y = s / (s.pow(2).mean(-1, keepdim=True) + eps).sqrt()
    return s, y if w is None else y * w.double()


def _codes32(x, r, w, eps, group):
    """The operations of the definition, each rounded to fp32 by itself: (codes as float32 values, scales)."""
    import torch
    s = x.float().cpu().numpy()
    if r is not None:
        s = s + r.float().cpu().numpy()
    T, n = s.shape
    with np.errstate(all="ignore"):
        q = s * s
        p = [q[:, i::8] for i in range(8)]
        tree = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]))
        total = tree.astype(np.float64).sum(-1).astype(F32)
        inv_norm = F32(1) / np.sqrt(total * F32(1.0 / n) + F32(eps))
        y = s * inv_norm[:, None]
        if w is not None:
            y = y * w.float().cpu().numpy()
        z = y.reshape(T, -1, group)
        top = np.abs(z).max(-1)
        bad = ~np.isfinite(top)
        if group == 32:
            m, e = np.frexp(top.astype(np.float64))
            e = np.clip(e - 9 + (m > 0.875), -127, 127)
            scales = np.where(bad, 255, np.where(top == 0, 0, e + 127)).astype(np.uint8)
            inv = np.where(top == 0, 1.0, np.exp2(-e.astype(np.float64))).astype(F32)
        else:
            scales = top * F32(1.0 / 448.0)
            scales = np.where(scales < F32(1.17549435e-38), F32(0), scales)
            scales = np.where(bad, F32(np.nan), scales)
            inv = np.where(scales == 0, F32(0), F32(1) / scales)
        c = np.where(bad[..., None], F32(0), z * inv[..., None]).astype(F32).reshape(T, n)
    return torch.from_numpy(c).to(torch.float8_e4m3fn).float(), torch.from_numpy(scales)


SHAPES = [(1, 8), (3, 64), (2, 256), (5, 1000), (9, 1032), (40, 128), (4, 4096), (33, 4104), (7, 14336), (2, 8192),
          (2, 32768), (3, 16416), (700, 4096), (5000, 96), (260, 14336), (600, 1032)]


@pytest.mark.parametrize("T,n", SHAPES)
@pytest.mark.parametrize("residual", [False, True])
def test_rows(T, n, residual):
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    x, r, w = _tensors(T, n, residual, T * 7 + n)
    w = None if (T + n) % 3 == 0 else w
    out = _filled((T, n), torch.bfloat16)
    r_out = _filled((T, n), torch.bfloat16) if residual else None
    dev = torch.cuda.current_device()
    lb.add_norm(lb.norm_args(x=x, weight=w, eps=1e-5, residual=r, residual_out=r_out, out=out, device=dev), T)
    s, y = _rows64(x, r, w, 1e-5)
    # half a bf16 step, and in fp32: the sum, three roundings of the squares' tree (halved by the root), the
    # total, mean, eps, root, reciprocal and two products, 2^-24 each
    assert ((out.double() - y).abs() <= y.abs() * (2.0 ** -8 + 10 * 2.0 ** -24)).all()
    if residual:
        assert torch.equal(r_out, (x.float() + r.float()).bfloat16())


@pytest.mark.parametrize("group,T,n", [
    (32, 3, 32), (32, 4, 4096), (32, 5, 1056), (32, 2, 32768), (32, 700, 4096), (32, 3000, 96),
    (128, 3, 128), (128, 4, 4096), (128, 3, 1152), (128, 2, 32768), (128, 700, 4096), (128, 900, 384), (128, 60, 14336),
    (0, 3, 8), (0, 4, 4096), (0, 3, 1000), (0, 2, 32768), (0, 700, 4096), (0, 900, 400), (0, 60, 14336), (0, 3, 8200)])
def test_codes_are_equal_and_near(group, T, n):
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    x, r, w = _tensors(T, n, True, T + 3 * n + group)
    if T > 2:
        x[1], r[1] = 0, 0                                   # a row of zeros
        r[2, : n // 2] = -x[2, : n // 2]                    # groups of zeros in a row that has others
    g = group or n
    codes = _filled((T, n), torch.float8_e4m3fn)
    scales = _filled((T, n // g), torch.uint8 if g == 32 else torch.float32)
    out, r_out = _filled((T, n), torch.bfloat16), _filled((T, n), torch.bfloat16)
    dev = torch.cuda.current_device()
    lb.add_norm(lb.norm_args(x=x, weight=w, eps=1e-6, residual=r, residual_out=r_out, out=out, codes=codes,
                             scales=scales, group=g, device=dev), T)
    c, s = _codes32(x, r, w, 1e-6, g)
    assert torch.equal(scales.cpu(), s)
    assert torch.equal(codes.float().cpu(), c)
    _, y = _rows64(x, r, w, 1e-6)
    step = torch.exp2(s.double() - 127).cuda() if g == 32 else s.double().cuda()
    z = y.view(T, -1, g)
    back = codes.double().view(T, -1, g) * step[..., None]
    # half an e4m3 step: 2^-4 of the value, below 2^-6 of the scale half of 2^-9 of it; and fp32's roundings
    assert ((back - z).abs() <= z.abs() * (2.0 ** -4 + 2.0 ** -19) + step[..., None] * (2.0 ** -10 + 2.0 ** -19)).all()
    assert torch.equal(r_out, (x.float() + r.float()).bfloat16())
    assert ((out.double() - y).abs() <= y.abs() * (2.0 ** -8 + 10 * 2.0 ** -24)).all()
    # the same codes without the other outputs
    again = _filled((T, n), torch.float8_e4m3fn)
    lb.add_norm(lb.norm_args(x=x, weight=w, eps=1e-6, residual=r, codes=again, scales=scales, group=g, device=dev), T)
    assert torch.equal(again.view(torch.uint8), codes.view(torch.uint8)) and torch.equal(scales.cpu(), s)


@pytest.mark.parametrize("T,n", [(5, 512), (300, 4096)])
def test_parts_of_wider_rows_and_outputs_in_place(T, n):
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    dev = torch.cuda.current_device()
    x, r, w = _tensors(T, n, True, 5, ld_more=24)
    want_y, want_r = torch.empty(T, n, dtype=torch.bfloat16, device="cuda"), torch.empty_like(r.contiguous())
    lb.add_norm(lb.norm_args(x=x, weight=w, residual=r, residual_out=want_r, out=want_y, device=dev), T)
    s, y = _rows64(x, r, w, 1e-6)
    assert ((want_y.double() - y).abs() <= y.abs() * (2.0 ** -8 + 10 * 2.0 ** -24)).all()
    # outputs as parts of one wider row, with what lies between left as it was
    wide = _filled((T, 2 * n + 64), torch.bfloat16)
    was = wide.clone()
    lb.add_norm(lb.norm_args(x=x, weight=w, residual=r, residual_out=wide[:, 8:8 + n], out=wide[:, n + 40:2 * n + 40],
                             device=dev), T)
    assert torch.equal(wide[:, 8:8 + n], want_r) and torch.equal(wide[:, n + 40:2 * n + 40], want_y)
    for a, b in ((0, 8), (8 + n, n + 40), (2 * n + 40, 2 * n + 64)):
        assert torch.equal(wide[:, a:b], was[:, a:b])
    # the stream in place, the norm over x
    lb.add_norm(lb.norm_args(x=x, weight=w, residual=r, residual_out=r, out=x, device=dev), T)
    assert torch.equal(r, want_r) and torch.equal(x, want_y)


def test_rows_that_are_not_finite_stay_alone():
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    dev = torch.cuda.current_device()
    T, n = 6, 1024
    for g in (32, 128, n):
        x, r, w = _tensors(T, n, True, 9)
        x[1, 5], x[3, 77], r[4, 1000] = float("nan"), float("inf"), float("-inf")
        w[200] = float("inf")                               # one channel whose weight is not finite
        codes, out = _filled((T, n), torch.float8_e4m3fn), _filled((T, n), torch.bfloat16)
        scales = _filled((T, n // g), torch.uint8 if g == 32 else torch.float32)
        lb.add_norm(lb.norm_args(x=x, weight=w, residual=r, out=out, codes=codes, scales=scales, group=g, device=dev), T)
        c, s = _codes32(x, r, w, 1e-6, g)
        assert torch.equal(scales.cpu().float().nan_to_num(-1.0), s.float().nan_to_num(-1.0))
        assert torch.equal(codes.float().cpu(), c)
        assert torch.isfinite(out[[0, 2, 5]][:, :200]).all() and torch.isfinite(out[[0, 2, 5]][:, 201:]).all()
        assert not torch.isfinite(out[[0, 2, 5]][:, 200]).any() and torch.isnan(out[1]).all()
        bad = (s == 255) if g == 32 else torch.isnan(s)
        assert bad[1].all() and bad[0].any() and (g == n or not bad[0].all())


@pytest.mark.parametrize("size", [1e-30, 1e-19, 1e18, 3e38])
def test_sizes_of_values(size):
    """Squares that vanish or overflow: the formula in fp32 says what comes out."""
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    dev = torch.cuda.current_device()
    x = (torch.rand(4, 256, device="cuda") + 0.5).mul_(size).bfloat16()
    for g in (32, 128, 256):
        codes = _filled((4, 256), torch.float8_e4m3fn)
        scales = _filled((4, 256 // g), torch.uint8 if g == 32 else torch.float32)
        lb.add_norm(lb.norm_args(x=x, eps=1e-12, codes=codes, scales=scales, group=g, device=dev), 4)
        c, s = _codes32(x, None, None, 1e-12, g)
        assert torch.equal(scales.cpu().float().nan_to_num(-1.0), s.float().nan_to_num(-1.0))
        assert torch.equal(codes.float().cpu(), c)


def test_streams_and_graphs():
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    dev = torch.cuda.current_device()
    T, n = 50, 2048
    x, r, w = _tensors(T, n, True, 3)
    start = r.clone()
    out = torch.empty(T, n, dtype=torch.bfloat16, device="cuda")
    args = lb.norm_args(x=x, weight=w, residual=r, residual_out=r, out=out, device=dev)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    before = lb.launch_count()
    with torch.cuda.stream(side):
        lb.add_norm(args, T, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert lb.launch_count() == before + 1
    one, once = out.clone(), r.clone()
    r.copy_(start)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lb.add_norm(args, T, stream=torch.cuda.current_stream())
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    twice = (x.float() + once.float()).bfloat16()          # each replay advances the stream
    assert torch.equal(r, twice) and not torch.equal(out, one)
    lb.add_norm(args, 0)
