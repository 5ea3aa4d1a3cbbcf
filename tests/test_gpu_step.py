"""The example's whole step: token ids through norm, projections with adapters, positions on three axes, the cache,
attention, residual and norm, logits and sampling, to the next token ids; each part against its definition on what
the part before it gave."""
import os
import sys

import numpy as np
import pytest

import kv_ref as ref
from gpu_util import require_gpu
from test_gpu_axes import _by_hand, _turned_by
from test_gpu_sample import _reference

pytestmark = pytest.mark.gpu


def _np(t):
    import torch
    torch.cuda.synchronize()
    return t.float().cpu().numpy() if t.dtype == torch.bfloat16 else t.cpu().numpy()


@pytest.mark.parametrize("greedy", [True, False])
def test_steps_from_tokens_to_tokens(greedy):
    require_gpu()
    import torch
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    from attention_step import ServedStep
    hq, hkv, d, R = 8, 2, 128, 3
    axis = np.array([p % 3 if p < 48 else 0 for p in range(64)])
    media = [[(2, 1, 4, 5, 1)], [], [(0, 3, 2, 3, 2), (30, 1, 6, 6, 1)]]
    served = ServedStep(vocab=1500, pages=64, max_positions=256, axis_of_pair=axis)
    layer = served.layer
    layer.admit(R, 200, media=media)
    seen = {}
    inner = layer.step

    def spied(h, q_len, adapters):
        out, attn, qkv = inner(h, q_len, adapters)
        seen.update(h=h, out=out.clone(), attn=attn, qkv=qkv)
        return out, attn, qkv

    layer.step = spied
    norms = []
    inner_norm = served._norm

    def spied_norm(x, weight, residual=None):
        before = (x.clone(), None if residual is None else residual.clone(), weight)
        stream, h = inner_norm(x, weight, residual)
        norms.append((before, stream.clone(), h.clone()))
        return stream, h

    served._norm = spied_norm
    g = torch.Generator(device="cuda").manual_seed(7)
    owner = torch.tensor([0, 2, -1], dtype=torch.int32, device="cuda")
    tau = torch.tensor([0.0, 0.0, 0.0] if greedy else [0.7, 1.0, 1.3], device="cuda")
    k = None if greedy else torch.tensor([0, 40, 0], dtype=torch.int32, device="cuda")
    p = None if greedy else torch.tensor([0.9, 1.0, 1.0], device="cuda")
    mp = None if greedy else torch.tensor([0.0, 0.0, 0.05], device="cuda")
    length = [0] * R
    keys, values = [np.zeros((0, hkv, d)) for _ in range(R)], [np.zeros((0, hkv, d)) for _ in range(R)]
    qw, kw, cs = _np(layer.q_weight), _np(layer.k_weight), _np(layer.angles)
    ids = torch.randint(0, 1500, (40 + 9 + 70,), generator=g, device="cuda", dtype=torch.int32)
    for q_len in ([40, 9, 70], [1, 1, 1], [1, 1, 1]):
        T = sum(q_len)
        u = torch.rand(R, generator=g, device="cuda")
        token, logprob, logits = served.step(ids, q_len, torch.repeat_interleave(owner, torch.tensor(q_len, device="cuda")),
                                             u, tau, top_k=k, top_p=p, min_p=mp)
        # both norms (tolerances as of the norm's own tests)
        (x, _, w), stream, h = norms[-2]
        y = x.double() / (x.double().pow(2).mean(-1, keepdim=True) + 1e-6).sqrt() * w.double()
        assert ((h.double() - y).abs() <= y.abs() * (2.0 ** -8 + 10 * 2.0 ** -24)).all() and torch.equal(seen["h"], h)
        (x, r, w), stream, h = norms[-1]
        s = x.double() + r.double()
        y = s / (s.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt() * w.double()
        assert torch.equal(x, seen["out"]) and torch.equal(stream, (x.float() + r.float()).bfloat16())
        assert ((h.double() - y).abs() <= y.abs() * (2.0 ** -8 + 10 * 2.0 ** -24)).all()
        # positions, rotation, cache, attention
        rows, got = _np(seen["qkv"]), _np(seen["attn"]).reshape(T, hq, d)
        t0 = 0
        for i, n in enumerate(q_len):
            pos = np.array([_by_hand(media[i], length[i] + t) for t in range(n)]).T
            turn = _turned_by(cs, axis, pos)
            part = rows[t0:t0 + n].reshape(n, hq + 2 * hkv, d)
            q = ref.bf16(ref.rotate(ref.norm32(part[:, :hq].reshape(-1, d), qw, 1e-6), np.repeat(turn, hq, 0), d, False))
            kk = ref.rotate(ref.norm32(part[:, hq:hq + hkv].reshape(-1, d), kw, 1e-6), np.repeat(turn, hkv, 0), d, False)
            for store, val in ((keys, kk), (values, part[:, hq + hkv:].reshape(-1, d))):
                c, sc, low = ref.quantise(val)
                store[i] = np.concatenate([store[i], (c.astype(np.float64) * sc[:, None] + low[:, None]).reshape(n, hkv, d)])
            length[i] += n
            L = length[i]
            want, _, mag = ref.attention(q.astype(np.float64).reshape(n, hq, d), keys[i], values[i],
                                         np.arange(-(-L // 16))[None], 16, 1 << 20, [0, n], [L - n], d ** -0.5)
            bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2.0 ** -12) * mag + 2.0 ** -25 * np.abs(values[i]).max() * L
            assert (np.abs(got[t0:t0 + n] - want) <= bound).all()
            t0 += n
        # the next tokens
        xs = _np(logits)
        for i in range(R):
            want, lp, _ = _reference(xs[i], _np(tau)[i], 0 if k is None else int(k[i]), 1.0 if p is None else _np(p)[i],
                                     0.0 if mp is None else _np(mp)[i], _np(u)[i])
            assert int(token[i]) == want and abs(float(logprob[i]) - lp) <= 4e-11 + 2.0 ** -24 * abs(lp)
        ids = token
    assert layer.kv.status()[:2] == [0, 0]
    served.close()
