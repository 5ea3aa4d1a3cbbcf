"""Host-only checks of positions on several axes: refusals before any device call, the argument block, spans."""
import numpy as np
import pytest

from paper_2602_24044_b200 import binding as lb
from paper_2602_24044_b200 import build as lbuild
from paper_2602_24044_b200.harness import media_spans


@pytest.fixture(scope="module", autouse=True)
def lib():
    lbuild.build()


BASE = 1 << 20


@pytest.mark.parametrize("bad,status", [
    (dict(num_axes=0), 2), (dict(num_axes=5), 2), (dict(num_axes=2), 2), (dict(ld_positions=2), 2),
    (dict(axis_of_pair=[0] * 63), 2), (dict(axis_of_pair=[0] * 63 + [3]), 2), (dict(axis_of_pair=[0] * 63 + [-1]), 2),
    (dict(axis_of_pair=[256] * 64), 2), (dict(cos_sin=None), 1), (dict(positions=None), 1), (dict(head_dim=96), 2),
    (dict(q_out=None), 1), (dict(T=-1), 2)])
def test_rotation_refusals(bad, status):
    """Addresses that are never followed: every one of these is refused on the host."""
    kw = dict(num_q_heads=2, num_kv_heads=1, head_dim=128, q=BASE, ldq=512, k=BASE + 512, ldk=512, rot_dim=128,
              num_positions=4, positions=BASE, q_out=BASE + (1 << 16), ldqo=256, k_out=BASE + (1 << 17), ldko=128,
              axis_of_pair=[0, 1, 2, 0] * 16, num_axes=3, ld_positions=3)
    kw.update({k: v for k, v in bad.items() if k not in ("T", "cos_sin")})
    with pytest.raises(lb.LoraError) as e:
        a = lb.qk_args(**kw)
        a.cos_sin = bad.get("cos_sin", BASE)
        lb.qk_norm_rope(a, bad.get("T", 3))
    assert e.value.status == status


def test_positions_that_share_memory_are_refused():
    """Rows closer to each other than the tokens are many (one row expanded to all axes): their distance is no leading
    dimension."""
    import torch
    buf = torch.zeros(5, 8, dtype=torch.int32)
    for bad in (buf[:1].expand(3, 8), torch.as_strided(buf, (3, 8), (4, 1)), buf.t()[:3], buf[0]):
        with pytest.raises(lb.LoraError, match="a row of tokens for each axis") as e:
            lb.qk_args(num_q_heads=1, num_kv_heads=1, head_dim=64, rot_dim=64, axis_of_pair=[0, 1, 2, 0] * 8, positions=bad)
        assert e.value.status == 1


def test_null_arguments_are_rejected():
    a = lb.qk_args(num_q_heads=1, num_kv_heads=1, head_dim=64, rot_dim=64, axis_of_pair=[0] * 32, num_axes=1)
    lib = lb._lib()
    assert lib.lora_qk_norm_rope_axes(a, None, 1, None) == 1
    assert lib.lora_kv_append_axes(None, 0, a, a.axes, None, 1, None) == 1
    assert lib.lora_kv_append_axes(None, 0, a, None, None, 1, None) == 1
    for call in (lambda: lb.kv_append(None, 0, a, None, 1),
                 lambda: lb.kv_axis_positions(None, BASE, 1, 1, BASE, BASE, 1, BASE, 1)):
        with pytest.raises(lb.LoraError) as e:
            call()
        assert e.value.status == 1
    lb.qk_norm_rope(a, 0)


def test_spans():
    spans, begin = media_spans([[], [(3, 1, 4, 6), (30, 3, 2, 2, 5)], [(0, 2, 1, 1, 0)]])
    assert begin.tolist() == [0, 0, 2, 3] and spans.dtype == np.int32
    # three tokens of text, a grid of 4 x 6 (position 3, then on from 9), three tokens, three frames five apart
    assert spans.tolist() == [[3, 1, 4, 6, 3, 1, 0, 0], [30, 3, 2, 2, 12, 5, 0, 0], [0, 2, 1, 1, 0, 0, 0, 0]]
    empty, begin = media_spans([[], []])
    assert empty.shape == (0, 8) and begin.tolist() == [0, 0, 0]
    for bad in ([(5, 1, 2, 2), (8, 1, 1, 1)], [(-1, 1, 1, 1)], [(0, 0, 1, 1)], [(0, 1, 1, 1, -1)]):
        with pytest.raises(ValueError):
            media_spans([bad])
