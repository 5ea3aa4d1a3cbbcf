"""Host-only checks of the cache entry points: sizes, and refusals before any device call."""
import numpy as np
import pytest

import kv_ref as ref
from paper_2602_24044_b200 import binding as lb
from paper_2602_24044_b200 import build as lbuild


@pytest.fixture(scope="module", autouse=True)
def lib():
    lbuild.build()


SHAPE = dict(num_layers=2, num_pages=10, page_size=16, num_q_heads=32, num_kv_heads=8, head_dim=128)


@pytest.mark.parametrize("page,hkv,d", [(16, 8, 128), (128, 3, 64), (64, 1, 64)])
def test_sizes(page, hkv, d):
    kw = dict(SHAPE, page_size=page, num_kv_heads=hkv, num_q_heads=2 * hkv, head_dim=d)
    layer = 10 * hkv * page * (d + 8)          # K and V: d / 2 + 4 bytes each, a token and head
    padded = (layer + 255) // 256 * 256
    assert lb.kv_bytes(**kw) == 256 + 2 * padded
    assert lb.kv_layer_range(1, **kw) == (256 + padded, layer)


@pytest.mark.parametrize("bad,status", [
    (dict(num_layers=0), 1), (dict(num_pages=0), 1), (dict(page_size=24), 2), (dict(page_size=256), 2),
    (dict(head_dim=96), 2), (dict(head_dim=256), 2), (dict(num_q_heads=30), 2), (dict(num_kv_heads=0), 2),
    (dict(num_q_heads=0), 2), (dict(num_q_heads=8 * 129), 2), (dict(num_pages=1 << 28), 2)])
def test_shapes_that_are_refused(bad, status):
    with pytest.raises(lb.LoraError) as e:
        lb.kv_bytes(**dict(SHAPE, **bad))
    assert e.value.status == status


def test_create_rejects_bad_buffers_before_any_device_call():
    buf = np.zeros(1 << 20, np.uint8)
    at = buf.ctypes.data + (-buf.ctypes.data) % 256
    for ptr, n, status in ((at + 16, 1 << 19, 1), (None, 1 << 19, 1), (at, 1024, 7)):
        with pytest.raises(lb.LoraError) as e:
            lb.kv_create(**SHAPE, device_buf=ptr, device_buf_bytes=n)
        assert e.value.status == status
    with pytest.raises(lb.LoraError) as e:
        lb.kv_layer_range(2, **SHAPE)
    assert e.value.status == 3


def test_null_handles_are_rejected():
    a = lb.qk_args(num_q_heads=1, num_kv_heads=1, head_dim=64)
    for call in (lambda: lb.kv_destroy(None), lambda: lb.kv_tables_bytes(None, 1, 1), lambda: lb.kv_workspace_bytes(None),
                 lambda: lb.kv_append(None, 0, a, None, 1), lambda: lb.kv_read(None, 0, None, 1, None, 0, None, 0),
                 lambda: lb.kv_check_status(None), lambda: lb.kv_release(None, None, 1, 1, None, None, 1, None, None),
                 lambda: lb.kv_attention(None, 0, None, 0, None, 0, None, 1.0, None, 1, 1, None, 1, None),
                 lambda: lb.kv_build_tables(None, None, None, 1, 1, None, None, None, 1, None, tables_bytes=0)):
        with pytest.raises(lb.LoraError) as e:
            call()
        assert e.value.status == 1


@pytest.mark.parametrize("bad,status", [
    (dict(head_dim=96), 2), (dict(num_q_heads=-1), 2), (dict(num_q_heads=0, num_kv_heads=0), 2),
    (dict(ldq=248), 2), (dict(ldq=260), 2), (dict(ldqo=8), 2), (dict(q=None), 1), (dict(q_out=None), 1),
    (dict(k_out=None), 1), (dict(rot_dim=24), 2), (dict(rot_dim=144), 2), (dict(num_positions=0), 2),
    (dict(positions=None), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(T=-1), 2),
    (dict(q_out="q+16"), 1), (dict(q_out="k"), 1), (dict(k_out="q_out"), 1), (dict(q="odd"), 1)])
def test_norm_rope_refusals(bad, status):
    """Addresses that are never followed: every one of these is refused on the host."""
    base = 1 << 20
    at = {"q+16": base + 16, "k": base + 512, "q_out": base + (1 << 16), "odd": base + 2}
    kw = dict(num_q_heads=2, num_kv_heads=1, head_dim=128, q=base, ldq=512, k=base + 512, ldk=512, q_weight=base,
              eps=1e-6, cos_sin=None, rot_dim=128, num_positions=4, positions=base, q_out=base + (1 << 16), ldqo=256,
              k_out=base + (1 << 17), ldko=128)
    kw.update({k: at.get(v, v) if isinstance(v, str) else v for k, v in bad.items() if k != "T"})
    if kw["ldqo"] == 256 and bad.get("q_out") in ("q+16", "k"):
        kw["ldqo"] = 512
    a = lb.qk_args(**kw)
    a.cos_sin = base
    with pytest.raises(lb.LoraError) as e:
        lb.qk_norm_rope(a, bad.get("T", 3))
    assert e.value.status == status


def test_nothing_to_do_is_fine():
    lb.qk_norm_rope(lb.qk_args(num_q_heads=2, num_kv_heads=1, head_dim=128), 0)


def test_the_reference_quantiser_stays_within_half_a_step():
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((200, 128)) * np.exp(3 * rng.standard_normal((200, 1)))).astype(np.float32)
    c, s, l = ref.quantise(x)
    y = ref.dequantise32(c, s, l)
    # half a step, and what the roundings of scale and low to 8 bits add at the ends of the range
    assert (np.abs(y - x) <= s[:, None] * (0.5 + 15 * 2.0 ** -8) + np.abs(l)[:, None] * 2.0 ** -8).all()
    assert c.min() == 0 and c.max() == 15
