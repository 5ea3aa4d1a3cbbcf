"""Host-only checks of the norm of rows: refusals before any device call, and the argument block."""
import pytest

from paper_2602_24044_b200 import binding as lb
from paper_2602_24044_b200 import build as lbuild


@pytest.fixture(scope="module", autouse=True)
def lib():
    lbuild.build()


BASE = 1 << 24


@pytest.mark.parametrize("bad,status", [
    (dict(width=12), 2), (dict(width=0), 2), (dict(width=32776), 2), (dict(group=64), 2), (dict(group=-1), 2),
    (dict(width=1000, group=128), 2), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1),
    (dict(T=-1), 2), (dict(x=None), 1), (dict(x=BASE + 8), 1), (dict(weight=BASE + 2), 1), (dict(ldx=248), 2),
    (dict(ldx=260), 2), (dict(residual=None), 1), (dict(ldr=8), 2), (dict(ldro=255), 2), (dict(ldo=0), 2),
    (dict(codes=None), 1), (dict(scales=None), 1), (dict(codes=BASE + (4 << 20) + 4), 1), (dict(ldc=260), 2),
    (dict(scales=BASE + (5 << 20) + 2), 1), (dict(lds=1), 2), (dict(group=0), 1),
    (dict(out=None, codes=None, scales=None, group=0, residual=None, residual_out=None), 1),
    (dict(out=BASE + 16), 1), (dict(out=BASE + (1 << 20)), 1), (dict(out=BASE, ldo=512), 1),
    (dict(residual_out=BASE + (2 << 20), out=BASE + (2 << 20)), 1), (dict(codes=BASE), 1), (dict(scales=BASE), 1),
    (dict(codes=BASE + (3 << 20)), 1), (dict(weight=BASE + (3 << 20) + 512), 1)])
def test_refusals(bad, status):
    """Addresses that are never followed: every one of these is refused on the host."""
    kw = dict(x=BASE, ldx=256, weight=BASE + (6 << 20), residual=BASE + (1 << 20), ldr=256,
              residual_out=BASE + (2 << 20), ldro=256, out=BASE + (3 << 20), ldo=256, codes=BASE + (4 << 20), ldc=256,
              scales=BASE + (5 << 20), lds=2, group=128, width=256, eps=1e-6)
    kw.update({k: v for k, v in bad.items() if k != "T"})
    if bad.get("out") == BASE + (1 << 20):
        kw["ldo"] = 512
    with pytest.raises(lb.LoraError) as e:
        lb.add_norm(lb.norm_args(**kw), bad.get("T", 3))
    assert e.value.status == status


def test_nothing_to_do_is_fine():
    lb.add_norm(lb.norm_args(x=None, width=64), 0)


def test_tensors_are_looked_at():
    import torch
    bf = dict(dtype=torch.bfloat16)
    x = torch.zeros(4, 64, **bf)
    # (a tensor of the host: the block is for device 0)
    for kw in (dict(x=x), dict(x=BASE, ldx=64, width=64, out=x), dict(x=BASE, ldx=64, width=64, weight=x[0]),
               dict(x=x[:, ::2]), dict(x=x.t()), dict(x=x[0])):
        with pytest.raises(lb.LoraError) as e:
            lb.norm_args(**kw)
        assert e.value.status == 1
