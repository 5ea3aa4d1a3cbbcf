"""Host-only checks of sampling: refusals before any device call, and the argument block."""
import pytest

from paper_2602_24044_b200 import binding as lb
from paper_2602_24044_b200 import build as lbuild


@pytest.fixture(scope="module", autouse=True)
def lib():
    lbuild.build()


BASE = 1 << 24


@pytest.mark.parametrize("bad,status", [
    (dict(vocab=0), 2), (dict(vocab=(1 << 20) - 7, ld=1 << 20), 2), (dict(logits_type=2), 1), (dict(logits_type=-1), 1),
    (dict(R=-1), 2), (dict(R=(1 << 24) + 1), 2), (dict(ld=999), 2), (dict(logits=None), 1), (dict(temperature=None), 1),
    (dict(uniform=None), 1), (dict(token=None), 1), (dict(logits=BASE + 2), 1), (dict(token=BASE + (1 << 20) + 2), 1),
    (dict(top_k=BASE + 1), 1), (dict(logprob=BASE + (1 << 20)), 1), (dict(token=BASE + 400), 1),
    (dict(token=BASE + (2 << 20) + 8), 1), (dict(logprob=BASE + (6 << 20)), 1), (dict(logprob=BASE + 3999 * 3), 1),
    (dict(workspace=BASE + (8 << 20) + 8, workspace_bytes=1 << 20), 1),
    (dict(workspace=BASE + (8 << 20), workspace_bytes=63), 7)])
def test_refusals(bad, status):
    """Addresses that are never followed: every one of these is refused on the host."""
    kw = dict(logits=BASE, ld=1000, vocab=1000, logits_type=lb.LOGITS_FP32, token=BASE + (1 << 20),
              temperature=BASE + (2 << 20), top_k=BASE + (3 << 20), top_p=BASE + (4 << 20), min_p=BASE + (5 << 20),
              uniform=BASE + (6 << 20), logprob=BASE + (7 << 20))
    kw.update({k: v for k, v in bad.items() if k != "R"})
    with pytest.raises(lb.LoraError) as e:
        lb.sample(lb.sample_args(**kw), bad.get("R", 3))
    assert e.value.status == status


@pytest.mark.parametrize("other", ["token", "logprob", "temperature", "top_k", "top_p", "min_p", "uniform", "logits"])
@pytest.mark.parametrize("before", [0, 4, 48])
def test_workspace_on_other_memory_is_refused(other, before):
    """64 bytes are written for three rows: they may not begin at, inside or at the end of anything else."""
    kw = dict(logits=BASE, ld=1000, vocab=1000, logits_type=lb.LOGITS_FP32, token=BASE + (1 << 20),
              temperature=BASE + (2 << 20), top_k=BASE + (3 << 20), top_p=BASE + (4 << 20), min_p=BASE + (5 << 20),
              uniform=BASE + (6 << 20), logprob=BASE + (7 << 20), workspace=BASE + (8 << 20), workspace_bytes=64)
    kw[other] = BASE + (8 << 20) + before
    with pytest.raises(lb.LoraError) as e:
        lb.sample(lb.sample_args(**kw), 3)
    assert e.value.status == 1


def test_workspace_bytes():
    assert lb.sample_workspace_bytes(0) == 16 and lb.sample_workspace_bytes(3) == 16 + 3 * 16
    for R in (-1, (1 << 24) + 1):
        with pytest.raises(lb.LoraError) as e:
            lb.sample_workspace_bytes(R)
        assert e.value.status == 2


def test_nothing_to_do_is_fine():
    lb.sample(lb.sample_args(logits=None, vocab=5, temperature=None, uniform=None, token=None), 0)


def test_tensors_are_looked_at():
    import torch
    kw = dict(logits=BASE, ld=64, vocab=64, temperature=BASE, uniform=BASE, token=BASE)
    for bad in (dict(logits=torch.zeros(2, 64), ld=None), dict(temperature=torch.zeros(2)),
                dict(top_k=torch.zeros(2, dtype=torch.int64)), dict(logits=torch.zeros(2, 64).t(), ld=None)):
        with pytest.raises(lb.LoraError) as e:
            lb.sample_args(**dict(kw, **bad))
        assert e.value.status == 1
