"""The paged 4-bit cache on the GPU where it went wrong, or was never run: several handles at once, tables in
turn, probabilities far below the largest, groups of every size, batches of many rows."""
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
    with pytest.raises(lb.LoraError) as e:
        lb.qk_norm_rope(lb.qk_args(num_q_heads=2, num_kv_heads=0, head_dim=64, q=x, ldq=128, q_out=out, device=99), 3)
    assert e.value.status == 9 and lb.launch_count() == before and (_np(out) == 0).all()
