"""Several pools on one GPU, used in turn: what one launches does not depend on the others."""
import numpy as np
import pytest

from gpu_util import require_gpu
from test_gpu_kv import _i32, _np

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,slots", [(900, (2600, 2200)), (4000, (330, 250)), (16000, (120, 60))])
def test_two_pools_build_segments_in_turn(T, slots):
    """The three list kernels with more than 48 KB of shared memory: the pool that needs less comes second."""
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    pools = []
    for n in slots:
        buf = torch.zeros(lb.pool_bytes(n, 8, [(16, 16)]) + 256, dtype=torch.uint8, device="cuda")
        mem = buf[(-buf.data_ptr()) % 256:]
        pools.append((lb.pool_create(n, 8, [(16, 16)], mem), n, buf))
    rng = np.random.default_rng(T)
    try:
        first = {}
        for which in (0, 1, 0, 1):
            pool, n, _ = pools[which]
            idx = _i32(rng.integers(0, n, T)) if which not in first else first[which][0]
            meta = torch.zeros((lb.segments_bytes(T, n, 16) + 3) // 4, dtype=torch.int32, device="cuda")
            lb.build_segments(pool, idx, T, 16, 128, meta)
            got = _np(meta)
            if which in first:
                assert np.array_equal(got, first[which][1])
            first[which] = idx, got
    finally:
        torch.cuda.synchronize()
        for pool, _, _ in pools:
            lb.pool_destroy(pool)
