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


@pytest.mark.parametrize("kind,ranks,tuning", [("bgmv", ([64], [8]), ({}, {})), ("bgmv", ([8], [8]), ({5: 3}, {5: 2})),
                                               ("sgmv", ([64], [8]), ({}, {}))])
def test_two_pools_apply_in_turn(kind, ranks, tuning):
    """Pools of different ranks or ring depths: the one whose kernels need less shared memory comes second."""
    require_gpu()
    from paper_2602_24044_b200 import workloads as W
    from paper_2602_24044_b200.harness import Session, bf16_bits
    wls = [W.make_custom(90, 512, 512, 6, r, kind=kind, scale=0.5, weight_mode="unitB", seed=60 + i, tile_m=16)
           for i, r in enumerate(ranks)]
    with Session(wls[0], tuning=tuning[0]) as a, Session(wls[1], tuning=tuning[1]) as b:
        want = bf16_bits(a.apply()), bf16_bits(b.apply())
        for s, w in ((a, want[0]), (b, want[1]), (a, want[0])):
            assert np.array_equal(bf16_bits(s.apply()), w)


def test_lists_built_again_are_not_the_oldest():
    """A pool knows the last 256 lists that it built: one that was built first, and again just now, is among them
    when the 257th comes."""
    require_gpu()
    import torch
    from paper_2602_24044_b200 import binding as lb
    buf = torch.zeros(lb.pool_bytes(2, 8, [(16, 16)]) + 256, dtype=torch.uint8, device="cuda")
    pool = lb.pool_create(2, 8, [(16, 16)], buf[(-buf.data_ptr()) % 256:])
    try:
        n = (lb.segments_bytes(1, 2, 16) + 15) // 16 * 4
        lists = torch.zeros((257, n), dtype=torch.int32, device="cuda")
        slot = _i32([0])
        ws = torch.zeros(max(lb.workspace_bytes(pool, 1), 16), dtype=torch.uint8, device="cuda")
        x = torch.zeros((1, 16), dtype=torch.bfloat16, device="cuda")

        def apply(i):
            lb.bgmv_apply(pool, 0, x, 16, x, 16, x, 16, slot, 1, lists[i], ws)

        for i in [*range(256), 0, 256]:
            lb.build_segments(pool, slot, 1, 16, 128, lists[i])
        apply(0)
        apply(256)
        with pytest.raises(lb.LoraError) as e:       # the oldest now
            apply(1)
        assert e.value.status == 1
        apply(2)
        torch.cuda.synchronize()
    finally:
        lb.pool_destroy(pool)
