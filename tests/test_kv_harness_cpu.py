"""KVCache's own part (buffers, streams) without a GPU: the library and torch's device side are stand-ins."""
import contextlib

import pytest
import torch

from paper_2602_24044_b200 import binding as lb
from paper_2602_24044_b200 import harness


class Tensor:
    """What KVCache asks of a device tensor: contiguous, with a record of the streams it was kept for."""

    def __init__(self, *shape, dtype=torch.int32, made_on=0):
        self.shape, self.dtype, self.made_on, self.kept = shape, dtype, made_on, set()

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        out = [1]
        for s in self.shape[:0:-1]:
            out.insert(0, out[0] * s)
        return tuple(out) if i is None else out[i]

    def data_ptr(self):
        return 4096

    def is_contiguous(self):
        return True

    def get_device(self):
        return 0

    def record_stream(self, stream):
        self.kept.add(stream.cuda_stream)

    def __getitem__(self, i):
        return self


class Stream:
    def __init__(self, handle, device=None):
        self.cuda_stream, self.waited = handle, 0

    def synchronize(self):
        self.waited += 1


class Outside(Stream):
    """A stream that is not torch's."""


class Cuda:
    def __init__(self):
        self.on, self.waited = [Stream(0)], 0

    def synchronize(self, device=None):
        self.waited += 1

    def current_stream(self, device=None):
        return self.on[-1]

    default_stream = staticmethod(lambda device=None: Stream(0))
    ExternalStream = Outside
    is_current_stream_capturing = staticmethod(lambda: False)

    @contextlib.contextmanager
    def stream(self, s):
        self.on.append(s)
        yield
        self.on.pop()


class Torch:
    def __init__(self):
        self.cuda, self.made = Cuda(), []

    def __getattr__(self, name):
        return getattr(torch, name)

    def empty(self, n, dtype, device):
        t = Tensor(n, dtype=dtype, made_on=self.cuda.on[-1].cuda_stream)
        self.made.append(t)
        return t


class Library:
    """The binding, with the entry points that need a handle replaced; `calls` are the launches."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        if name in ("kv_build_tables", "kv_append", "kv_read", "kv_attention", "kv_release"):
            return lambda *a, **k: self.calls.append(name)
        return getattr(lb, name)

    kv_create = staticmethod(lambda *a, **k: 1)
    kv_destroy = staticmethod(lambda kv: None)
    kv_workspace_bytes = staticmethod(lambda kv: 1024)
    kv_tables_bytes = staticmethod(lambda kv, R, T: 4 * (64 + 16 * R + 16 * T))


@pytest.fixture
def cache(monkeypatch):
    monkeypatch.setattr(harness, "torch", Torch())
    monkeypatch.setattr(harness, "lb", Library())
    c = harness.KVCache(1, 8, 16, 4, 2, 64)
    yield c
    c.kv = 0                                     # the handle is a stand-in: nothing to destroy


def _build(c, R, stream):
    c.build_tables(Tensor(R), Tensor(R), R, Tensor(8), Tensor(1), Tensor(R, 4), stream=stream)


def test_tables_that_grow_are_kept_for_the_streams_that_use_them(cache):
    c = cache
    _build(c, 1, Stream(7))
    old = c.tables
    assert old.made_on == 7                      # recycled memory is free in the order of the stream that writes it
    rows = Tensor(1, 256, dtype=torch.bfloat16)
    c.attention(0, rows, Tensor(1, 256, dtype=torch.bfloat16), scale=1.0, stream=Stream(9))
    _build(c, 1, None)
    assert c.tables is old and not old.kept
    _build(c, 500, Stream(11))
    assert c.tables is not old and c.tables.made_on == 11
    assert {7, 9, 0} <= old.kept and harness.torch.cuda.waited == 0


@pytest.mark.parametrize("stream", [11, Outside(11)])
def test_streams_that_are_not_torchs_are_waited_for(cache, stream):
    """They may be gone when the memory is given back, so nothing is asked of them then."""
    _build(cache, 1, stream)
    old = cache.tables
    _build(cache, 500, Stream(7))
    assert cache.tables is not old and not old.kept and harness.torch.cuda.waited == 1


def test_room_made_beforehand_is_ready_for_any_stream(cache):
    here = harness.torch.cuda.on[-1]
    cache.reserve(4, 4)
    assert here.waited == 1 and cache.tables.made_on == 0
    cache.reserve(2, 2)
    assert here.waited == 1                      # nothing moved


def test_buffers_of_a_dropped_cache_are_kept_for_its_streams(monkeypatch):
    monkeypatch.setattr(harness, "torch", Torch())
    monkeypatch.setattr(harness, "lb", Library())
    c = harness.KVCache(1, 8, 16, 4, 2, 64)
    _build(c, 1, Stream(7))
    c.read(0, Tensor(1), Tensor(1, 128, dtype=torch.bfloat16), None, stream=Stream(5))
    made = list(harness.torch.made)
    del c
    assert len(made) == 3 and all({5, 7} <= t.kept for t in made)


# -- what a tensor has to be (CPU tensors, which the cache is told are on its device) -------------------------
def _i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def _bf16(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


TABLE = dict(kv_len=_i32(3), q_len=_i32(3), T=5, free_pages=_i32(8), free_count=_i32(1), block_table=_i32(3, 4))


@pytest.mark.parametrize("bad", [
    dict(kv_len=torch.zeros(3, dtype=torch.int64)), dict(q_len=torch.zeros(3)), dict(q_len=_i32(6)[::2]),
    dict(q_len=_i32(2)), dict(free_pages=torch.zeros(8, dtype=torch.int64)), dict(free_count=_i32(0)),
    dict(free_count=torch.zeros(1, dtype=torch.int64)), dict(kv_len_out=_i32(2)), dict(kv_len_out=_i32(6)[::2]), dict(free_count_out=torch.zeros(1)),
    dict(block_table=_i32(2, 4)), dict(block_table=_i32(12)), dict(block_table=_i32(3, 8)[:, ::2]),
    dict(block_table=_i32(4, 3).t()), dict(block_table=torch.zeros((3, 4), dtype=torch.int64)),
    dict(block_table=_i32(1, 4).expand(3, 4)),
    dict(block_table=_i32(3, 8)[:, 4:])])          # rows that reach past the end of the memory
def test_tables_that_are_refused(cache, bad):
    cache._index = -1
    with pytest.raises(ValueError):
        cache.build_tables(**{**TABLE, **bad})
    assert harness.lb.calls == []


@pytest.mark.parametrize("good", [
    {}, dict(block_table=_i32(5, 4)[:3]), dict(block_table=_i32(3, 8)[:, :4]), dict(free_pages=_i32(2)),
    dict(block_table=_i32(3, 0)), dict(kv_len=_i32(1), q_len=_i32(1), T=1, block_table=_i32(4).unsqueeze(0)),
    dict(kv_len=_i32(0), q_len=_i32(0), T=0, block_table=_i32(0, 4)),
    dict(kv_len=_i32(0), q_len=_i32(0), T=0, block_table=_i32(4, 0).t())])
def test_tables_that_are_accepted(cache, good):
    cache._index = -1
    a = {**TABLE, **good}
    cache.build_tables(**a)
    t = a["block_table"]
    assert harness.lb.calls == ["kv_build_tables"] and cache.ld_table == (t.stride(0) if t.numel() else t.shape[1])


def test_attention_that_is_refused(cache):
    cache._index = -1
    with pytest.raises(ValueError):                # no tables
        cache.attention(0, _bf16(5, 256), _bf16(5, 256), scale=1.0)
    with pytest.raises(ValueError):
        cache.append(0, lb.qk_args(num_q_heads=4, num_kv_heads=2, head_dim=64))
    cache.build_tables(**TABLE)
    good = dict(q=_bf16(5, 256), out=_bf16(5, 256), lse=torch.zeros(5, 4))
    for bad in (dict(q=_bf16(4, 256)), dict(q=_bf16(5, 255)), dict(q=_bf16(5, 512)[:, ::2]), dict(q=_bf16(256, 5).t()),
                dict(q=torch.zeros(5, 256)), dict(q=_bf16(5 * 256)), dict(q=_bf16(5, 64, 4).transpose(1, 2)),
                dict(out=_bf16(4, 256)), dict(out=torch.zeros((5, 256), dtype=torch.float16)),
                dict(lse=torch.zeros(5, 3)), dict(lse=torch.zeros(4, 5).t()), dict(lse=_bf16(5, 4))):
        with pytest.raises(ValueError):
            cache.attention(0, scale=1.0, **{**good, **bad})
    cache._index = 0                               # tensors of another device
    with pytest.raises(ValueError):
        cache.attention(0, scale=1.0, **good)
    cache._index = -1
    assert harness.lb.calls == ["kv_build_tables"]
    for q in (_bf16(5, 256), _bf16(9, 256), _bf16(5, 400)[:, 16:272], _bf16(5, 4, 64), _bf16(5, 6, 64)[:, 2:]):
        cache.attention(0, q, good["out"], scale=1.0)
    assert len(harness.lb.calls) == 6


def test_rows_that_are_refused(cache):
    cache._index = -1
    slots = _i32(5)
    for bad in (dict(slots=torch.zeros(5, dtype=torch.int64)), dict(slots=_i32(10)[::2]), dict(k_out=_bf16(4, 128)),
                dict(v_out=_bf16(5, 100)), dict(k_out=torch.zeros(5, 128))):
        with pytest.raises(ValueError):
            cache.read(0, **{**dict(slots=slots, k_out=_bf16(5, 128), v_out=_bf16(5, 128)), **bad})
    args = lb.qk_args(num_q_heads=4, num_kv_heads=2, head_dim=64)
    for slots in (_i32(4), torch.zeros(5, dtype=torch.int64)):
        with pytest.raises(ValueError):
            cache.append(0, args, slots, 5)
    good = dict(requests=_i32(2), kv_len=_i32(3), block_table=_i32(3, 4), free_pages=_i32(8), free_count=_i32(1))
    for bad in (dict(requests=torch.zeros(2, dtype=torch.int64)), dict(block_table=_i32(2, 4)), dict(free_pages=_i32(7)),
                dict(kv_len=torch.zeros(3)), dict(free_count=_i32(0))):
        with pytest.raises(ValueError):
            cache.release(**{**good, **bad})
    assert harness.lb.calls == []
    cache.read(0, _i32(5), _bf16(5, 136), None)
    cache.append(0, args, _i32(5), 5)
    cache.release(**good)
    assert len(harness.lb.calls) == 3


ROWS = dict(num_q_heads=4, num_kv_heads=2, head_dim=64, ldq=512, ldk=512, ldv=512, device=-1)


def test_argument_blocks_know_how_many_tokens_they_hold():
    fused = _bf16(5, 512)
    kw = dict(ROWS, q=fused, k=fused[:, 256:], v=fused[:, 384:], q_out=_bf16(6, 256), k_out=_bf16(5, 128))
    assert lb.qk_args(**kw).max_tokens == 5
    assert lb.qk_args(**dict(kw, q_out=_bf16(4, 256))).max_tokens == 4
    assert lb.qk_args(**dict(kw, k=fused[:, 400:])).max_tokens == 4       # its last row reaches past the end
    a = lb.qk_args(**dict(kw, cos_sin=torch.zeros(9, 64), positions=_i32(3)))
    assert a.max_tokens == 3
    # (positions of a table buffer that holds more than the batch the view was made for)
    assert lb.qk_args(**dict(kw, cos_sin=torch.zeros(9, 64), positions=_i32(9)[2:4])).max_tokens == 5
    for call in (lambda: lb.qk_norm_rope(a, 4), lambda: lb.kv_append(None, 0, a, None, 4)):
        with pytest.raises(lb.LoraError) as e:
            call()
        assert e.value.status == 1


@pytest.mark.parametrize("bad", [
    dict(q=torch.zeros((5, 512), dtype=torch.float16)), dict(q_weight=_bf16(63)), dict(k_weight=_bf16(128)[::2]),
    dict(k_weight=torch.zeros(64)), dict(positions=torch.zeros(5, dtype=torch.int64)), dict(positions=_i32(10)[::2]),
    dict(cos_sin=torch.zeros(9, 64, dtype=torch.float64)), dict(cos_sin=torch.zeros(9, 128)[:, ::2]),
    dict(num_positions=10), dict(device=0)])
def test_argument_blocks_that_are_refused(bad):
    fused = _bf16(5, 512)
    kw = dict(ROWS, q=fused, k=fused[:, 256:], v=fused[:, 384:], q_out=_bf16(5, 256), k_out=_bf16(5, 128),
              q_weight=_bf16(64), k_weight=_bf16(64), cos_sin=torch.zeros(9, 64), positions=_i32(5))
    lb.qk_args(**kw)
    with pytest.raises(lb.LoraError) as e:
        lb.qk_args(**dict(kw, **bad))
    assert e.value.status == 1
