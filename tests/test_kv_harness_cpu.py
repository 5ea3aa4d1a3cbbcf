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

    def storage_offset(self):
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


class Cuda:
    def __init__(self):
        self.on = [Stream(0)]

    def current_stream(self, device=None):
        return self.on[-1]

    default_stream = staticmethod(lambda device=None: Stream(0))
    ExternalStream = Stream
    is_current_stream_capturing = staticmethod(lambda: False)
    synchronize = staticmethod(lambda device=None: None)

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
    _build(c, 500, 11)                           # (a stream's handle as an integer)
    assert c.tables is not old and c.tables.made_on == 11
    assert {7, 9, 0} <= old.kept


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
