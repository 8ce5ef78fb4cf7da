"""What a call on another stream than the current one does about the memory it
allocates itself, with the streams, the allocator and the library replaced by records
(no GPU): a workspace comes from the pool of the call's stream; an output comes from
the current stream's, so the call's stream first waits for the work pending there, and
the allocator hears of a stream object's use.  Without that, memory freed with work on it still
pending is written by that work while the call uses it."""
import contextlib
import ctypes
import sys

import pytest
import torch

import paper_2501_04266_amd as zq
from paper_2501_04266_amd import _lib


class Stream:
    def __init__(self, cuda_stream, log):
        self.cuda_stream, self.log = cuda_stream, log

    def wait_stream(self, other):
        self.log.append(("wait", self.cuda_stream, other.cuda_stream))


class Memory(torch.Tensor):
    """A tensor that says on which streams it is recorded."""
    log = None
    is_cuda = True

    def record_stream(self, stream):
        self.log.append(("record", self.kind, stream.cuda_stream))


class Torch:
    """torch with the streams of this test; `empty` notes the stream it is called on."""

    def __init__(self, log):
        self.log, self.cuda = log, self
        self.now = Stream(1, log)

    def __getattr__(self, name):
        return getattr(torch, name)

    def current_stream(self, device=None):
        return self.now

    def ExternalStream(self, handle, device=None):
        return Stream(handle, self.log)

    @contextlib.contextmanager
    def stream(self, stream):
        before, self.now = self.now, stream
        yield
        self.now = before

    def empty(self, *size, dtype=None, device=None):
        t = torch.empty(*size, dtype=dtype).as_subclass(Memory)
        t.log, t.kind = self.log, "workspace" if sys._getframe(1).f_code.co_name == "_workspace" else "output"
        self.log.append(("empty", t.kind, self.now.cuda_stream))
        return t


class Library:
    def __init__(self, log):
        self.log = log

    def __getattr__(self, name):
        def call(*args):
            if name.endswith("_bytes"):
                return 4096
            self.log.append(("call", name, args[-1]))
            return 0
        return call


@pytest.fixture
def log(monkeypatch):
    log = []
    monkeypatch.setattr(_lib, "torch", Torch(log))
    monkeypatch.setattr(_lib, "lib", lambda: Library(log))
    monkeypatch.setattr(_lib, "_dev", lambda t, name: 4096)
    monkeypatch.setattr(_lib, "_ptr", lambda t, name, count, dtypes: 4096)
    monkeypatch.setattr(_lib, "_stream", lambda s: 1 if s is None else getattr(s, "cuda_stream", s))
    return log


IDS, DY, TABLE = torch.zeros(6, dtype=torch.int64), torch.zeros(6, 8), torch.zeros(10, 8)
X, CODES = torch.zeros(2, 64, dtype=torch.bfloat16), torch.zeros(64, dtype=torch.uint8)
GRADS = zq.GradTable([DY], [None], _lib._GradPlan(), torch.zeros(64, dtype=torch.uint8))
U8, F32 = torch.zeros(128, dtype=torch.uint8), torch.zeros(128)
CALLS = {
    "qwz_quantize": lambda s: zq.qwz_quantize(DY, 32, stream=s),
    "qwz_dequantize": lambda s: zq.qwz_dequantize(torch.zeros(64, dtype=torch.int8), F32, 32, stream=s),
    "qgz_quantize": lambda s: zq.qgz_quantize(DY, 32, stream=s),
    "qgz_dequantize": lambda s: zq.qgz_dequantize(U8, F32, 64, 32, stream=s),
    "qgz_reduce_level": lambda s: zq.qgz_reduce_level(U8, F32, 2, 64, 32, stream=s),
    "qgz_reduce_dequantize": lambda s: zq.qgz_reduce_dequantize(U8, F32, 2, 64, 32, stream=s),
    "qgz_reduce_level_gather": lambda s: zq.qgz_reduce_level_gather([U8, U8], [F32, F32], 64, 32, stream=s,
                                                                    tables=(IDS, IDS)),
    "qwz_dequant_gemm": lambda s: zq.qwz_dequant_gemm(X, torch.zeros(128, dtype=torch.int8), F32, 2, 32, stream=s),
    "embedding": lambda s: zq.embedding(IDS, TABLE, stream=s),
    "qwz_embedding": lambda s: zq.qwz_embedding(IDS, torch.zeros(80, dtype=torch.int8), torch.zeros(1), 10, 8, stream=s),
    "embedding_grad": lambda s: zq.embedding_grad(IDS, DY, 10, stream=s),
    "grad_norm": lambda s: zq.grad_norm(GRADS, stream=s),
    "int4_dequant_gemm": lambda s: zq.int4_dequant_gemm(X, CODES, torch.zeros(4), 2, 32, stream=s),
}


@pytest.mark.parametrize("kind", ["stream", "handle"])
@pytest.mark.parametrize("name", CALLS)
def test_memory_of_a_call_on_another_stream(log, name, kind):
    CALLS[name](Stream(7, log) if kind == "stream" else 7)
    call = [i for i, e in enumerate(log) if e[0] == "call"]
    assert len(call) == 1 and log[call[0]][2] == 7
    assert ("empty", "workspace", 1) not in log, "a workspace from the current stream's pool"
    outs = [i for i, e in enumerate(log) if e == ("empty", "output", 1)]
    waits = [i for i, e in enumerate(log) if e == ("wait", 7, 1)]
    assert outs and waits and outs[-1] < waits[-1] < call[0], "the output's memory may have pending work"
    # a handle's stream may be gone when the output is freed
    assert (("record", "output", 7) in log) == (kind == "stream")


@pytest.mark.parametrize("name", CALLS)
def test_memory_of_a_call_on_the_current_stream(log, name):
    for stream in (None, Stream(1, log), 1):
        log.clear()
        CALLS[name](stream)
        assert [e[0] for e in log if e[0] in ("wait", "record")] == []
        assert all(e[2] == 1 for e in log if e[0] == "empty")


def test_given_buffers_keep_the_streams_apart(log):
    """With the output and the workspace given, a call waits for nothing."""
    zq.embedding_grad(IDS, DY, 10, out=torch.zeros(10, 8), workspace=torch.zeros(4096, dtype=torch.uint8),
                      stream=Stream(7, log))
    assert [e[0] for e in log] == ["call"]


def test_table_made_for_a_call(log, monkeypatch):
    """The table of a list of gradients stays until the call's stream has passed it."""
    table = torch.zeros(64, dtype=torch.uint8).as_subclass(Memory)
    table.log, table.kind = log, "table"
    monkeypatch.setattr(_lib, "grad_table", lambda g: zq.GradTable(g, [None], _lib._GradPlan(), table))
    zq.grad_norm([DY], out=torch.zeros(()), stream=7)
    assert ("record", "table", 7) in log
    assert ctypes.sizeof(_lib._GradPlan) == 32
