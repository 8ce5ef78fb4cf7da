"""What the norm, its gradient and the loss do about the memory they allocate themselves on
another stream than the current one, with the streams, the allocator and the library
replaced by records (no GPU): as the calls around the path do."""
import pytest
import torch

import paper_2501_04266_amd as zq
from paper_2501_04266_amd import _lib
from tests.test_binding_streams import Stream, log  # noqa: F401  -- the fixture


@pytest.fixture(autouse=True)
def _anywhere(monkeypatch):
    monkeypatch.setattr(_lib, "_here", lambda **tensors: None)
    monkeypatch.setattr(_lib, "_logits", lambda t, name, dtypes, rows=None: (4096, t.shape[0], t.shape[1], t.shape[1]))


X, W, RSTD = torch.zeros(4, 64), torch.ones(64), torch.zeros(4)
IDS, ROW = torch.zeros(4, dtype=torch.int64), torch.zeros(4)
CALLS = {
    "rms_norm": lambda s: zq.rms_norm(X, W, X, stream=s),
    "qwz_rms_norm": lambda s: zq.qwz_rms_norm(X, W, X, block=32, stream=s),
    "rms_norm_grad": lambda s: zq.rms_norm_grad(X, X, W, RSTD, stream=s),
    "token_logp": lambda s: zq.token_logp(X, IDS, stream=s),
    "policy_loss": lambda s: zq.policy_loss(X, IDS, ROW, ROW, stream=s),
}


@pytest.mark.parametrize("kind", ["stream", "handle"])
@pytest.mark.parametrize("name", CALLS)
def test_memory_of_a_call_on_another_stream(log, name, kind):  # noqa: F811
    CALLS[name](Stream(7, log) if kind == "stream" else 7)
    call = [i for i, e in enumerate(log) if e[0] == "call"]
    assert len(call) == 1 and log[call[0]][2] == 7
    assert ("empty", "workspace", 1) not in log, "a workspace from the current stream's pool"
    outs = [i for i, e in enumerate(log) if e == ("empty", "output", 1)]
    waits = [i for i, e in enumerate(log) if e == ("wait", 7, 1)]
    assert outs and waits and outs[-1] < waits[-1] < call[0], "the output's memory may have pending work"
    assert (("record", "output", 7) in log) == (kind == "stream")


@pytest.mark.parametrize("name", CALLS)
def test_memory_of_a_call_on_the_current_stream(log, name):  # noqa: F811
    for stream in (None, Stream(1, log), 1):
        log.clear()
        CALLS[name](stream)
        assert [e[0] for e in log if e[0] in ("wait", "record")] == []
        assert all(e[2] == 1 for e in log if e[0] == "empty")


def test_given_buffers_keep_the_streams_apart(log):  # noqa: F811
    """With outputs and workspace given, a call waits for nothing."""
    other = Stream(7, log)
    zq.rms_norm(X, W, X, out=torch.zeros(4, 64), hidden=torch.zeros(4, 64), rstd=ROW, stream=other)
    zq.rms_norm_grad(X, X, W, RSTD, out=torch.zeros(4, 64), dweight=torch.zeros(64),
                     workspace=torch.zeros(4096, dtype=torch.uint8), stream=other)
    zq.token_logp(X, IDS, out=torch.zeros(4), stream=other)
    assert [e[0] for e in log] == ["call"] * 3
