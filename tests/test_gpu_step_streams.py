"""The norm, its gradient and the loss on another stream than the current one, while the
current one still has work on memory that was freed: that work must not reach the call's
workspace or outputs."""
import pytest
import torch

import paper_2501_04266_amd as zq
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu


def pending(sizes):
    """Work on the current stream that takes some milliseconds and then writes freed
    memory of these sizes."""
    a = torch.ones(4096, 4096, device=DEV)
    for _ in range(20):
        a = a @ a * 0.0
    for n in sizes:
        torch.empty(n, dtype=torch.uint8, device=DEV).fill_(0x7F)


def rows(seed):
    return torch.randn(700, 520, generator=torch.Generator().manual_seed(seed)).bfloat16().to(DEV)


X, W = (700, 520), 520


def norm():
    x, r, w = rows(1), rows(2), torch.ones(W, device=DEV)
    return (lambda **k: zq.rms_norm(x, w, r, **k)), [700 * 520 * 2, 700 * 520 * 2, 2800]


def int8_norm():
    x, r, w = rows(1), rows(2), torch.ones(W, device=DEV)
    return (lambda **k: zq.qwz_rms_norm(x[:, :512].contiguous(), w[:512].contiguous(), block=128, **k)), [700 * 512, 700 * 16, 2800]


def gradient():
    h, dy, w = rows(1), rows(2), torch.ones(W, device=DEV)
    rstd = torch.ones(700, device=DEV)
    return ((lambda **k: zq.rms_norm_grad(dy, h, w, rstd, **k)),
            [700 * 520 * 2, 2080, zq.rms_norm_grad_bytes(700, 520)])


def loss():
    z, ids, f = rows(1), torch.arange(700, device=DEV) % 520, torch.full((700,), -6.0, device=DEV)
    adv = torch.randn(700, generator=torch.Generator().manual_seed(3)).to(DEV)
    return ((lambda **k: zq.policy_loss(z, ids, f, adv, **k)), [700 * 520 * 2, 16, 2800, zq.policy_loss_bytes(700)])


def logp():
    z, ids = rows(1), torch.arange(700, device=DEV) % 520
    return (lambda **k: (zq.token_logp(z, ids, **k),)), [2800]


@pytest.mark.parametrize("make", [norm, int8_norm, gradient, loss, logp])
@pytest.mark.parametrize("kind", ["stream", "handle"])
def test_pending_work_on_freed_memory(make, kind):
    call, sizes = make()
    want = call()
    torch.cuda.synchronize()
    for _ in range(3):
        side = torch.cuda.Stream()
        pending(sizes)
        got = call(stream=side if kind == "stream" else side.cuda_stream)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_two_streams_at_once():
    """Calls on two streams share nothing."""
    call, _ = gradient()
    other, _ = loss()
    want, want_other = call(), other()
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    got = [(call(stream=a), other(stream=b), call(stream=b), other(stream=a)) for _ in range(8)]
    torch.cuda.synchronize()
    for g1, l1, g2, l2 in got:
        assert all(torch.equal(x, y) for x, y in zip(g1, want)) and all(torch.equal(x, y) for x, y in zip(g2, want))
        assert all(torch.equal(x, y) for x, y in zip(l1, want_other)) and all(torch.equal(x, y) for x, y in zip(l2, want_other))
