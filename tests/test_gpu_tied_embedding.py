"""The lookup, its gradient, the norm, clipping and the INT4 product together: a tied
embedding's training step and its logits against 64-bit ones."""
import math

import pytest
import torch

import paper_2501_04266_amd as zq
from paper_2501_04266_amd.tied_embedding import G_BLOCK, W_BLOCK, TiedEmbedding, main, token_ids
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V,D,T,max_norm", [(501, 64, 300, 0.5), (1000, 320, 77, 1e6)])
def test_step(V, D, T, max_norm):
    g = torch.Generator().manual_seed(V)
    start = torch.randn(V, D, generator=g) * 0.02
    emb = TiedEmbedding(start.to(DEV), max_norm=max_norm)
    batches = [token_ids(T, V, b, DEV) for b in range(2)]
    dys = [(torch.randn(T, D, generator=g) / T).bfloat16().to(DEV) for _ in range(2)]

    table = zq.qwz_dequantize(*zq.qwz_quantize(start.view(-1).to(DEV), W_BLOCK), W_BLOCK, out_dtype=torch.float32)
    rows = table.view(V, D)[batches[0]].double()
    # a product and a rounding to bf16
    assert bool(((emb.forward(batches[0]).double() - math.sqrt(D) * rows).abs() <= 2.0**-8 * math.sqrt(D) * rows.abs()).all())

    slices = []
    for b in range(2):
        emb.backward(b, batches[b], dys[b])
        want = torch.zeros(V, D, dtype=torch.float64, device=DEV).index_add_(0, batches[b], dys[b].double())
        mags = torch.zeros_like(want).index_add_(0, batches[b], dys[b].double().abs())
        # at most T additions and a product, each within 2^-24 of the sum of magnitudes
        assert bool(((emb.dw.double() - math.sqrt(D) * want).abs() <= (T + 1) * 2.0**-24 * math.sqrt(D) * mags).all())
        slices.append(zq.qgz_dequantize(emb.sent[b], emb.sent_scales[b], V * D, G_BLOCK).double())

    norm = float(emb.step())
    mean = zq.qgz_dequantize(emb.reduced, emb.reduced_scales, V * D, G_BLOCK).double() / 2
    # the reduce level requantises: half a step of a block's scale, which is its largest / 7
    largest = torch.nn.functional.pad((slices[0] + slices[1]).abs(), (0, -V * D % G_BLOCK)).view(-1, G_BLOCK).amax(1)
    step = (largest / 7).repeat_interleave(G_BLOCK)[:V * D]
    assert bool(((2 * mean - slices[0] - slices[1]).abs() <= 0.5001 * step).all())
    exact = float(mean.norm())
    assert abs(norm - exact) <= 2.0**-22 * exact
    c = min(1.0, max_norm / (exact + 1e-6))
    assert (c < 1.0) == (max_norm < 1.0)
    want = start.view(-1).double().to(DEV) - emb.lr * c * mean
    # clipping and the update: products of binary32 roundings, well within 2^-20 of either term
    assert bool(((emb.master.view(-1).double() - want).abs()
                 <= 2.0**-20 * (start.view(-1).double().to(DEV).abs() + emb.lr * mean.abs())).all())


def test_logits_follow_the_update():
    V, D = 700, 128
    emb = TiedEmbedding((torch.randn(V, D, generator=torch.Generator().manual_seed(1)) * 0.02).to(DEV))
    x = emb.forward(token_ids(3, V, 1, DEV))

    def check():
        w = zq.qgz_dequantize(*zq.qgz_quantize(emb.master.view(-1), G_BLOCK), V * D, G_BLOCK).double().view(V, D)
        mags = x.double().abs() @ w.abs().t()
        assert bool(((emb.logits(x).double() - x.double() @ w.t()).abs() <= (D + 65) * 2.0**-23 * mags).all())

    check()
    ids = token_ids(50, V, 2, DEV)
    for b in range(2):
        emb.backward(b, ids, torch.ones(50, D, dtype=torch.bfloat16, device=DEV))
    emb.step()
    check()


def test_command(capsys):
    main(["--vocab", "1000", "--hidden", "128", "--tokens", "512", "--steps", "3"])
    lines = capsys.readouterr().out.splitlines()
    losses = [float(ln.split("loss ")[1].split()[0]) for ln in lines if ln.startswith("step")]
    assert len(losses) == 3 and losses[2] < losses[0] and lines[-1].startswith("greedy tokens")
