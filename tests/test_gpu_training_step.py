"""The norm, the loss, their gradients and the optimizer's step together, as tied_policy
runs them, against 64 bits; and the whole of them captured into one graph."""
import math

import pytest
import torch

import paper_2501_04266_amd as zq
from paper_2501_04266_amd.tied_policy import G_BLOCK, STATE_BLOCK, W_BLOCK, TiedPolicy, main
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu


def batch(V, R, seed):
    g = torch.Generator().manual_seed(seed)
    tokens = torch.randint(0, V, (R, 2), generator=g).to(DEV)
    tokens[3] = tokens[4]  # a row that occurs twice, and one token twice in a row
    tokens[5, 1] = tokens[5, 0]
    drawn = torch.randint(0, V, (R,), generator=g).to(DEV)
    drawn[7] = -1
    adv = torch.randn(R, generator=g).to(DEV)
    w = torch.full((R,), 1.0 / R)
    w[9] = 0.0
    return tokens, drawn, adv, w.to(DEV)


def reference(policy, tokens, drawn, old, adv, w, ref):
    """loss and gradients of the table and the norm's weight by autograd in 64 bits, from
    the INT8 table as it stands for values."""
    V, D = policy.V, policy.D
    table = zq.qwz_dequantize(policy.codes, policy.scales, W_BLOCK, torch.float32).view(V, D).double().requires_grad_()
    weight = policy.weight.double().requires_grad_()
    h = (table[tokens[:, 0]] + table[tokens[:, 1]]) * policy.scale
    y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + 1e-6) * weight
    logp_all = torch.log_softmax(y @ table.t().contiguous(), 1)
    real = drawn >= 0
    logp = torch.where(real, logp_all.gather(1, drawn.clamp(min=0)[:, None])[:, 0], torch.zeros_like(old.double()))
    r, A, u = torch.exp(logp - old.double()), adv.double(), ref.double() - logp
    each = -torch.minimum(r * A, r.clamp(1 - policy.clip[0], 1 + policy.clip[1]) * A) + policy.kl * (torch.exp(u) - u - 1)
    loss = (torch.where(real, w.double(), torch.zeros_like(r)) * each).sum()
    loss.backward()
    return loss.detach(), logp.detach(), table.grad, weight.grad


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


@pytest.mark.parametrize("V,D,R", [(501, 128, 60), (1000, 320, 333)])
def test_gradients_and_step(V, D, R):
    g = torch.Generator().manual_seed(V)
    start = torch.randn(V, D, generator=g) * 0.02
    policy = TiedPolicy(start.to(DEV), max_norm=0.05, lr=0.01)
    kept = []
    for b in range(2):
        tokens, drawn, adv, w = batch(V, R, b)
        y, _ = policy.hidden(tokens)
        old = zq.token_logp(zq.qwz_dequant_gemm(y, policy.codes, policy.scales, V, W_BLOCK), drawn)
        ref = old + 0.1
        sums, logp = policy.loss_and_grads(b, tokens, drawn, old - 0.05, adv, w, ref)
        loss, logp64, dtable, dweight = reference(policy, tokens, drawn, old - 0.05, adv, w, ref)
        # looked-up rows, the normed row, the weight's values and the logits' gradient are
        # rounded to bf16 (2^-9 of each, some of them twice on the way), as is the gradient of
        # y: in all well within 8 of 2^-8 of any of the results' norms
        tol = 8 * 2.0**-8
        assert off(sums[0], loss) < tol and float((logp - logp64).abs().max()) < tol * 8
        assert off(policy.dw, dtable) < tol, off(policy.dw, dtable)
        kept.append((policy.dw.clone(), dweight))
    assert off(policy.dweight, kept[0][1] + kept[1][1]) < tol
    dweight = policy.dweight.clone()

    norm = policy.step()
    mean = zq.qgz_dequantize(*policy.reduced[:2], V * D, G_BLOCK).double() / 2
    exact = math.sqrt(float(mean.square().sum() + (dweight.double() / 2).square().sum()))
    assert abs(float(norm) - exact) <= 2.0**-22 * exact
    # the first step: m = 0.1 g, v = 0.001 g^2, the corrections take both factors out
    c = min(1.0, 0.05 / (exact + 1e-6))
    for param, p0, grad, decay in ((policy.master.view(-1), start.view(-1).to(DEV), mean, 0.01),
                                   (policy.weight, torch.ones(D, device=DEV), dweight.double() / 2, 0.0)):
        want = p0.double() * (1 - 0.01 * decay) - 0.01 * (c * grad) / ((c * grad).abs() + 1e-8)
        # binary32 roundings of the update (at most 0.01; some 30 of them) and of the weight
        assert bool(((param.double() - want).abs() <= 32 * 2.0**-24 * 0.01 + 4 * 2.0**-24 * p0.double().abs()).all())
    # the table that is gathered next is the new one
    codes, scales = zq.qwz_quantize(policy.master.view(-1), W_BLOCK)
    assert torch.equal(codes, policy.codes) and torch.equal(scales, policy.scales)
    # 8-bit moments: within a step of their codes (an eighth, a quarter) of the unrounded
    m8, v8 = policy.optimizer.tensors[2][0], policy.optimizer.tensors[3][0]
    cg = (c * mean).cpu()
    for (q, s, block), value, step, least in ((m8, 0.1 * cg, 1 / 8, 2.0**-9), (v8, 0.001 * cg.square(), 1 / 4, 2.0**-16)):
        assert block == STATE_BLOCK
        scale = s.double().cpu().repeat_interleave(block)[:V * D]
        held = q.cpu().float().double() * scale
        assert bool(((held - value).abs() <= 1.001 * step * value.abs() + 1.001 * least * scale).all())


def test_drawing():
    V, D = 700, 128
    policy = TiedPolicy((torch.randn(V, D, generator=torch.Generator().manual_seed(1)) * 0.1).to(DEV))
    tokens = torch.randint(0, V, (5, 2), generator=torch.Generator().manual_seed(2)).to(DEV)
    token, logp = policy.draw(tokens, torch.Generator(device=DEV).manual_seed(3))
    y, _ = policy.hidden(tokens)
    table = zq.qgz_dequantize(*policy.head, V * D, G_BLOCK).double().view(V, D)
    want = torch.log_softmax(y.double() @ table.t().contiguous(), 1).gather(1, token[:, None])[:, 0]
    assert bool(((logp.double() - want).abs() <= 1e-4).all())  # (D + 64) 2^-23 of logits' terms, a few hundred


def test_one_graph():
    """Norm, loss, gradients, reduction and the optimizer's step in one captured graph, with the
    count of steps on the device; replays with eager work between them give the eager
    program's bits."""
    V, D, R = 600, 128, 100

    def program(policy, x):
        """Without the library's own products (the logits come in)."""
        y, h, rstd = zq.rms_norm(x["x"], policy.weight, x["res"])
        sums, logp, dz = zq.policy_loss(x["logits"], x["ids"], x["old"], x["adv"], None, x["old"], kl=0.1,
                                        grad_dtype=torch.bfloat16)
        dh, _ = zq.rms_norm_grad(x["dy"], h, policy.weight, rstd, dweight=policy.dweight, accumulate=True)
        for b in (0, 1):
            zq.embedding_grad(x["rows"], dh, V, out=policy.dw)
            zq.qgz_quantize(policy.dw.view(-1), G_BLOCK, packed=policy.sent[b], scales=policy.sent_scales[b])
        zq.qgz_reduce_level(policy.sent.view(-1), policy.sent_scales.view(-1), 2, V * D, G_BLOCK,
                            packed_out=policy.reduced[0], scales_out=policy.reduced[1])
        norm = zq.grad_norm(policy.grads, 0.5)
        return y, sums, logp, dz, dh, norm

    def inputs(seed):
        g = torch.Generator().manual_seed(seed)
        x = {k: torch.randn(R, D, generator=g).bfloat16().to(DEV) for k in ("x", "res", "dy")}
        x.update(logits=torch.randn(R, V, generator=g).to(DEV), ids=torch.randint(0, V, (R,), generator=g).to(DEV),
                 rows=torch.randint(0, V, (R,), generator=g).to(DEV), old=torch.full((R,), -6.0, device=DEV),
                 adv=torch.randn(R, generator=g).to(DEV))
        return x

    start = (torch.randn(V, D, generator=torch.Generator().manual_seed(0)) * 0.02).to(DEV)
    a, b = TiedPolicy(start.clone()), TiedPolicy(start.clone())
    held = inputs(0)
    count, rate = torch.zeros(1, dtype=torch.int64, device=DEV), torch.full((1,), 1e-3, device=DEV)
    program(TiedPolicy(start.clone()), held)  # the same inputs, eagerly, before the capture
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        got = program(a, held)
        count.add_(1)
        zq.adamw_step(a.optimizer, count, rate, norm=got[-1], max_norm=1.0, scale=0.5)
        a.dweight.zero_()
    for t in (1, 2, 3):
        new = inputs(t)
        for k, v in held.items():
            v.copy_(new[k])
        graph.replay()
        torch.cuda.synchronize()
        want = program(b, new)
        zq.adamw_step(b.optimizer, t, float(rate), norm=want[-1], max_norm=1.0, scale=0.5)
        b.dweight.zero_()
        for x, y in zip(got, want):
            assert torch.equal(x, y), f"replay {t}"
        assert torch.equal(a.master, b.master) and torch.equal(a.codes, b.codes) and torch.equal(a.weight, b.weight)
        for k in (2, 3):
            assert torch.equal(a.optimizer.tensors[k][0][0].view(torch.uint8), b.optimizer.tensors[k][0][0].view(torch.uint8))


def test_command(capsys):
    main(["--vocab", "1000", "--hidden", "128", "--rows", "64", "--steps", "2"])
    lines = capsys.readouterr().out.splitlines()
    assert [ln.split(":")[0] for ln in lines] == ["step 0", "step 1"]
    assert all(math.isfinite(float(ln.split("loss ")[1].split()[0])) for ln in lines)
