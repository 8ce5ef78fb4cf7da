"""A policy over a tied table trained in its compressed forms: lookups and output product
from the gathered INT8 table, the norm between them, the clipped policy loss at the end,
and the optimizer's step from the reduced INT4 gradient back to the INT8 table.

    python -m paper_2501_04266_amd.tied_policy [--vocab V] [--hidden D] [--rows R] [--steps N]

The policy draws a token from a row's last two tokens: their rows of the table are added,
normed, and multiplied with the table again.  Each step draws a batch with the table as an
INT4 output head (int4_dequant_gemm, token_logp), then trains on it: rms_norm,
qwz_dequant_gemm and policy_loss forward; the logits' gradient, rms_norm_grad and
embedding_grad backward; the gradient as INT4 blocks through a reduce level, its norm with
the norm weight's, and one adamw_step, which clips it, keeps 8-bit moments, updates the
binary32 table and writes the INT8 codes and scales that are gathered next.

Data is synthetic: a token's reward is whether its id is even.
"""
import argparse
import math
import time

import torch

import paper_2501_04266_amd as zq

W_BLOCK, G_BLOCK, STATE_BLOCK = 256, 128, 256


class TiedPolicy:
    """A V x D table (D a multiple of 64), a norm weight, and their optimizer on one GPU."""

    def __init__(self, master, batches=2, lr=1e-3, max_norm=1.0, kl=0.02, clip=(0.2, 0.2), decay=0.01):
        self.V, self.D = master.shape
        self.master, self.batches, self.lr, self.max_norm = master, batches, lr, max_norm
        self.kl, self.clip, self.scale, self.steps = kl, clip, math.sqrt(self.D), 0
        n, dev = master.numel(), master.device
        self.n = n
        self.weight = torch.ones(self.D, device=dev)
        # what the other ranks get: written by the optimizer's step from then on
        self.codes, self.scales = zq.qwz_quantize(master.view(-1), W_BLOCK)
        # gradients: micro-batches' INT4 slices back to back, their sum, the norm weight's
        self.dw = torch.empty((self.V, self.D), dtype=torch.float32, device=dev)
        self.dweight = torch.zeros(self.D, device=dev)
        self.sent = torch.empty((batches, zq.int4_bytes(n)), dtype=torch.uint8, device=dev)
        self.sent_scales = torch.empty((batches, zq.num_scales(n, G_BLOCK)), dtype=torch.float32, device=dev)
        reduced = (torch.empty(zq.int4_bytes(n), dtype=torch.uint8, device=dev),
                   torch.empty(zq.num_scales(n, G_BLOCK), dtype=torch.float32, device=dev), n, G_BLOCK)
        self.reduced = reduced
        self.grads = zq.grad_table([reduced, self.dweight])
        params = [master.view(-1), self.weight]
        m8, v8 = zq.adamw_states(params[:1], 8, STATE_BLOCK)
        m, v = zq.adamw_states(params[1:])
        self.optimizer = zq.adamw_table(params, [reduced, self.dweight], m8 + m, v8 + v,
                                        [(self.codes, self.scales, W_BLOCK), None], weight_decay=[decay, 0.0])
        self.head = None

    def hidden(self, tokens):
        """(normed rows in bf16, what the norm's gradient takes) of tokens [R, 2]."""
        rows = [zq.qwz_embedding(tokens[:, k].contiguous(), self.codes, self.scales, self.V, self.D, W_BLOCK, self.scale)
                for k in (0, 1)]
        y, h, rstd = zq.rms_norm(rows[1], self.weight, rows[0])
        return y, (h, rstd)

    def draw(self, tokens, gen=None):
        """A token for each row, and its log-probability, from the INT4 head."""
        if self.head is None:
            self.head = zq.qgz_quantize(self.master.view(-1), G_BLOCK)
        y, _ = self.hidden(tokens)
        logits = zq.int4_dequant_gemm(y, *self.head, self.V, G_BLOCK)
        noise = -torch.log(-torch.log(torch.rand(logits.shape, generator=gen, device=logits.device).clamp_(1e-9, 1 - 1e-7)))
        token = (logits + noise).argmax(-1)
        return token, zq.token_logp(logits, token)

    def loss_and_grads(self, batch, tokens, drawn, old_logp, advantages, weights, ref_logp):
        """The sums of policy_loss over a micro-batch; its gradients into slice `batch` and
        added to the norm weight's."""
        y, (h, rstd) = self.hidden(tokens)
        logits = zq.qwz_dequant_gemm(y, self.codes, self.scales, self.V, W_BLOCK)
        sums, logp, dlogits = zq.policy_loss(logits, drawn, old_logp, advantages, weights, ref_logp, clip=self.clip,
                                             kl=self.kl, grad_dtype=torch.bfloat16)
        table = zq.qwz_dequantize(self.codes, self.scales, W_BLOCK).view(self.V, self.D)
        dy = dlogits @ table
        torch.mm(dlogits.t().float(), y.float(), out=self.dw)  # the table as output head
        dh, _ = zq.rms_norm_grad(dy, h, self.weight, rstd, dweight=self.dweight, accumulate=True)
        for k in (0, 1):  # and as both rows that were looked up
            zq.embedding_grad(tokens[:, k].contiguous(), dh, self.V, self.scale, out=self.dw, accumulate=True)
        zq.qgz_quantize(self.dw.view(-1), G_BLOCK, packed=self.sent[batch], scales=self.sent_scales[batch])
        return sums, logp

    def step(self):
        """Reduces the slices to their mean and updates; returns the mean's norm."""
        self.steps += 1
        zq.qgz_reduce_level(self.sent.view(-1), self.sent_scales.view(-1), self.batches, self.n, G_BLOCK,
                            packed_out=self.reduced[0], scales_out=self.reduced[1])
        norm = zq.grad_norm(self.grads, 1.0 / self.batches)
        zq.adamw_step(self.optimizer, self.steps, self.lr, norm=norm, max_norm=self.max_norm, scale=1.0 / self.batches)
        self.dweight.zero_()
        self.head = None
        return norm


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--vocab", type=int, default=50000)
    ap.add_argument("--hidden", type=int, default=2048)
    ap.add_argument("--rows", type=int, default=1024, help="of each of two micro-batches")
    ap.add_argument("--steps", type=int, default=4)
    a = ap.parse_args(argv)
    if a.hidden % 64 or min(a.vocab, a.hidden, a.rows, a.steps) < 1:
        ap.error("sizes must be positive, and --hidden a multiple of 64")
    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator().manual_seed(0)
    policy = TiedPolicy((torch.randn(a.vocab, a.hidden, generator=g) * 0.02).to(dev))
    gen = torch.Generator(device=dev).manual_seed(1)
    for i in range(a.steps):
        torch.cuda.synchronize()
        at = time.perf_counter()
        total = torch.zeros(4, device=dev)
        for b in range(policy.batches):
            tokens = torch.randint(0, a.vocab, (a.rows, 2), generator=gen, device=dev)
            drawn, logp = policy.draw(tokens, gen)
            reward = (drawn % 2 == 0).float()
            weights = torch.full((a.rows,), 1.0 / a.rows, device=dev)
            total += policy.loss_and_grads(b, tokens, drawn, logp, reward - reward.mean(), weights, logp)[0]
        norm = policy.step()
        torch.cuda.synchronize()
        loss, _, kl, clipped = (total / policy.batches).tolist()
        print(f"step {i}: loss {loss:.5f}  KL {kl:.5f}  clipped {clipped:.3f}  gradient norm {float(norm):.4f}  "
              f"{(time.perf_counter() - at) * 1e3:.2f} ms")


if __name__ == "__main__":
    main()
