"""A tied embedding table trained and used in its compressed forms: the lookup, its
gradient, the gradients' norm and clipping, and the output product with INT4 weights,
as one program calls them around the qwZ / qgZ path.

    python -m paper_2501_04266_amd.tied_embedding [--vocab V] [--hidden D] [--tokens T] [--steps N]

The table is kept in binary32 by its owner.  What the other ranks would gather is its
INT8 form (qwz_quantize), and the lookup reads that as it is.  Each of P micro-batches
(they stand for P ranks' shares) gives a dense gradient, which travels as INT4 blocks
(qgz_quantize) into one reduce level; its INT4 result is measured and clipped without a
dequantised copy, and comes out in binary32 for the update.  For generation the table
is the output head too, as INT4 codes and scales; a token then costs one read of them.

Data and gradients are synthetic: token ids of frequency 1 / rank, and the gradient of
0.5 * |y - target|^2 at the embedding's output.
"""
import argparse
import math
import time

import torch

import paper_2501_04266_amd as zq

W_BLOCK, G_BLOCK = 256, 128


class TiedEmbedding:
    """A V x D table (D a multiple of 64) and its compressed forms on one GPU."""

    def __init__(self, master, batches=2, lr=0.1, max_norm=1.0):
        self.V, self.D = master.shape
        self.master, self.lr, self.max_norm, self.batches = master, lr, max_norm, batches
        n, dev = master.numel(), master.device
        self.n, self.scale = n, math.sqrt(self.D)
        self.codes = torch.empty(n, dtype=torch.int8, device=dev)
        self.scales = torch.empty(zq.num_scales(n, W_BLOCK), dtype=torch.float32, device=dev)
        # the micro-batches' slices, back to back as qgz_reduce_level reads them
        self.dw = torch.empty((self.V, self.D), dtype=torch.float32, device=dev)
        self.sent = torch.empty((batches, zq.int4_bytes(n)), dtype=torch.uint8, device=dev)
        self.sent_scales = torch.empty((batches, zq.num_scales(n, G_BLOCK)), dtype=torch.float32, device=dev)
        self.reduced = torch.empty(zq.int4_bytes(n), dtype=torch.uint8, device=dev)
        self.reduced_scales = torch.empty(zq.num_scales(n, G_BLOCK), dtype=torch.float32, device=dev)
        # the gradient stays in one place, so its table is made once; clipping writes dw
        self.grads = zq.grad_table([(self.reduced, self.reduced_scales, n, G_BLOCK)], [self.dw])
        self.norm = torch.empty(1, dtype=torch.float32, device=dev).view(())
        self.head = None
        self.gather()

    def gather(self):
        """The table as the other ranks get it."""
        zq.qwz_quantize(self.master.view(-1), W_BLOCK, codes=self.codes, scales=self.scales)

    def forward(self, ids, out_dtype=torch.bfloat16):
        return zq.qwz_embedding(ids, self.codes, self.scales, self.V, self.D, W_BLOCK, self.scale, out_dtype)

    def backward(self, batch, ids, dy):
        """Micro-batch `batch`'s gradient into its slice."""
        zq.embedding_grad(ids, dy, self.V, self.scale, out=self.dw)
        zq.qgz_quantize(self.dw.view(-1), G_BLOCK, packed=self.sent[batch], scales=self.sent_scales[batch])

    def step(self):
        """Reduces the slices to their mean, clips it and updates the table; returns the
        mean's norm (on the GPU, in a buffer that the next step writes)."""
        zq.qgz_reduce_level(self.sent.view(-1), self.sent_scales.view(-1), self.batches, self.n, G_BLOCK,
                            packed_out=self.reduced, scales_out=self.reduced_scales)
        zq.grad_norm(self.grads, 1.0 / self.batches, out=self.norm)
        zq.grad_clip(self.grads, self.norm, self.max_norm, 1.0 / self.batches)
        self.master.sub_(self.dw, alpha=self.lr)
        self.gather()
        self.head = None
        return self.norm

    def logits(self, x):
        """The output head for a few rows x (bf16 / fp16 [M, D]): binary32 [M, V]."""
        if self.head is None:
            self.head = zq.qgz_quantize(self.master.view(-1), G_BLOCK)
        return zq.int4_dequant_gemm(x, *self.head, self.V, G_BLOCK)


def token_ids(T, V, seed, device):
    """T ids of frequency about 1 / rank."""
    u = torch.rand(T, generator=torch.Generator().manual_seed(seed))
    return (torch.exp(u * math.log(V + 1)).long() - 1).clamp_(0, V - 1).to(device)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--vocab", type=int, default=50000)
    ap.add_argument("--hidden", type=int, default=2048)
    ap.add_argument("--tokens", type=int, default=8192, help="of each of two micro-batches")
    ap.add_argument("--steps", type=int, default=8)
    a = ap.parse_args(argv)
    if a.hidden % 64 or min(a.vocab, a.hidden, a.tokens, a.steps) < 1:
        ap.error("sizes must be positive, and --hidden a multiple of 64")
    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator().manual_seed(0)
    emb = TiedEmbedding((torch.randn(a.vocab, a.hidden, generator=g) * 0.02).to(dev))
    target = torch.randn(a.hidden, generator=g).to(dev)
    batches = [token_ids(a.tokens, a.vocab, 1 + b, dev) for b in range(emb.batches)]

    def train_step():
        loss = 0.0
        for b, ids in enumerate(batches):
            diff = emb.forward(ids).float() - target
            loss = loss + 0.5 * diff.square().sum() / a.tokens
            emb.backward(b, ids, (diff / a.tokens).bfloat16())
        return loss / emb.batches, emb.step()

    for i in range(a.steps):
        torch.cuda.synchronize()
        at = time.perf_counter()
        loss, norm = train_step()
        torch.cuda.synchronize()
        print(f"step {i}: loss {float(loss):.4f}  gradient norm {float(norm):.4f}  {(time.perf_counter() - at) * 1e3:.2f} ms")

    token, said = batches[0][:1], []
    for _ in range(8):
        token = emb.logits(emb.forward(token)).argmax(-1)
        said.append(int(token))
    print("greedy tokens:", said)


if __name__ == "__main__":
    main()
