"""token_logp and policy_loss on the GPU against the definition in 64 bits."""
import itertools
import math

import pytest
import torch

import paper_2501_04266_amd as zq
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = 2.0**-24  # a binary32 rounding
INF = math.inf


class Case:
    def __init__(self, T, V, dt="f32", seed=0, std=2.0, kl=0.05, scale=1.0, ids=torch.int64, pad=0.2, offset=0, ld=None, clip=(0.2, 0.3)):
        g = torch.Generator().manual_seed(seed * 1000 + V)
        self.scale, self.kl, self.clip = scale, kl, clip
        ld = ld or V
        base = torch.full((T * ld + offset,), math.nan, dtype=DT[dt], device=DEV)
        self.logits = base[offset:].view(T, ld)[:, :V] if T else torch.empty(0, V, dtype=DT[dt], device=DEV)
        self.base = base
        self.logits.copy_(torch.randn(T, V, generator=g) * std)
        self.ids = torch.randint(0, V, (T,), generator=g).to(ids).to(DEV)
        real = torch.log_softmax(self.logits.double() * scale, 1).gather(1, self.ids.long()[:, None])[:, 0] if T else torch.empty(0, device=DEV, dtype=torch.float64)
        self.old = (real + 0.3 * torch.randn(T, generator=g).to(DEV)).float()
        self.ref = (real + 0.3 * torch.randn(T, generator=g).to(DEV)).float() if kl else None
        self.adv = torch.randn(T, generator=g).to(DEV)
        self.w = torch.rand(T, generator=g).to(DEV)
        pads = torch.rand(T, generator=g).to(DEV) < pad
        self.ids[pads] = -1
        self.w[torch.rand(T, generator=g).to(DEV) < pad] = 0

    def call(self, **more):
        return zq.policy_loss(self.logits, self.ids, self.old, self.adv, self.w, self.ref, clip=self.clip, kl=self.kl,
                              scale=self.scale, **more)

    def reference(self):
        """sums, logp, grad in 64 bits, and what binary32 terms may move them by."""
        z = self.logits.double() * self.scale
        T, V = z.shape
        top = z.amax(1, keepdim=True)
        empty = (top[:, 0] == -INF) | (self.ids < 0) | (self.ids >= V)
        d = torch.where(empty[:, None], torch.zeros_like(z), z - top)
        e = torch.exp(d)
        S = e.sum(1, keepdim=True)
        p = e / S
        at = self.ids.long().clamp(0, V - 1)[:, None]
        logp = torch.where(empty, torch.zeros_like(S[:, 0]), (d.gather(1, at) - torch.log(S))[:, 0])
        # the exponent: a difference, two constants (scale times log2 e), a product, each 2^-24 of it;
        # exp2: 2^-22 to be safe of the instruction's 1 ulp; a thread's sum of up to 128 terms
        finite = torch.where(torch.isfinite(d), d, torch.zeros_like(d))
        exp_off = 4 * U * finite.abs() + 2.0**-22
        logp_off = (p * exp_off).sum(1) + 128 * U
        w = torch.where(empty, torch.zeros_like(logp), self.w.double())
        A = self.adv.double()
        r = torch.exp(logp - self.old.double())
        lo, hi = 1 - float(torch.tensor(self.clip[0])), 1 + float(torch.tensor(self.clip[1]))
        clipped = ((A > 0) & (r > hi)) | ((A < 0) & (r < lo))
        # no token may be undecided
        assert bool(((r - lo).abs() > 4 * logp_off)[w > 0].all() and ((r - hi).abs() > 4 * logp_off)[w > 0].all())
        pg = -torch.minimum(r * A, r.clamp(lo, hi) * A)
        slope, slope_off = torch.where(clipped, 0 * A, -A * r), torch.where(clipped, 0 * A, (A * r).abs() * logp_off)
        kl = torch.zeros_like(pg)
        k = float(torch.tensor(self.kl, dtype=torch.float32))
        if self.ref is not None:
            u = self.ref.double() - logp
            kl = torch.exp(u) - u - 1
            slope = slope + k * (1 - torch.exp(u))
            slope_off = slope_off + k * torch.exp(u) * logp_off
        live = w != 0
        pg, kl, slope, slope_off = (torch.where(live, x, torch.zeros_like(x)) for x in (pg, kl, slope, slope_off))
        sums = torch.stack([(w * x).sum() for x in (pg + k * kl, pg, kl, clipped.double())])
        term_off = (w * (slope.abs() + slope_off * 2 + A.abs() * r * live) * logp_off)
        sums_off = 4 * torch.where(live, term_off, torch.zeros_like(term_off)).sum() + 2 * U * (w * (pg.abs() + kl)).sum()
        hot = torch.zeros_like(z).scatter_(1, at, 1.0)
        g = (w * self.scale * slope)[:, None]
        grad = g * (hot - p)
        # the factor's own error; each probability's: its exp, the sum, two more roundings
        grad_off = 2 * (w * self.scale * slope_off)[:, None] * (hot + p) + g.abs() * (p * (exp_off + logp_off[:, None] + 4 * U) + 2 * U * hot)
        grad = torch.where(live[:, None], grad, torch.zeros_like(grad))
        grad_off = torch.where(live[:, None], grad_off, torch.zeros_like(grad))
        return sums, logp, grad, sums_off, logp_off + U * logp.abs(), grad_off

    def check(self, sums, logp, grad, grad_scale=1.0, what=""):
        s, lp, g, s_off, lp_off, g_off = self.reference()
        assert bool(((logp.double() - lp).abs() <= 1.01 * lp_off).all()), f"{what} logp"
        assert bool(((sums.double() - s).abs() <= s_off + U * s.abs() * 2 + 1e-30).all()), f"{what} sums {sums} {s}"
        if grad is None:
            return
        half = torch.finfo(grad.dtype).eps / 2
        # what the type holds of tiny values; exp2's results below 2^-126 are taken as 0
        tiny = torch.finfo(grad.dtype).smallest_normal * half * 2 + 2.0**-125
        want = g * grad_scale
        tol = g_off * abs(grad_scale) + 1.01 * half * want.abs() + tiny
        off = (grad.double() - want).abs()
        assert bool((off <= tol).all()), f"{what} grad: {float((off / tol).max())} of what it may be off by"


VOCABS = [1, 2, 3, 5, 64, 1000, 2047, 2049, 4096, 5001, 8200, 16384, 16411, 24577, 33000, 50000, 65537, 98000, 131072, 140001]


@pytest.mark.parametrize("V", VOCABS)
@pytest.mark.parametrize("dt", DT)
def test_vocabularies(V, dt):
    """Every cut of a row over threads; rows at any element's address."""
    for T, offset in ((1, 0), (6, 3)):
        c = Case(T, V, dt, seed=T, offset=offset)
        sums, logp, grad = c.call()
        c.check(sums, logp, grad, what=f"{T} x {V}")
        assert torch.equal(zq.token_logp(c.logits, c.ids, c.scale), logp)


@pytest.mark.parametrize("dt,gt", itertools.product(DT, DT))
def test_types(dt, gt):
    for ids in (torch.int32, torch.int64):
        c = Case(40, 777, dt, seed=3, ids=ids, scale=1.25)
        sums, logp, grad = c.call(grad_dtype=DT[gt], grad_scale=1024.0)
        assert grad.dtype == DT[gt]
        c.check(sums, logp, grad, 1024.0)
        assert torch.equal(zq.token_logp(c.logits, c.ids, c.scale), logp)


@pytest.mark.parametrize("scale,kl,clip", [(0.5, 0.0, (0.2, 0.2)), (2.0, 0.3, (0.1, 0.28)), (1.0, 0.0, (1.0, 3.0)), (1.0, 0.01, (0.0, 0.0))])
def test_numbers(scale, kl, clip):
    c = Case(500, 300, seed=5, scale=scale, kl=kl, clip=clip)
    c.check(*c.call())
    c.weights, c.w = c.w, torch.ones_like(c.w)
    sums, logp, grad = zq.policy_loss(c.logits, c.ids, c.old, c.adv, None, c.ref, clip=clip, kl=kl, scale=scale)
    c.check(sums, logp, grad)


@pytest.mark.parametrize("dt,V,ld", [("bf16", 50001, 50048), ("f32", 1000, 1003), ("f16", 5, 8), ("bf16", 140001, 140032)])
def test_padded_heads(dt, V, ld):
    """Rows further apart than they are long: what lies between is neither read nor written."""
    c = Case(4, V, dt, ld=ld, offset=1)
    held = torch.full((4, ld), 7.0, dtype=DT[dt], device=DEV)
    sums, logp, grad = c.call(grad=held[:, :V])
    c.check(sums, logp, grad)
    assert bool((held[:, V:] == 7).all())
    assert bool(c.base.view(-1)[1:].view(4, ld)[:, V:].isnan().all())


@pytest.mark.parametrize("V", [700, 50000, 140001])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_gradient_in_place(V, dt):
    c = Case(5, V, dt)
    sums, logp, grad = c.call()
    keep = c.logits.clone()
    s2, l2, g2 = zq.policy_loss(keep, c.ids, c.old, c.adv, c.w, c.ref, clip=c.clip, kl=c.kl, grad=keep)
    assert g2 is keep and torch.equal(g2, grad) and torch.equal(sums, s2) and torch.equal(logp, l2)


def test_without_gradient():
    c = Case(30, 900)
    a, b = c.call(), c.call(grad=False)
    assert b[2] is None and torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("V", [600, 50000, 140001])
def test_masked_logits_and_rows(V):
    """-infinity masks logits; a row of nothing else, an id outside the vocabulary and a
    weight of 0 give no loss and a gradient of zeros, whatever else they hold."""
    c = Case(8, V, "bf16", pad=0.0)
    c.w[:] = 0.5
    c.logits[0, ::2] = -INF
    c.ids[0] = 1
    c.old[0] = c.ref[0] = -3.0
    c.logits[1] = -INF
    c.logits[2, 1:] = -INF  # one token left: certain
    c.ids[2], c.old[2], c.ref[2] = 0, -0.1, -0.05
    c.ids[3], c.ids[4] = V, -7
    c.w[5], c.old[5], c.adv[5] = 0.0, math.nan, INF
    for k in (3, 4):
        c.old[k] = c.adv[k] = c.ref[k] = math.nan
    sums, logp, grad = c.call()
    assert bool(sums.isfinite().all()) and bool(logp.isfinite().all())
    for k in (1, 3, 4):
        assert float(logp[k]) == 0.0
    for k in (1, 3, 4, 5):
        assert not bool(grad[k].any())
    assert not bool(grad[0, ::2].any()) and float(logp[2]) == 0.0 and not bool(grad[2].any())
    safe = Case(8, V, "bf16", pad=0.0)  # the same without what may be anything
    safe.__dict__.update(c.__dict__)
    safe.old, safe.adv, safe.ref = (torch.nan_to_num(x, posinf=0.0) for x in (c.old, c.adv, c.ref))
    s, lp, g, s_off, lp_off, g_off = safe.reference()
    assert bool(((logp.double() - lp).abs() <= 1.01 * lp_off).all())
    assert bool(((sums.double() - s).abs() <= s_off + 2 * U * s.abs()).all())
    assert bool(((grad.double() - g).abs() <= g_off + 2.0**-8 * 1.01 * g.abs() + 1e-37).all())


@pytest.mark.parametrize("V", [600, 50000, 140001])
def test_what_is_not_finite_shows(V):
    """A NaN among a row's logits makes its logp NaN, and the loss; the other rows' are theirs."""
    c = Case(4, V, "f32", pad=0.0)
    clean = c.call()
    c.logits[1, V // 2] = math.nan
    c.logits[2] = -INF
    c.logits[2, V - 1] = math.nan  # no number at all, but no mask either
    sums, logp, grad = c.call()
    assert bool(logp[1].isnan()) and bool(logp[2].isnan()) and bool(sums[0].isnan())
    assert torch.equal(logp[[0, 3]], clean[1][[0, 3]]) and torch.equal(grad[[0, 3]], clean[2][[0, 3]])
    assert bool(grad[1].isnan().any())


def test_the_chosen_token_masked():
    """A chosen token that cannot occur: logp -infinity, ratio 0; without a KL no loss but 0 * A."""
    c = Case(2, 100, kl=0.0, pad=0.0)
    c.logits[0, 7], c.ids[0], c.adv[0] = -INF, 7, 1.0
    sums, logp, grad = c.call()
    assert float(logp[0]) == -INF and not bool(grad[0].any()) and bool(sums.isfinite().all())


def test_large_logits():
    """Differences are taken before scaling: rows far from 0 lose nothing."""
    c = Case(20, 3000, "f32", std=3.0, pad=0.0)
    a = zq.token_logp(c.logits, c.ids)
    shifted = (c.logits * 64).round() / 64  # what +-2^15 still holds exactly
    for shift in (2.0**15, -(2.0**15)):
        assert torch.equal(zq.token_logp(shifted + shift, c.ids), zq.token_logp(shifted, c.ids))
    assert bool(a.isfinite().all())
    huge = torch.tensor([[3e38, -3e38, 0.0]], device=DEV)
    assert zq.token_logp(huge, torch.tensor([0], device=DEV)).tolist() == [0.0]


def test_gradient_against_differences():
    """Central differences of the loss in 64 bits: their own error at a step of 1e-5 is
    about 1e-9 of the terms."""
    c = Case(6, 23, seed=11, pad=0.0, kl=0.1, scale=0.8)
    sums, logp, grad = c.call()

    def loss(z):
        lp = torch.log_softmax(z * c.scale, 1).gather(1, c.ids[:, None])[:, 0]
        r = torch.exp(lp - c.old.double())
        A, u = c.adv.double(), c.ref.double() - lp
        lo, hi = 1 - float(torch.tensor(c.clip[0])), 1 + float(torch.tensor(c.clip[1]))
        return (c.w.double() * (-torch.minimum(r * A, r.clamp(lo, hi) * A) + c.kl * (torch.exp(u) - u - 1))).sum()

    z, d = c.logits.double(), 1e-5
    for i in range(z.numel()):
        e = torch.zeros_like(z)
        e.view(-1)[i] = d
        slope = float((loss(z + e) - loss(z - e)) / (2 * d))
        assert abs(float(grad.view(-1)[i]) - slope) <= 2e-6 * (1 + abs(slope))


def test_same_bits_again_and_no_rows():
    c = Case(3000, 501)
    a, b = c.call(), c.call()
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    none = Case(0, 64)
    sums, logp, grad = none.call()
    assert sums.tolist() == [0.0] * 4 and logp.shape == (0,) and grad.shape == (0, 64)
    assert zq.token_logp(none.logits, none.ids).shape == (0,)


def test_graph_and_streams():
    c = Case(200, 5000, "bf16")
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    c.call()  # the same leaves, eagerly, before the capture
    with torch.cuda.graph(graph, stream=side):
        got = c.call()
        alone = zq.token_logp(c.logits, c.ids)
    for turn in range(3):
        c.logits.normal_()
        graph.replay()
        torch.cuda.synchronize()
        want = c.call()
        assert all(torch.equal(x, y) for x, y in zip(got, want)), f"replay {turn}"
        assert torch.equal(alone, zq.token_logp(c.logits, c.ids)), f"replay {turn}"
    other = c.call(stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(other, want))


def test_rows_beyond_2_32_elements():
    T, V = 2**32 // 50000 + 3, 50000
    logits = torch.zeros(T, V, dtype=torch.bfloat16, device=DEV)
    logits[-2:] = (torch.randn(2, V, generator=torch.Generator().manual_seed(1)) * 2).bfloat16().to(DEV)
    ids = torch.arange(T, device=DEV) % V
    zeros, adv = torch.zeros(T, device=DEV), torch.ones(T, device=DEV)
    small = logits[-2:].clone()
    want = zq.policy_loss(small, ids[-2:].contiguous(), zeros[-2:].contiguous(), adv[-2:].contiguous(), clip=(1.0, 100.0))
    sums, logp, grad = zq.policy_loss(logits, ids, zeros, adv, clip=(1.0, 100.0), grad=logits)
    assert torch.equal(logp[-2:], want[1]) and torch.equal(grad[-2:], want[2])
    assert bool(((logp[:-2] + math.log(V)).abs() <= 2.0**-20).all())


@pytest.mark.parametrize("V", [1000, 50001, 140001])
def test_gradient_in_place_of_a_padded_head(V):
    c = Case(5, V, "bf16", ld=V + 15)
    sums, logp, grad = c.call()
    s2, l2, g2 = c.call(grad=c.logits)
    assert g2 is c.logits and torch.equal(g2, grad) and torch.equal(sums, s2) and torch.equal(logp, l2)
    assert bool(c.base.view(5, V + 15)[:, V:].isnan().all())


def test_shapes_of_rows():
    """One row alone, and rows in more dimensions."""
    c = Case(12, 70, kl=0.0)
    sums, logp, grad = c.call()
    s2, l2, g2 = zq.policy_loss(c.logits.view(3, 4, 70), c.ids.view(3, 4), c.old.view(3, 4), c.adv.view(3, 4), c.w.view(3, 4),
                                clip=c.clip)
    assert torch.equal(s2, sums) and torch.equal(l2.view(-1), logp) and torch.equal(g2.view(12, 70), grad)
    one = zq.token_logp(c.logits[5], c.ids[5])
    assert one.shape == () and float(one) == float(logp[5])


def test_no_slope():
    """A loss scale of 0, and clipped tokens without a KL term: gradients of zeros."""
    c = Case(40, 300, kl=0.0)
    assert not bool(c.call(grad_scale=0.0)[2].any())
    c.old -= 5.0  # ratios far beyond the clip
    c.adv.abs_()
    sums, logp, grad = c.call()
    assert not bool(grad.any()) and float(sums[3]) > 0
