"""token_logp and policy_loss where the result is infinite, or nearly nothing."""
import itertools
import math

import pytest
import torch

import paper_2501_04266_amd as zq
from tests.gpu_util import DEV
from tests.test_gpu_policy_loss import DT, INF, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V,dt", itertools.product([600, 50000, 140001], DT))
@pytest.mark.parametrize("kl", [0.0, 0.05])
def test_the_chosen_token_masked_with_a_reference(V, dt, kl):
    """An infinite KL term: its token's logp is -infinity (or far below the others), the sums
    that hold it are infinite, and no NaN is anywhere.  Rows 0 and 1 have a masked token
    (in row 1 the other policies mask it too), row 3 one that is too unlikely for binary64."""
    c = Case(4, V, dt, pad=0.0, kl=0.05)
    c.kl, c.w[:] = kl, 0.5
    c.adv.copy_(torch.tensor([1.0, -1.0, 0.5, 0.25]))
    clean = c.call()
    alone = c.w.clone()
    alone[[0, 1, 3]] = 0.0
    alone = zq.policy_loss(c.logits, c.ids, c.old, c.adv, alone, c.ref, clip=c.clip, kl=kl)[0]
    c.logits[:2, ::2] = -INF
    c.logits[:2, 5] = -300.0  # an exponential of 0 without a mask
    c.ids[:2] = 2
    c.old[1] = c.ref[1] = -INF
    c.ids[3], c.logits[3, 7], c.old[3], c.ref[3] = 7, -900.0, -INF, -0.5
    c.adv[3] = 1.0  # and a ratio beyond the clip
    sums, logp, grad = c.call()
    assert logp[:2].tolist() == [-INF, -INF] and float(logp[3]) < -800
    assert float(sums[2]) == INF and (float(sums[0]) == INF) == (kl > 0) and bool(sums[1].isfinite())
    # -min(r A, clip(r) A) with r = 0, and with r beyond the clip
    lo, hi = 1 - float(torch.tensor(c.clip[0])), 1 + float(torch.tensor(c.clip[1]))
    want = float(alone[1]) + 0.5 * (0.0 + lo - hi)
    assert abs(float(sums[1]) - want) <= 2.0**-22 * (abs(want) + lo + hi)
    assert float(sums[3]) == float(alone[3]) + 1.0
    assert not bool(grad.isnan().any()) and torch.equal(grad[2], clean[2][2])
    if kl == 0:
        assert not bool(grad[[0, 1, 3]].any())
    else:
        # the others' exponentials are above 2^-126: logits of a few units
        live = torch.ones(V, dtype=torch.bool, device=DEV)
        live[::2] = live[5] = False
        for k in (0, 1):
            assert bool((grad[k][live] == INF).all()) and not bool(grad[k][~live].any())
        assert float(grad[3, 7]) == -INF
        assert bool((torch.cat((grad[3, :7], grad[3, 8:])) == INF).all())
    keep = c.logits.clone()
    s2, l2, g2 = zq.policy_loss(keep, c.ids, c.old, c.adv, c.w, c.ref, clip=c.clip, kl=kl, grad=keep)
    assert torch.equal(g2, grad) and torch.equal(s2, sums) and torch.equal(l2, logp)


def test_a_gradient_beyond_its_type():
    """A factor beyond binary32: infinite where the product is, and not where a small
    probability brings it back."""
    logits = torch.tensor([[0.0, -60.0, 1.0, -INF]], device=DEV)
    ids, row = torch.tensor([0], device=DEV), torch.zeros(1, device=DEV)
    old = row - 1.3
    sums, logp, grad = zq.policy_loss(logits, ids, old, row + 3e38, grad_scale=1000.0, clip=(1.0, 9.0))
    p = torch.softmax(logits.double(), 1)[0]
    want = float((logp.double() - old.double()).exp()) * float(row + 3e38) * 1000.0 * float(p[1])
    assert float(grad[0, 0]) == -INF and float(grad[0, 2]) == INF and float(grad[0, 3]) == 0.0
    # the exponential (4 roundings of its exponent of 60, an ulp), logp's rounding
    assert abs(float(grad[0, 1]) - want) <= (4 * 61 + 8) * 2.0**-24 * want


@pytest.mark.parametrize("V,dt", itertools.product([2, 3, 64, 1000, 2049, 5001, 8200, 16411, 24577, 33000, 50000, 65537, 98000,
                                                    131072, 140001], DT))
def test_near_certain_tokens(V, dt):
    """A token whose probability is 1 but for what the others' exponentials add up to, each
    below half a step of 1 in binary32: none of them is lost beside it."""
    at = torch.tensor(sorted({0, 1, V // 3, V // 2, V - 2, V - 1}), device=DEV)
    z = (torch.randn(len(at), V, generator=torch.Generator().manual_seed(V)) * 0.5 - 20.0).to(DEV)
    z[torch.arange(len(at)), at] = 0.0
    z = z.to(DT[dt])
    d = z.double()
    e = torch.exp(d)
    e[torch.arange(len(at)), at] = 0.0
    rest = e.sum(1)
    want = -torch.log1p(rest)
    # an exponential: its exponent's 4 roundings, the instruction's 2^-22 to be safe, 3 additions
    # of 8 neighbours; sums in binary64 of up to 256 and a 1,024th of the row's terms, one after
    # the other; the result's rounding
    U = 2.0**-24
    off = (e * (4 * U * d.abs() + 2.0**-22 + 3 * U)).sum(1) + (256 + V / 1024) * 2.0**-53 + U * want.abs()
    logp = zq.token_logp(z, at)
    assert bool(((logp.double() - want).abs() <= 1.01 * off).all()), f"{logp.tolist()} {want.tolist()}"
    row = torch.zeros(len(at), device=DEV)
    assert torch.equal(zq.policy_loss(z, at, row, row)[1], logp)


@pytest.mark.parametrize("V", [1023, 1025, 1400, 1537, 2048, 2500, 3073, 4095, 4097])
@pytest.mark.parametrize("dt", DT)
def test_rows_of_one_wave(V, dt):
    """Rows that one wave holds in up to 8 vectors a thread, and the next longer ones."""
    c = Case(7, V, dt, seed=9, offset=1)
    sums, logp, grad = c.call()
    c.check(sums, logp, grad)
    assert torch.equal(zq.token_logp(c.logits, c.ids, c.scale), logp)
