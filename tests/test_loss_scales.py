"""The loss refuses scales whose exponents binary32 cannot hold (no GPU needed: checks come
before any work), and takes the largest and the smallest that it can."""
import ctypes
import math

import pytest
import torch

import paper_2501_04266_amd as zq
from paper_2501_04266_amd import _lib
from tests.gpu_util import DEV

LARGEST = 2.0**127
BEYOND = float(torch.nextafter(torch.tensor(LARGEST), torch.tensor(math.inf)))
SIZE, NULL = -5, -1


@pytest.mark.parametrize("scale,status", [(LARGEST, NULL), (BEYOND, SIZE), (2.4e38, SIZE), (3.4e38, SIZE), (math.inf, SIZE),
                                          (1e-45, NULL), (0.0, SIZE), (-0.0, SIZE), (math.nan, SIZE)])
def test_scales(scale, status):
    """Scales that are taken go on to the next check: here addresses that are missing."""
    L = _lib.lib()
    assert L.zq_token_logp(None, _lib.ZQ_F32, 4, 9, 9, None, _lib.ZQ_I64, scale, None, None) == status
    policy = _lib._Policy(None, None, None, None, 0.2, 0.2, 0.0, scale, 1.0, 0)
    assert L.zq_policy_loss(None, _lib.ZQ_F32, 4, 9, 9, None, _lib.ZQ_I64, ctypes.byref(policy), None, None, None, 0, 9, None,
                            128, None) == status


@pytest.mark.gpu
@pytest.mark.parametrize("V", [7, 3000, 70001])
def test_the_largest_and_smallest_scale(V):
    """The largest: all of the probability on the row's largest logits.  The smallest: none to tell apart."""
    z = torch.randn(3, V, generator=torch.Generator().manual_seed(V)).to(DEV)
    z[0, 2], z[1, 4], z[2, 1], z[2, 5] = 9.0, 9.0, 9.0, 9.0
    ids = torch.tensor([2, 3, 5], device=DEV)
    logp = zq.token_logp(z, ids, scale=LARGEST)
    assert float(logp[0]) == 0.0 and float(logp[1]) == -math.inf
    assert abs(float(logp[2]) + math.log(2)) <= 2.0**-24
    row = torch.zeros(3, device=DEV)
    sums, again, grad = zq.policy_loss(z, ids, row, row + 1, scale=LARGEST, grad_scale=2.0**-127)
    assert torch.equal(again, logp) and bool(sums.isfinite().all())
    want = torch.zeros(3, V, device=DEV)  # -r A ((v == a) - p) with r = 1, 0 and a half
    want[2, 5], want[2, 1] = -0.25, 0.25
    assert bool(((grad - want).abs() <= 2.0**-22).all())
    assert bool(((zq.token_logp(z, ids, scale=1e-45) + math.log(V)).abs() <= 2.0**-24 * math.log(V) + 2.0**-22).all())
