"""The INT4 product at the ends of the range that its error bound, (K + 64) * 2^-23 *
sum_k |x w|, is stated for: x of magnitudes from 2^-110 to below 2^122, sums of
magnitudes from 2^-122 on."""
import numpy as np
import pytest
import torch

import paper_2501_04266_amd as zq
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu

# a kernel of each kind: up to 4 rows, x in LDS, x in registers, a tile a wave
SIZES = [(1, 40, 512), (4, 40, 512), (5, 8240, 256), (8, 40, 512), (20, 40, 256), (33, 4112, 256)]


def check(x, codes, scales, block):
    M, K = x.shape
    N = codes.shape[0]
    nib = (codes & 15).astype(np.uint8).reshape(-1)
    packed = torch.from_numpy(nib[0::2] | (nib[1::2] << 4)).to(DEV)
    got = zq.int4_dequant_gemm(x.to(DEV), packed, torch.from_numpy(scales).to(DEV), N, block).double().cpu()
    w = torch.from_numpy((codes.reshape(-1) * scales.astype(np.float64).repeat(block)[:N * K]).reshape(N, K))
    want, mags = x.double() @ w.t(), x.double().abs() @ w.abs().t()
    assert bool((mags.min() >= 2.0**-122) & (mags.max() < 2.0**127)), "the case's own range"
    assert bool(((got - want).abs() <= (K + 64) * 2.0**-23 * mags).all())


@pytest.mark.parametrize("block", [64, 128, 256])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_largest_x(M, N, K, block):
    """All products of one sign, as large as they can be: whole blocks of code -8."""
    x = torch.full((M, K), 2.0**122 * (1 - 2.0**-8)).bfloat16()
    assert float(x[0, 0]) < 2.0**122
    check(x, np.full((N, K), -8), np.full(-(-N * K // block), 2.0**-12, np.float32), block)


@pytest.mark.parametrize("xe,se", [(-110, 0), (-110, -9), (-60, -58), (0, -118), (100, -149), (121, -149), (121, -20)])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_magnitudes(M, N, K, xe, se):
    """Mixed signs and significands around one magnitude of x and one of the scales."""
    g = np.random.default_rng(abs(xe) + M)
    x = torch.from_numpy(g.choice([-1.0, 1.0], (M, K)) * g.integers(128, 256, (M, K)) * 2.0**(xe - 7)).bfloat16()
    assert float(x.abs().min()) >= 2.0**-110 and float(x.abs().max()) < 2.0**122
    codes = g.integers(-8, 8, (N, K))
    codes[:, 0] = 7
    scales = np.full(N * K // 128, 2.0**se, np.float32)
    check(x, codes, scales, 128)
