"""Every kernel of the INT4 product and every way it is cut, against 64-bit products on
the GPU.  Exact: x multiples of 1/4 up to 2, about 1,000 a row of them not zero, and
scales powers of two between 2^-4 and 1, so that every partial sum in sixteenths is a
multiple of 2^-10 below 2^14.  Bounded: within (K + 64) * 2^-23 * sum_k |x w|."""
import pytest
import torch

import paper_2501_04266_amd as zq
from tests.gpu_util import DEV, poisoned
from tests.int4_routes import ROUTES
from tests.test_int4_plan import LAYERS

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16}


def weight(N, K, block, g, powers):
    packed = torch.randint(0, 256, (N * K // 2,), dtype=torch.uint8, device=DEV, generator=g)
    n = -(-N * K // block)
    scales = (2.0 ** -torch.randint(0, 5, (n,), device=DEV, generator=g).float() if powers
              else torch.rand(n, device=DEV, generator=g) * 1e-2)
    return packed, scales


def products(x, packed, scales, N, block):
    """(product, sum of magnitudes) in 64 bits, some weight rows at a time"""
    K = x.shape[1]
    got, mags, step = [], [], max(1, (1 << 23) // K)
    for n in range(0, N, step):
        b = packed.view(N, K // 2)[n:n + step]
        q = (torch.stack((b & 15, b >> 4), -1).view(len(b), K).to(torch.int8) ^ 8) - 8
        w = q.double() * scales[torch.arange(n * K, n * K + q.numel(), device=DEV) // block].double().view_as(q)
        got.append(x.double() @ w.t())
        mags.append(x.double().abs() @ w.abs().t())
    return torch.cat(got, 1), torch.cat(mags, 1)


def run(x, packed, scales, N, block):
    M = x.shape[0]
    buf = poisoned(M * N + 2, torch.float32)
    guard = buf.clone()
    y = buf[1:1 + M * N].view(M, N)
    zq.int4_dequant_gemm(x, packed, scales, N, block, y=y)
    assert torch.equal(buf[[0, -1]].view(torch.int32), guard[[0, -1]].view(torch.int32))
    return y.double()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("name,M,N,K,block", ROUTES)
def test_routes(name, M, N, K, block, dtype):
    g = torch.Generator(device=DEV).manual_seed(M + N + K)
    packed, scales = weight(N, K, block, g, True)
    x = torch.randint(-8, 9, (M, K), device=DEV, generator=g) / 4.0
    x = (x * (torch.rand(M, K, device=DEV, generator=g) < min(1.0, 1000.0 / K))).to(DT[dtype])
    want, _ = products(x, packed, scales, N, block)
    bad = (run(x, packed, scales, N, block) != want).nonzero()
    assert len(bad) == 0, f"{len(bad)} of {want.numel()} differ, first at {bad[0].tolist()}"

    packed, scales = weight(N, K, block, g, False)
    x = torch.randn(M, K, device=DEV, generator=g).to(DT[dtype])
    want, mags = products(x, packed, scales, N, block)
    got, again = run(x, packed, scales, N, block), run(x, packed, scales, N, block)
    assert torch.equal(got, again)
    assert bool(((got - want).abs() <= (K + 64) * 2.0**-23 * mags).all())


@pytest.mark.parametrize("M,N,K,block", [s for s in LAYERS if s[0] in (17, 64) and s[1] * s[2] < 3 << 26])
def test_layers(M, N, K, block):
    """Layers whole, many weight rows and K in slices."""
    g = torch.Generator(device=DEV).manual_seed(N + K)
    packed, scales = weight(N, K, block, g, False)
    x = torch.randn(M, K, device=DEV, generator=g).bfloat16()
    want, mags = products(x, packed, scales, N, block)
    assert bool(((run(x, packed, scales, N, block) - want).abs() <= (K + 64) * 2.0**-23 * mags).all())
