"""Products with INT4 weights against 64-bit ones.

Exact: x multiples of 1/4 up to 2 and scales powers of two between 2^-4 and 1, so that
every partial sum is a multiple of 2^-10 (sixteenths of codes included) below 2^14 and
any order of additions gives the same bits.  Bounded: random values, within (K + 64) *
2^-23 * sum_k |x w| (K + 64 roundings, of a whole unit each).
"""
import numpy as np
import pytest
import torch

import paper_2501_04266_amd as zq
from tests.gpu_util import DEV, poisoned

pytestmark = pytest.mark.gpu
DT = {"f16": torch.float16, "bf16": torch.bfloat16}


def weight(N, K, block, seed, powers):
    g = np.random.default_rng(seed)
    codes = g.integers(-8, 8, N * K)
    scales = (2.0 ** -g.integers(0, 5, -(-N * K // block)) if powers
              else g.uniform(1e-3, 1e-2, -(-N * K // block))).astype(np.float32)
    nib = (codes & 15).astype(np.uint8)
    packed = nib[0::2] | (nib[1::2] << 4)
    w = torch.from_numpy((codes * scales.astype(np.float64).repeat(block)[:N * K]).reshape(N, K))
    return torch.from_numpy(packed).to(DEV), torch.from_numpy(scales).to(DEV), w


def run(x, packed, scales, N, block):
    M = x.shape[0]
    buf = poisoned(M * N + 2, torch.float32)
    guard = buf.clone()
    y = buf[1:1 + M * N].view(M, N)
    zq.int4_dequant_gemm(x.to(DEV), packed, scales, N, block, y=y)
    torch.cuda.synchronize()
    assert torch.equal(buf[[0, -1]].view(torch.int32), guard[[0, -1]].view(torch.int32))
    return y.double().cpu()


# (M, N, K, block): rows of x at the edges of 16-row tiles; weight rows that no tile
# divides; K of one half step, odd numbers of 64s, several rounds of the waves and more
# than one staged range; blocks that straddle rows
CASES = [(1, 1, 64, 32), (1, 15, 64, 1024), (2, 17, 128, 64), (3, 33, 192, 128), (1, 100, 320, 256), (5, 130, 448, 32),
         (1, 2049, 2048, 128), (1, 300, 6144, 128), (1, 48, 24576, 256), (4, 1000, 1088, 1024), (8, 257, 2112, 64),
         (15, 65, 4160, 128), (16, 100, 6208, 256), (16, 64, 2048, 32), (16, 31, 12352, 512), (17, 100, 704, 128),
         (31, 77, 2240, 64), (32, 128, 4096, 128), (33, 50, 960, 32), (48, 96, 6144, 256), (63, 40, 1600, 128),
         (64, 200, 2048, 64), (65, 33, 1024, 128), (130, 90, 576, 256), (2, 6145, 512, 128), (9, 50001, 128, 128)]
# weight rows that share x in groups of one, two and three tiles, and more groups than run at
# once; a K summed in slices, the last one shorter
CASES += [(1, 16400, 192, 64), (5, 8320, 448, 128), (16, 8208, 5440, 64), (12, 8210, 576, 32), (4, 40, 24576, 128),
          (2, 24, 49152, 32), (9, 4500, 64, 32), (20, 4300, 320, 128), (40, 4300, 192, 64), (24, 8300, 320, 128),
          (50, 8300, 256, 256), (64, 12400, 128, 32), (10, 40, 24576, 128), (33, 70, 16448, 64), (20, 100, 14400, 32)]
# more than 16 rows and many weight rows: a tile a wave, x through LDS
CASES += [(24, 16400, 320, 128), (32, 16390, 1088, 64), (17, 16500, 64, 32), (40, 16400, 576, 64), (48, 16385, 512, 256),
          (35, 16400, 192, 32), (64, 16390, 832, 32), (49, 16400, 1280, 128), (60, 16400, 320, 64), (70, 16400, 192, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M,N,K,block", CASES)
def test_exact(M, N, K, block, dtype):
    g = np.random.default_rng(M + N + K)
    packed, scales, w = weight(N, K, block, N + K, True)
    # few and small enough for exact sums of K up to 24,576: at most 2 * 8 * K / 24 of them count
    x = torch.from_numpy(g.integers(-8, 9, (M, K)) / 4.0 * (g.random((M, K)) < min(1.0, 1000.0 / K)))
    got = run(x.to(DT[dtype]), packed, scales, N, block)
    want = x.double() @ w.t()
    bad = (got != want).nonzero()
    assert len(bad) == 0, f"{len(bad)} of {got.numel()} differ, first at {bad[0].tolist()}"


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M,N,K,block", CASES)
def test_bounded(M, N, K, block, dtype):
    packed, scales, w = weight(N, K, block, N + K + 1, False)
    x = torch.randn(M, K, generator=torch.Generator().manual_seed(K)).to(DT[dtype])
    got, again = run(x, packed, scales, N, block), run(x, packed, scales, N, block)
    assert torch.equal(got, again)
    want, mags = x.double() @ w.t(), x.double().abs() @ w.abs().t()
    far = (got - want).abs() / ((K + 64) * 2.0**-23 * mags)
    assert float(far.max()) <= 1.0


def test_the_quantisers_weight():
    """A weight as qgz_quantize stores it: the product with the dequantised weight."""
    N, K, block = 513, 1344, 128
    w = torch.randn(N * K, generator=torch.Generator().manual_seed(1)) * 0.02
    packed, scales = zq.qgz_quantize(w.to(DEV), block)
    x = torch.randn(3, K, generator=torch.Generator().manual_seed(2)).bfloat16()
    deq = zq.qgz_dequantize(packed, scales, N * K, block).cpu().double().view(N, K)
    got = zq.int4_dequant_gemm(x.to(DEV), packed, scales, N, block).cpu().double()
    mags = x.double().abs() @ deq.abs().t()
    # the dequantised weight is rounded once, by 2^-24 at most
    assert bool(((got - x.double() @ deq.t()).abs() <= ((K + 64) * 2.0**-23 + 2.0**-24) * mags).all())


def test_special_values():
    """NaN and infinities of x stay in their own rows; codes of zero, scales of zero,
    infinite and NaN scales in their own columns; large and small scales."""
    M, N, K, block = 6, 40, 512, 64
    packed, scales, _ = weight(N, K, block, 4, True)
    x = torch.ones(M, K, dtype=torch.bfloat16)
    x[1, 200], x[3, 511] = float("nan"), float("inf")
    packed.view(N, K // 2)[7] = 0
    s = scales.view(N, K // block)
    s[9], s[11, 3], s[13, 0], s[15], s[17] = 0.0, float("inf"), float("nan"), 2.0**100, 2.0**-126
    packed.view(N, K // 2)[11] = 0x11
    packed.view(N, K // 2)[15] = 0x11
    packed.view(N, K // 2)[17] = 0x77
    got = zq.int4_dequant_gemm(x.to(DEV), packed, scales, N, block).cpu()
    rows = [0, 2, 4, 5]
    assert bool(got[1].isnan().all())
    # the infinite element meets code 0 in row 7 of the weight, and scale 0 in row 9
    assert math_nan(got[3, 7]) and math_nan(got[3, 9])
    fine = [n for n in range(N) if n not in (11, 13)]
    assert bool(got[rows][:, fine].isfinite().all())
    assert got[rows][:, 7].eq(0).all() and got[rows][:, 9].eq(0).all()
    assert got[rows][:, 11].eq(float("inf")).all() and got[rows][:, 13].isnan().all()
    assert got[rows][:, 15].eq(512 * 2.0**100).all() and got[rows][:, 17].eq(7 * 512 * 2.0**-126).all()


@pytest.mark.parametrize("M,N,K", [(3, 40, 24576), (12, 8320, 512), (12, 8320, 8192), (12, 40, 24576), (40, 4300, 512),
                                   (20, 16400, 640)])
def test_special_rows(M, N, K):
    """NaN and infinities of x stay in their rows, those of scales in their columns,
    whichever way the product is cut."""
    packed, scales, _ = weight(N, K, 128, 4, True)
    packed.view(N, K // 2)[17] = 0x11
    s = scales.view(N, K // 128)
    s[17] = 1.0
    s[19, 1], s[N - 1] = float("nan"), 0.0
    x = torch.ones(M, K, dtype=torch.bfloat16)
    x[1, K - 1], x[2, 200] = float("nan"), float("inf")
    got = zq.int4_dequant_gemm(x.to(DEV), packed, scales, N, 128).cpu()
    rows = [m for m in range(M) if m not in (1, 2)]
    assert bool(got[1].isnan().all()) and math_nan(got[2, N - 1])
    assert bool(got[:, 19].isnan().all())
    assert bool(got[rows][:, [n for n in range(N) if n != 19]].isfinite().all())
    assert bool(got[rows][:, 17].eq(K).all()) and bool(got[rows][:, N - 1].eq(0).all()) and got[2, 17] == float("inf")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M,N,K,block", [
    (16, 5003, 20544, 64), (31, 5003, 20544, 64), (13, 5003, 20480, 128), (16, 5003, 20480, 32),  # slices of K
    (9, 4500, 384, 128), (9, 4500, 320, 64), (20, 4300, 384, 128), (20, 4300, 384, 32), (20, 300, 320, 32), (24, 8300, 384, 256),
    (24, 8300, 320, 32), (40, 4300, 512, 32), (40, 4300, 512, 64), (40, 4300, 512, 128), (50, 8300, 512, 32),
    (50, 8300, 576, 64), (30, 16400, 768, 128), (64, 20011, 2176, 128), (12, 20011, 10560, 256), (3, 6001, 24576, 64)])
def test_against_the_gpu(M, N, K, block, dtype):
    """Weights of many rows, against 64-bit products on the GPU."""
    g = torch.Generator(device=DEV).manual_seed(M)
    packed = torch.randint(0, 256, (N * K // 2,), dtype=torch.uint8, device=DEV, generator=g)
    scales = torch.rand(-(-N * K // block), device=DEV, generator=g) * 1e-2
    x = torch.randn(M, K, device=DEV, generator=g).to(DT[dtype])
    got = zq.int4_dequant_gemm(x, packed, scales, N, block).double()
    step = max(1, (1 << 23) // K)
    for n in range(0, N, step):
        b = packed.view(N, K // 2)[n:n + step]
        q = (torch.stack((b & 15, b >> 4), -1).view(len(b), K).to(torch.int8) ^ 8) - 8
        at = torch.arange(n * K, n * K + q.numel(), device=DEV) // block
        w = q.double() * scales[at].double().view_as(q)
        far = (got[:, n:n + step] - x.double() @ w.t()).abs()
        assert bool((far <= (K + 64) * 2.0**-23 * (x.double().abs() @ w.abs().t())).all())


def test_workspace():
    """Given, it is used; too small, it is refused; what it held does not count."""
    M, N, K, block = 7, 33, 24576, 128
    need = zq.int4_dequant_gemm_bytes(M, N, K)
    assert need > 0 and zq.int4_dequant_gemm_bytes(M, N, 64) == 0
    packed, scales, _ = weight(N, K, block, 3, False)
    x = torch.randn(M, K, generator=torch.Generator().manual_seed(1)).half().to(DEV)
    want = zq.int4_dequant_gemm(x, packed, scales, N, block)
    ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device=DEV)
    assert torch.equal(zq.int4_dequant_gemm(x, packed, scales, N, block, workspace=ws), want)
    assert bool((ws[need:] == 0xFF).all())
    with pytest.raises(ValueError):
        zq.int4_dequant_gemm(x, packed, scales, N, block, workspace=ws[:need - 1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = zq.int4_dequant_gemm(x, packed, scales, N, block, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


def math_nan(v):
    return bool(v.isnan())


def test_x_of_any_size():
    """Subnormal and large fp16 values of x count as they are."""
    K = 64
    packed, scales, w = weight(16, K, 32, 6, True)
    for v in (2.0**-24, 2.0**-15, 65504.0):
        x = torch.zeros(1, K, dtype=torch.float16)
        x[0, 5], x[0, 40] = v, -v
        got = zq.int4_dequant_gemm(x.to(DEV), packed, scales, 16, 32).cpu().double()
        assert torch.equal(got, x.double() @ w.t()), v


def test_beyond_32_bits():
    """Codes past 2^32 elements."""
    K, block = 1 << 17, 1024
    N = (1 << 32) // K + 20
    packed = torch.zeros(N * K // 2, dtype=torch.uint8, device=DEV)
    packed.view(N, K // 2)[N - 1] = 0x11
    packed.view(N, K // 2)[N - 3, -1] = 0x70
    scales = torch.full((N * K // block,), 0.25, device=DEV)
    y = zq.int4_dequant_gemm(torch.ones(2, K, dtype=torch.bfloat16, device=DEV), packed, scales, N, block).cpu()
    want = torch.zeros(2, N)
    want[:, N - 1], want[:, N - 3] = 0.25 * K, 0.25 * 7
    assert torch.equal(y, want)


def test_empty():
    z = torch.zeros(64, dtype=torch.uint8, device=DEV)
    s = torch.zeros(4, device=DEV)
    x = torch.zeros((0, 64), dtype=torch.bfloat16, device=DEV)
    assert zq.int4_dequant_gemm(x, z, s, 2, 32).shape == (0, 2)
    assert zq.int4_dequant_gemm(torch.zeros((3, 64), dtype=torch.bfloat16, device=DEV), z, s, 0, 32).shape == (3, 0)
    y = zq.int4_dequant_gemm(torch.zeros((3, 0), dtype=torch.bfloat16, device=DEV), z, s, 5, 32)
    assert torch.equal(y.cpu(), torch.zeros(3, 5))


def test_streams_and_graphs():
    M, N, K, block = 4, 300, 2176, 128
    packed, scales, w = weight(N, K, block, 2, True)
    x = (torch.randint(-8, 9, (M, K), generator=torch.Generator().manual_seed(1)) / 4).half().to(DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = zq.int4_dequant_gemm(x, packed, scales, N, block, stream=side)
    side.synchronize()
    assert torch.equal(y.double().cpu(), x.double().cpu() @ w.t())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        zq.int4_dequant_gemm(x, packed, scales, N, block, y=y)
    for _ in range(3):
        x.neg_()
        y.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, zq.int4_dequant_gemm(x, packed, scales, N, block))
