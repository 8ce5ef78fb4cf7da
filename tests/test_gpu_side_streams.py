"""Calls on another stream than the current one, while the current one still has work
on memory that was freed: that work must not reach the call's workspace or output."""
import pytest
import torch

import paper_2501_04266_amd as zq
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu


def pending(sizes):
    """Work on the current stream that takes some milliseconds and then writes freed
    memory of these sizes."""
    a = torch.ones(4096, 4096, device=DEV)
    for _ in range(20):
        a = a @ a * 0.0
    for n in sizes:
        torch.empty(n, dtype=torch.uint8, device=DEV).fill_(0x7F)


def gradient():
    V, D, T = 500, 136, 900
    g = torch.Generator().manual_seed(1)
    ids = torch.randint(0, V, (T,), generator=g).to(DEV)
    dy = torch.randn(T, D, generator=g).to(DEV)
    return (lambda **k: zq.embedding_grad(ids, dy, V, **k)), [V * D * 4, zq.embedding_grad_bytes(T, V, D)]


def product():
    M, N, K, block = 7, 33, 24576, 128
    packed, scales = zq.qgz_quantize(torch.randn(N * K, generator=torch.Generator().manual_seed(2)).to(DEV), block)
    x = torch.randn(M, K, generator=torch.Generator().manual_seed(3)).half().to(DEV)
    return ((lambda **k: zq.int4_dequant_gemm(x, packed, scales, N, block, **k)),
            [M * N * 4, zq.int4_dequant_gemm_bytes(M, N, K)])


def lookup():
    table = torch.randn(300, 64, generator=torch.Generator().manual_seed(4)).to(DEV)
    ids = torch.arange(2000, device=DEV) % 311
    return (lambda **k: zq.embedding(ids, table, **k)), [2000 * 64 * 4]


def int8_lookup():
    codes, scales = zq.qwz_quantize(torch.randn(300 * 64, generator=torch.Generator().manual_seed(4)).to(DEV), 256)
    ids = torch.arange(2000, device=DEV) % 311
    return (lambda **k: zq.qwz_embedding(ids, codes, scales, 300, 64, 256, **k)), [2000 * 64 * 2]


def norm():
    table = zq.grad_table([torch.randn(100_000, generator=torch.Generator().manual_seed(5)).to(DEV)])
    return (lambda **k: zq.grad_norm(table, **k)), [4]


@pytest.mark.parametrize("make", [gradient, product, lookup, int8_lookup, norm])
@pytest.mark.parametrize("kind", ["stream", "handle"])
@pytest.mark.parametrize("given", [False, True])
def test_pending_work_on_freed_memory(make, kind, given):
    call, sizes = make()
    want = call()
    out = torch.empty_like(want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    pending(sizes)
    name = "y" if make is product else "out"
    got = call(stream=side if kind == "stream" else side.cuda_stream, **({name: out} if given else {}))
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def path_calls():
    n, block = 40_000, 64
    x = torch.randn(n, generator=torch.Generator().manual_seed(6)).to(DEV)
    codes, cs = zq.qwz_quantize(x, block)
    packed, ps = zq.qgz_quantize(x, block)
    pair, pair_s = torch.cat([packed, packed]), torch.cat([ps, ps])
    # whole numbers and one scale: the product's sums, which are added atomically over ranges of K, are exact
    xb = torch.randint(-8, 9, (10, 640), generator=torch.Generator().manual_seed(7)).bfloat16().to(DEV)
    one_scale = torch.full_like(cs, 2.0**-7)
    return {
        "qwz_quantize": (lambda **k: zq.qwz_quantize(x, block, **k), [n, 4 * len(ps)]),
        "qwz_dequantize": (lambda **k: zq.qwz_dequantize(codes, cs, block, **k), [2 * n]),
        "qgz_quantize": (lambda **k: zq.qgz_quantize(x, block, **k), [n // 2, 4 * len(ps)]),
        "qgz_dequantize": (lambda **k: zq.qgz_dequantize(packed, ps, n, block, **k), [4 * n]),
        "qgz_reduce_level": (lambda **k: zq.qgz_reduce_level(pair, pair_s, 2, n, block, **k), [n // 2, 4 * len(ps)]),
        "qgz_reduce_dequantize": (lambda **k: zq.qgz_reduce_dequantize(pair, pair_s, 2, n, block, **k), [4 * n]),
        "qgz_reduce_level_gather": (lambda **k: zq.qgz_reduce_level_gather([packed, packed], [ps, ps], n, block, **k),
                                    [n // 2, 4 * len(ps)]),
        "qwz_dequant_gemm": (lambda **k: zq.qwz_dequant_gemm(xb, codes[:62 * 640], one_scale, 62, block, **k), [10 * 62 * 4]),
    }


@pytest.mark.parametrize("name", ["qwz_quantize", "qwz_dequantize", "qgz_quantize", "qgz_dequantize",
                                  "qgz_reduce_level", "qgz_reduce_dequantize", "qgz_reduce_level_gather",
                                  "qwz_dequant_gemm"])
def test_pending_work_on_a_path_calls_output(name):
    call, sizes = path_calls()[name]
    want = call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    pending(sizes)
    got = call(stream=side)
    torch.cuda.synchronize()
    for g, w in zip(*((v if isinstance(v, tuple) else (v,)) for v in (got, want))):
        assert torch.equal(g, w)


def test_one_table_on_two_streams():
    """Calls that share a table's partial sums write the same ones."""
    grads = [torch.randn(n, generator=torch.Generator().manual_seed(n)).to(DEV) for n in (20_000_000, 3, 5_000_001)]
    table = zq.grad_table(grads)
    want = zq.grad_norm(table)
    outs = [torch.zeros(20, device=DEV) for _ in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i in range(20):
        for out, st in zip(outs, streams):
            zq.grad_norm(table, out=out[i], stream=st)
    torch.cuda.synchronize()
    assert all(bool((out == want).all()) for out in outs)
