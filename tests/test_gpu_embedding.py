"""The embedding calls against their formulas in 64 bits.

Tolerances, from the definitions (u = half a unit in the last place of the output
type, relative; 2^-24 for each binary32 rounding before it):
  lookup    one product (dense) or two (INT8), then the output's rounding
  gradient  n tokens of a row are n - 1 additions in any order, so the sum is off by
            at most n * 2^-24 * sum |dy|; then the product with scale and the output's
            rounding; accumulating adds one more addition
Subnormal results are off by at most the smallest subnormal instead.
"""
import numpy as np
import pytest
import torch

import paper_2501_04266_amd as zq
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {"f32": 2.0**-24, "f16": 2.0**-11, "bf16": 2.0**-8}
TINY = {"f32": 2.0**-149, "f16": 2.0**-24, "bf16": 2.0**-133}


def rand(shape, seed, dtype, std=0.02):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(DT[dtype])


def some_ids(T, V, seed, wide=True, outside=True):
    """Ids of which many are the same, some not rows of the table."""
    g = np.random.default_rng(seed)
    ids = np.minimum((V * g.random(T) ** 3).astype(np.int64), V - 1) if V else np.zeros(T, np.int64)
    if outside and T > 3:
        bad = [-1, V, V + 7, -(1 << 31)] + ([1 << 40, -(1 << 63), (1 << 32)] if wide else [])
        ids[g.random(T) < 0.15] = g.choice(bad)
        ids[T // 2] = -1
    return torch.from_numpy(ids if wide else ids.astype(np.int32))


def between(n, dtype, offset):
    """n elements `offset` past a 16-byte boundary, with guards on both sides."""
    buf = torch.empty(offset + n + 16, dtype=DT[dtype], device=DEV)
    buf.view(torch.uint8).fill_(0xA5)
    return buf, buf[offset:offset + n]


def guards_whole(buf, offset, n):
    rest = torch.cat([buf[:offset], buf[offset + n:]]).view(torch.uint8)
    return bool((rest == 0xA5).all())


def close(got, want, dtype, extra):
    """|got - want| within the output's rounding and `extra` (absolute, before it)."""
    got, want = got.double().cpu(), want.cpu()
    bound = extra + U[dtype] * (want.abs() + extra) + TINY[dtype]
    bad = ((got - want).abs() > bound) | got.isnan()
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} differ, first at {bad.nonzero()[0].tolist()}"


LOOKUPS = [(0, 5, 8), (1, 1, 1), (1, 50, 7), (3, 9, 8), (5, 33, 9), (64, 100, 64), (1, 1000, 6144), (257, 77, 127),
           (100, 3, 2051), (33, 500, 1032), (1000, 64, 3), (2, 4, 70001)]


@pytest.mark.parametrize("wide", [True, False])
@pytest.mark.parametrize("wt,yt", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f32", "f16"), ("f16", "bf16")])
@pytest.mark.parametrize("T,V,D", LOOKUPS)
def test_lookup(T, V, D, wt, yt, wide):
    table, ids = rand((V, D), T + V + D, wt), some_ids(T, V, D, wide)
    scale = 1.0 if T % 2 else 7.3
    off = D % 5  # tables and outputs need not start at a 16-byte boundary
    tbuf, t = between(V * D, wt, off)
    t.copy_(table.view(-1).to(DEV))
    buf, y = between(T * D, yt, off)
    got = zq.embedding(ids.to(DEV), t.view(V, D), scale=scale, out=y.view(T, D))
    torch.cuda.synchronize()
    real = (ids >= 0) & (ids < V)
    want = torch.zeros(T, D, dtype=torch.float64)
    want[real] = table[ids[real].long()].double() * float(np.float32(scale))
    close(got, want, yt, 2.0**-24 * want.abs())
    assert guards_whole(buf, off, T * D)


@pytest.mark.parametrize("block", [32, 256, 1024])
@pytest.mark.parametrize("yt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,V,D", LOOKUPS[1:])
def test_int8_lookup(T, V, D, yt, block):
    ids = some_ids(T, V, D + 1)
    codes, scales = zq.qwz_quantize(rand(V * D, D, "f32").to(DEV), block)
    whole = zq.qwz_dequantize(codes, scales, block, out_dtype=DT[yt]).view(V, D).cpu()
    real = (ids >= 0) & (ids < V)
    # scale 1: the rows that the dequantiser writes, bit for bit
    buf, y = between(T * D, yt, 3)
    got = zq.qwz_embedding(ids.to(DEV), codes, scales, V, D, block, out=y.view(T, D)).cpu()
    want = torch.zeros(T, D, dtype=DT[yt])
    want[real] = whole[ids[real]]
    assert torch.equal(got.view(torch.uint8), want.view(torch.uint8)) and guards_whole(buf, 3, T * D)
    # another scale, in 64 bits
    got = zq.qwz_embedding(ids.to(DEV), codes, scales, V, D, block, scale=-0.7, out_dtype=DT[yt])
    w = codes.double().cpu() * scales.double().cpu().repeat_interleave(block)[:V * D]
    want = torch.zeros(T, D, dtype=torch.float64)
    want[real] = w.view(V, D)[ids[real]] * float(np.float32(-0.7))
    close(got, want, yt, 2 * 2.0**-24 * want.abs())


def test_lookup_special_values():
    """NaN and infinities come through in their own places alone; ids of any shape."""
    table = rand((6, 40), 1, "f32")
    table[2, 5], table[2, 6], table[3, 39], table[4, 0] = float("nan"), float("inf"), -float("inf"), -0.0
    ids = torch.tensor([[2, -1, 3], [0, 2, 4]])
    got = zq.embedding(ids.to(DEV), table.to(DEV), scale=0.5).cpu()
    want = torch.where((ids < 0)[..., None], torch.zeros(()), table[ids.clamp(min=0)] * 0.5)
    assert got.shape == (2, 3, 40)
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(), want.nan_to_num())


def test_empty_table():
    """A table without rows: every id is outside it."""
    y = zq.embedding(torch.tensor([0, 3], device=DEV), torch.empty((0, 16), device=DEV))
    assert torch.equal(y.cpu(), torch.zeros(2, 16))


def grad64(ids, dy, V, scale):
    """(gradient, sum of magnitudes, tokens of each row), 64 bits"""
    D = dy.shape[-1]
    want, mags = torch.zeros(V, D, dtype=torch.float64), torch.zeros(V, D, dtype=torch.float64)
    count = torch.zeros(V, 1, dtype=torch.float64)
    ids, dy = ids.reshape(-1), dy.reshape(-1, D).double()
    real = (ids >= 0) & (ids < V)
    at = ids[real].long()
    want.index_add_(0, at, dy[real])
    mags.index_add_(0, at, dy[real].abs())
    count.index_add_(0, at, torch.ones(len(at), 1, dtype=torch.float64))
    s = float(np.float32(scale))
    return want * s, mags * abs(s), count


GRADS = [(0, 5, 8), (1, 1, 1), (1, 40, 7), (2, 3, 8), (63, 4, 9), (64, 1, 16), (65, 1, 16), (129, 2, 24), (300, 257, 40),
         (1000, 7, 130), (1025, 600, 33), (5000, 3, 3), (4097, 1000, 72), (700, 140001, 8), (20000, 300, 64),
         (200, 50, 2051), (513, 1, 16), (600, 4, 9), (700, 5, 24), (900, 50, 2051), (512, 70, 1030), (511, 1000, 2600),
         (17, 300, 8200), (512, 1, 64)]


@pytest.mark.parametrize("gt,yt", [("f32", "f32"), ("bf16", "f32"), ("f16", "f32"), ("bf16", "bf16"), ("f32", "f16")])
@pytest.mark.parametrize("T,V,D", GRADS)
def test_gradient(T, V, D, gt, yt):
    wide = D % 2 == 0
    ids, dy = some_ids(T, V, T + D, wide), rand((T, D), T + 7, gt, 1e-3)
    scale, off = (1.0, 0) if T % 2 else (-2.7, 5)
    gbuf, g = between(T * D, gt, off)
    g.copy_(dy.view(-1).to(DEV))
    buf, w = between(V * D, yt, off)
    args = (ids.to(DEV), g.view(T, D), V)
    zq.embedding_grad(*args, scale=scale, out=w.view(V, D))
    torch.cuda.synchronize()
    want, mags, count = grad64(ids, dy, V, scale)
    extra = (count + 1) * 2.0**-24 * mags + TINY["f32"]
    close(w.view(V, D), want, yt, extra)
    assert (w.view(V, D).cpu()[(count == 0).view(-1)] == 0).all()
    assert guards_whole(buf, off, V * D)
    first = w.clone()
    # the same bits again, and added to what is there
    again = zq.embedding_grad(*args, scale=scale, out_dtype=DT[yt])
    assert torch.equal(again.view(-1).view(torch.uint8), first.view(torch.uint8))
    old = rand(V * D, 3, yt, 1e-2).to(DEV)
    w.copy_(old)
    zq.embedding_grad(*args, scale=scale, out=w.view(V, D), accumulate=True)
    both = want + old.cpu().double().view(V, D)
    close(w.view(V, D), both, yt, extra + 2.0**-24 * (both.abs() + extra))
    none = (count == 0).view(-1)
    assert torch.equal(w.view(V, D).cpu()[none], old.view(V, D).cpu()[none]) and guards_whole(buf, off, V * D)


@pytest.mark.parametrize("T", [1, 63, 64, 65, 127, 128, 129, 511, 512, 513, 575, 576, 577, 640, 4096, 10007])
@pytest.mark.parametrize("V,v", [(1, 0), (9, 8), (70000, 65535)])
def test_gradient_of_one_row(T, V, v):
    """All tokens the same: whole 64s, and what is left before and after them; exact,
    as the values are multiples of 2^-10 with sums below 2^14."""
    D = 20
    dy = (torch.randint(-15, 16, (T, D), generator=torch.Generator().manual_seed(T)).float() / 1024)
    got = zq.embedding_grad(torch.full((T,), v, device=DEV), dy.to(DEV), V).cpu()
    want = torch.zeros(V, D)
    want[v] = dy.double().sum(0).float()
    assert torch.equal(got, want)


@pytest.mark.parametrize("seed", range(6))
def test_gradient_runs_of_any_length(seed):
    """Rows whose tokens start and end anywhere against the 64s; exact sums."""
    g = np.random.default_rng(seed)
    counts = g.choice([0, 1, 2, 5, 31, 62, 63, 64, 65, 66, 127, 128, 129, 200, 400], 40)
    ids = np.repeat(np.arange(40), counts)
    g.shuffle(ids)
    T, D = len(ids), int(g.choice([8, 12, 19]))
    dy = g.integers(-15, 16, (T, D)).astype(np.float32) / 64
    want = np.zeros((41, D), np.float64)
    np.add.at(want, ids, dy.astype(np.float64))
    got = zq.embedding_grad(torch.from_numpy(ids).to(DEV), torch.from_numpy(dy).to(DEV), 41).cpu().numpy()
    assert np.array_equal(got.astype(np.float64), want)


def test_gradient_against_differences():
    """The loss sum(dy * embedding(table)) is linear in the table: its differences are
    exact where tables and dy are small multiples of a power of two."""
    V, D, T = 6, 10, 40
    g = np.random.default_rng(5)
    ids = torch.from_numpy(np.where(g.random(T) < 0.1, -1, g.integers(0, V, T))).to(DEV)
    dy = torch.from_numpy(g.integers(-8, 9, (T, D)).astype(np.float32) / 8).to(DEV)
    table = torch.from_numpy(g.integers(-8, 9, (V, D)).astype(np.float32) / 8).to(DEV)
    grad = zq.embedding_grad(ids, dy, V, scale=0.5).cpu()

    def loss(t):
        return float((zq.embedding(ids, t, scale=0.5).double() * dy.double()).sum())

    for v in range(V):
        for d in range(D):
            up, down = table.clone(), table.clone()
            up[v, d] += 0.25
            down[v, d] -= 0.25
            assert (loss(up) - loss(down)) / 0.5 == float(grad[v, d]), (v, d)


def test_gradient_special_values():
    """NaN and infinities in a token's row reach that row's gradient alone; those of
    tokens that are padding reach none."""
    ids = torch.tensor([3, -1, 5, 3, 9, 5])
    dy = rand((6, 16), 2, "f32")
    dy[0, 1], dy[1], dy[2, 4], dy[5, 4], dy[4, 15] = float("nan"), float("nan"), float("inf"), -float("inf"), float("inf")
    got = zq.embedding_grad(ids.to(DEV), dy.to(DEV), 8).cpu()
    want = torch.zeros(8, 16)
    want[3], want[5] = dy[0] + dy[3], dy[2] + dy[5]
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(), want.nan_to_num())


def test_beyond_32_bits():
    """Elements past 2^31 of the table, of its gradient and of INT8 codes."""
    D = 4099
    V = (1 << 31) // D + 50
    ids = torch.tensor([V - 1, 0, V - 2, -1, V - 1], device=DEV)
    table = torch.zeros((V, D), dtype=torch.bfloat16, device=DEV)
    table[V - 1], table[V - 2], table[0] = 3.0, 2.0, 1.0
    y = zq.embedding(ids, table)
    assert torch.equal(y[:, [0, 77, D - 1]].float().cpu(), torch.tensor([3.0, 1, 2, 0, 3])[:, None].expand(5, 3))
    del table
    codes = torch.zeros(V * D, dtype=torch.int8, device=DEV)
    codes.view(V, D)[V - 1] = 100
    scales = torch.full((zq.num_scales(V * D, 1024),), 0.5, device=DEV)
    y = zq.qwz_embedding(ids, codes, scales, V, D, 1024)
    assert bool((y[0] == 50).all()) and bool((y[1:4] == 0).all()) and bool((y[4] == 50).all())
    del codes, scales
    dw = zq.embedding_grad(ids, torch.ones((5, D), dtype=torch.bfloat16, device=DEV), V, out_dtype=torch.bfloat16)
    assert bool((dw[V - 1] == 2).all()) and bool((dw[V - 2] == 1).all()) and bool((dw[0] == 1).all())
    assert bool((dw[1:V - 2] == 0).all())


def test_streams_and_graphs():
    """On a stream of its own with the workspace allocated by the call, and replayed
    from a graph between eager calls."""
    V, D, T = 500, 136, 900
    ids, dy = some_ids(T, V, 1).to(DEV), rand((T, D), 4, "bf16").to(DEV)
    table = rand((V, D), 9, "bf16").to(DEV)
    want_y, want_g = zq.embedding(ids, table, scale=3.0), zq.embedding_grad(ids, dy, V)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = zq.embedding(ids, table, scale=3.0, stream=side)
    g = zq.embedding_grad(ids, dy, V, stream=side.cuda_stream)
    torch.empty(zq.embedding_grad_bytes(T, V, D), dtype=torch.uint8, device=DEV).fill_(0xFF)
    side.synchronize()
    assert torch.equal(y, want_y) and torch.equal(g, want_g)

    ws = torch.empty(zq.embedding_grad_bytes(T, V, D), dtype=torch.uint8, device=DEV)
    y, g = torch.empty_like(want_y), torch.empty_like(want_g)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        zq.embedding(ids, table, scale=3.0, out=y)
        zq.embedding_grad(ids, dy, V, out=g, workspace=ws)
    for i in range(3):
        y.zero_(), g.fill_(float("nan")), ws.fill_(0xFF)
        new = some_ids(T, V, 10 + i).to(DEV)
        ids.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, zq.embedding(new, table, scale=3.0)) and torch.equal(g, zq.embedding_grad(new, dy, V))
