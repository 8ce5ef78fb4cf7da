"""rms_norm, qwz_rms_norm and rms_norm_grad on the GPU against the definition in 64 bits."""
import itertools

import numpy as np
import pytest
import torch

import paper_2501_04266_amd as zq
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = 2.0**-24  # a binary32 rounding


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def rand(shape, dtype, seed, std=1.0, offset=0):
    """Normal values at an element offset of their memory."""
    n = int(np.prod(shape))
    g = torch.Generator().manual_seed(seed)
    base = torch.zeros(n + offset, dtype=dtype, device=DEV)
    base[offset:].copy_((torch.randn(n, generator=g) * std).to(dtype))
    return base[offset:].view(shape)


def check_forward(x, res, w, eps, y, h, rstd, what=""):
    T, D = x.shape
    if res is None:
        assert h is x
    else:
        assert torch.equal(h, (x.float() + res.float()).to(x.dtype)), what
    h64 = h.double()
    want_r = 1.0 / torch.sqrt(h64.square().sum(1) / D + eps)
    # binary64 throughout and one rounding
    assert bool(((rstd.double() - want_r).abs() <= 1.0001 * U * want_r).all()), f"{what} rstd"
    want = h64 * want_r[:, None] * (1.0 if w is None else w.double())
    # rstd, two products; the result's own rounding (and what 16 bits hold of tiny values)
    tol = (3.01 * U + half_step(y.dtype) * 1.01) * want.abs() + torch.finfo(y.dtype).smallest_normal * half_step(y.dtype) * 2
    assert bool(((y.double() - want).abs() <= tol).all()), f"{what} y"


WIDTHS = [1, 2, 7, 8, 9, 63, 65, 511, 512, 513, 1000, 2047, 2048, 2051, 4096, 4100, 6144, 6145, 8192, 8199, 16384, 16390,
          40000]


@pytest.mark.parametrize("D", WIDTHS)
def test_widths(D):
    for T, (dt, residual, wt, out), offset in zip((1, 2, 3, 5, 9), (("bf16", True, "f32", "bf16"), ("f32", True, "bf16", "f32"),
                                                                   ("f16", False, "f16", "f32"), ("bf16", False, None, "f16"),
                                                                   ("f16", True, "f32", "bf16")), (0, 1, 3, 1, 5)):
        x = rand((T, D), DT[dt], D, 1.0, offset)
        res = rand((T, D), DT[dt], D + 1, 2.0, offset) if residual else None
        w = None if wt is None else rand((D,), DT[wt], D + 2, 1.0, offset)
        y, h, rstd = zq.rms_norm(x, w, res, eps=1e-5, out_dtype=DT[out])
        check_forward(x, res, w, 1e-5, y, h, rstd, f"{dt} {T} x {D}")


@pytest.mark.parametrize("dt,wt,out", itertools.product(DT, [*DT, None], DT))
def test_types(dt, wt, out):
    x, res = rand((6, 328), DT[dt], 1), rand((6, 328), DT[dt], 2)
    w = None if wt is None else rand((328,), DT[wt], 3)
    for r in (res, None):
        y, h, rstd = zq.rms_norm(x, w, r, eps=1e-6, out_dtype=DT[out])
        check_forward(x, r, w, 1e-6, y, h, rstd)


@pytest.mark.parametrize("D", [96, 2048, 5000, 20000])
def test_sum_in_place(D):
    """h may be the residual's memory, or x's."""
    x, res = rand((7, D), torch.bfloat16, 1), rand((7, D), torch.bfloat16, 2)
    w = rand((D,), torch.float32, 3)
    y, h, rstd = zq.rms_norm(x, w, res)
    for k in (0, 1):
        a, b = x.clone(), res.clone()
        y2, h2, rstd2 = zq.rms_norm(a, w, b, hidden=(a, b)[k])
        assert h2 is (a, b)[k] and torch.equal(h2, h) and torch.equal(y2, y) and torch.equal(rstd2, rstd)
        assert torch.equal((b, a)[k], (res, x)[k])


@pytest.mark.parametrize("block,D", [(32, 32), (32, 96), (64, 448), (128, 512), (256, 512), (512, 512), (1024, 1024),
                                     (256, 1280), (1024, 2048), (512, 2560), (1024, 4096), (128, 6144), (1024, 7168),
                                     (1024, 8192), (32, 8224), (1024, 16384), (256, 16640), (1024, 20480)])
@pytest.mark.parametrize("dt", DT)
def test_int8(block, D, dt):
    """The codes and scales that the weights' quantiser gives for the binary32 output."""
    T = 5
    x, res = rand((T, D), DT[dt], D), rand((T, D), DT[dt], D + 1)
    x[2] = 0
    res[2] = 0  # a row of zeros
    x[3] *= 1e-3
    w = rand((D,), torch.float32, D + 2)
    for r in (res, None):
        y, h, rstd = zq.rms_norm(x, w, r, eps=1e-6, out_dtype=torch.float32)
        codes, scales, h8, rstd8 = zq.qwz_rms_norm(x, w, r, eps=1e-6, block=block)
        want, want_scales = zq.qwz_quantize(y.view(-1), block)
        assert torch.equal(codes.view(-1), want) and torch.equal(scales, want_scales)
        assert torch.equal(h8, h) and torch.equal(rstd8, rstd)


def test_large_and_small_values():
    """Squares beyond binary32's range, and below it."""
    for std in (1e30, 1e-30):
        x, w = rand((3, 700), torch.float32, 5, std), rand((700,), torch.float32, 6)
        y, h, rstd = zq.rms_norm(x, w, eps=0.0, out_dtype=torch.float32)
        check_forward(x, None, w, 0.0, y, h, rstd)


def test_rows_that_are_not_finite_stay_their_own():
    x, w = rand((9, 600), torch.float32, 5), rand((600,), torch.float32, 6)
    clean = zq.rms_norm(x, w)[0]
    x[3, 17], x[5, 2] = float("nan"), float("inf")
    x[7] = 0
    y = zq.rms_norm(x, w, eps=0.0)[0]
    assert bool(y[3].isnan().all()) and bool(y[7].isnan().all())  # 0 / 0
    assert bool(y[5, 2].isnan()) and bool((y[5, 3:] == 0).all())  # rstd is 0
    keep = [0, 1, 2, 4, 6, 8]
    assert bool(((y[keep] - clean[keep]).abs() <= 2e-6 * clean[keep].abs()).all())  # 1e-6 of a square's mean about 1


# ---------------------------------------------------------------- gradient

def reference(dy, h, w, rstd, dh):
    """dx, dw in 64 bits from the rounded rstd, and what binary32 may differ by."""
    T, D = h.shape
    dy, h = dy.double(), h.double()
    w = torch.ones(D, dtype=torch.float64, device=DEV) if w is None else w.double()
    s = rstd.double()[:, None]
    xh, gw = h * s, dy * w
    c = (gw * xh).sum(1, keepdim=True) / D
    dx = s * (gw - xh * c)
    # xh one rounding, gw one; a term of the sum 3 more than its order of additions, at most D
    c_off = (D + 4) * U * (gw * xh).abs().sum(1, keepdim=True) / D
    off = s * (xh.abs() * c_off + 5 * U * (gw.abs() + (xh * c).abs()))
    if dh is not None:
        dx = dx + dh.double()
    return (dx, (dy * xh).sum(0)), (off + 2 * U * dx.abs(), (T + 4) * U * (dy * xh).abs().sum(0))


def check_grad(dy, h, w, rstd, dh, dx, dw, what=""):
    (want_dx, want_dw), (off_dx, off_dw) = reference(dy, h, w, rstd, dh)
    tiny = torch.finfo(dx.dtype).smallest_normal * half_step(dx.dtype) * 2
    assert bool(((dx.double() - want_dx).abs() <= off_dx + 1.01 * half_step(dx.dtype) * want_dx.abs() + tiny).all()), f"{what} dx"
    tiny = torch.finfo(dw.dtype).smallest_normal * half_step(dw.dtype) * 2
    assert bool(((dw.double() - want_dw).abs() <= off_dw + 1.01 * half_step(dw.dtype) * want_dw.abs() + tiny).all()), f"{what} dw"


def rstd_of(h, eps=1e-6):
    return torch.rsqrt(h.double().square().mean(1) + eps).float()


@pytest.mark.parametrize("D", WIDTHS)
def test_gradient_widths(D):
    for T, (dt, gt, wt, more), offset in zip((1, 2, 7, 600), (("bf16", "bf16", "f32", True), ("f32", "f32", "f32", False),
                                                             ("f16", "f32", None, True), ("bf16", "f16", "bf16", True)), (0, 1, 3, 1)):
        if T == 600 and D > 9000:
            T = 40
        h, dy = rand((T, D), DT[dt], D, 1.0, offset), rand((T, D), DT[gt], D + 1, 0.01, offset)
        dh = rand((T, D), DT[dt], D + 2, 0.01, offset) if more else None
        w = None if wt is None else rand((D,), DT[wt], D + 3, 1.0, offset)
        rstd = rstd_of(h)
        dx, dw = zq.rms_norm_grad(dy, h, w, rstd, dh)
        check_grad(dy, h, w, rstd, dh, dx, dw, f"{dt} {gt} {T} x {D}")


@pytest.mark.parametrize("D", [1, 7, 16, 125, 136, 250, 256, 499, 512])
def test_gradient_narrow_rows(D):
    """Several groups of rows a workgroup: the last with all of them, with one and without
    one; the sums' memory behind its bytes stays as it was."""
    for T in (3, 4, 5, 15, 16, 17, 4097, 20001):
        h, dy, w = rand((T, D), torch.bfloat16, D, 1.0), rand((T, D), torch.bfloat16, D + 1, 0.01), rand((D,), torch.float32, 3, 1.0)
        rstd, need = rstd_of(h), zq.rms_norm_grad_bytes(T, D)
        ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device=DEV)
        dx, dw = zq.rms_norm_grad(dy, h, w, rstd, workspace=ws)
        check_grad(dy, h, w, rstd, None, dx, dw, f"{T} x {D}")
        assert bool((ws[need:] == 0xFF).all())


@pytest.mark.parametrize("dt,gt", itertools.product(DT, DT))
def test_gradient_types(dt, gt):
    for D in (328, 6000, 17000):
        h, dy, dh = rand((9, D), DT[dt], 1), rand((9, D), DT[gt], 2, 0.01), rand((9, D), DT[dt], 3, 0.01)
        rstd, w = rstd_of(h), rand((D,), torch.float32, 4)
        for out in DT.values():
            dx, dw = zq.rms_norm_grad(dy, h, w, rstd, dh, dweight=torch.empty(D, dtype=out, device=DEV))
            check_grad(dy, h, w, rstd, dh, dx, dw)


def test_gradient_many_rows_and_accumulation():
    T, D = 20011, 96
    h, dy, w = rand((T, D), torch.bfloat16, 1), rand((T, D), torch.bfloat16, 2, 0.01), rand((D,), torch.float32, 3)
    rstd = rstd_of(h)
    dx, dw = zq.rms_norm_grad(dy, h, w, rstd)
    check_grad(dy, h, w, rstd, None, dx, dw)
    again = zq.rms_norm_grad(dy, h, w, rstd)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)  # a fixed order
    total = dw.clone()
    zq.rms_norm_grad(dy, h, w, rstd, dweight=total, accumulate=True)
    assert torch.equal(total, dw + dw)


@pytest.mark.parametrize("D", [300, 3000, 18000])
def test_gradient_in_the_place_of_dh(D):
    h, dy, dh = rand((11, D), torch.float16, 1), rand((11, D), torch.float16, 2, 0.01), rand((11, D), torch.float16, 3, 0.01)
    rstd, w = rstd_of(h), rand((D,), torch.float32, 4)
    dx, dw = zq.rms_norm_grad(dy, h, w, rstd, dh)
    keep = dh.clone()
    dx2, dw2 = zq.rms_norm_grad(dy, h, w, rstd, keep, out=keep)
    assert dx2 is keep and torch.equal(dx, dx2) and torch.equal(dw, dw2)


def test_gradient_against_differences():
    """dx and dw are the slopes of sum(dy * rms_norm(x)): central differences in 64 bits of
    the definition, whose own error at a step of 1e-4 is about 1e-8 of the terms."""
    T, D, eps = 3, 40, 1e-3
    x, res = rand((T, D), torch.float32, 1), rand((T, D), torch.float32, 2)
    w, dy, dh = rand((D,), torch.float32, 3), rand((T, D), torch.float32, 4), rand((T, D), torch.float32, 5)
    y, h, rstd = zq.rms_norm(x, w, res, eps=eps)
    dx, dw = zq.rms_norm_grad(dy, h, w, rstd, dh)

    def value(x, w):
        s = x + res.double()
        return (dy.double() * s / torch.sqrt(s.square().mean(1, keepdim=True) + eps) * w + dh.double() * s).sum()

    x64, w64, d = x.double(), w.double(), 1e-4
    slopes = torch.zeros_like(x64)
    for i in range(T * D):
        e = torch.zeros(T * D, dtype=torch.float64, device=DEV)
        e[i] = d
        slopes.view(-1)[i] = (value(x64 + e.view(T, D), w64) - value(x64 - e.view(T, D), w64)) / (2 * d)
    # the sum h is rounded (2^-24 of it), which moves the slope as little; binary32 as above
    assert bool(((dx.double() - slopes).abs() <= 1e-5 + 1e-5 * slopes.abs()).all())
    for i in range(D):
        e = torch.zeros(D, dtype=torch.float64, device=DEV)
        e[i] = d
        slope = (value(x64, w64 + e) - value(x64, w64 - e)) / (2 * d)
        assert abs(float(dw[i]) - float(slope)) <= 1e-5 * (1 + abs(float(slope)))


# ---------------------------------------------------------------- how it is called

def test_no_rows():
    x = torch.empty(0, 64, device=DEV)
    w = torch.ones(64, device=DEV)
    y, h, rstd = zq.rms_norm(x, w, x)
    assert y.shape == (0, 64) and rstd.numel() == 0
    zq.qwz_rms_norm(x, w, block=64)
    dx, dw = zq.rms_norm_grad(x, x, w, rstd)
    assert dx.shape == (0, 64) and not bool(dw.any())
    held = torch.full((64,), 3.0, device=DEV)
    zq.rms_norm_grad(x, x, w, rstd, dweight=held, accumulate=True)
    assert bool((held == 3.0).all())


def test_more_dimensions():
    x, res, w = rand((2, 3, 80), torch.bfloat16, 1), rand((2, 3, 80), torch.bfloat16, 2), rand((80,), torch.float32, 3)
    y, h, rstd = zq.rms_norm(x, w, res)
    assert y.shape == h.shape == x.shape and rstd.shape == (6,)
    check_forward(x.view(6, 80), res.view(6, 80), w, 1e-6, y.view(6, 80), h.view(6, 80), rstd)
    dx, _ = zq.rms_norm_grad(y, h, w, rstd)
    assert dx.shape == x.shape


def test_memory_around_the_rows_stays():
    for D in (9, 515, 2050, 5001, 17003):
        T = 3
        base = torch.full((T * D + 40,), 7.0, dtype=torch.bfloat16, device=DEV)
        out, h = base[11:11 + T * D].view(T, D), base.clone()[13:13 + T * D].view(T, D)
        x = rand((T, D), torch.bfloat16, 1)
        zq.rms_norm(x, None, x.clone(), out=out, hidden=h)
        hb = h._base if h._base is not None else h
        assert bool((base[:11] == 7).all()) and bool((base[11 + T * D:] == 7).all())
        assert bool((hb[:13] == 7).all()) and bool((hb[13 + T * D:] == 7).all())
        grad = torch.full((T * D + 40,), 7.0, dtype=torch.bfloat16, device=DEV)
        dw = torch.full((D + 9,), 7.0, device=DEV)
        zq.rms_norm_grad(x, h, None, rstd_of(h), out=grad[5:5 + T * D].view(T, D), dweight=dw[3:3 + D])
        assert bool((grad[:5] == 7).all()) and bool((grad[5 + T * D:] == 7).all())
        assert bool((dw[:3] == 7).all()) and bool((dw[3 + D:] == 7).all())


def test_graph_and_streams():
    T, D = 300, 1024
    x, res, dy, dh = (rand((T, D), torch.bfloat16, s) for s in range(4))
    w = rand((D,), torch.float32, 9)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    zq.rms_norm_grad(dy, x, w, rstd_of(x))  # the same leaves, eagerly, before the capture
    with torch.cuda.graph(graph, stream=side):
        y, h, rstd = zq.rms_norm(x, w, res)
        dx, dw = zq.rms_norm_grad(dy, h, w, rstd, dh)
        codes, scales, _, _ = zq.qwz_rms_norm(x, w, res, block=128)
    for turn in range(3):
        x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        y2, h2, rstd2 = zq.rms_norm(x, w, res)
        dx2, dw2 = zq.rms_norm_grad(dy, h2, w, rstd2, dh)
        c2, s2, _, _ = zq.qwz_rms_norm(x, w, res, block=128)
        for a, b in ((y, y2), (h, h2), (rstd, rstd2), (dx, dx2), (dw, dw2), (codes, c2), (scales, s2)):
            assert torch.equal(a, b), f"replay {turn}"
    other = zq.rms_norm_grad(dy, h2, w, rstd2, dh, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(other[0], dx2) and torch.equal(other[1], dw2)


def test_rows_beyond_2_32_elements():
    T, D = 2**32 // 6144 + 3, 6144
    x = torch.zeros(T, D, dtype=torch.bfloat16, device=DEV)
    x[-2:] = rand((2, D), torch.bfloat16, 1)
    w = rand((D,), torch.float32, 2)
    y, _, rstd = zq.rms_norm(x, w)
    small, _, small_r = zq.rms_norm(x[-2:].clone(), w)
    assert torch.equal(y[-2:], small) and torch.equal(rstd[-2:], small_r) and not bool(y[:-2].any())
    dx, dw = zq.rms_norm_grad(y, x, w, rstd)
    sdx, sdw = zq.rms_norm_grad(small, x[-2:].clone(), w, small_r)
    assert torch.equal(dx[-2:], sdx) and not bool(dx[:-2].any())
    assert bool(((dw - sdw).abs() <= 2.0**-22 * sdw.abs() + 1e-30).all())


@pytest.mark.parametrize("out", ["f16", "bf16", "f32"])
def test_weight_gradient_added_in_its_type(out):
    T, D = 50, 520
    h, dy, w = rand((T, D), torch.float32, 1), rand((T, D), torch.float32, 2), rand((D,), torch.float32, 3)
    rstd = rstd_of(h)
    held = rand((D,), DT[out], 4, 10.0)
    start = held.double()
    zq.rms_norm_grad(dy, h, w, rstd, dweight=held, accumulate=True)
    (_, want), (_, off) = reference(dy, h, w, rstd, None)
    assert bool(((held.double() - start - want).abs() <= off + 2 * U * (start + want).abs() + 1.01 * half_step(DT[out]) * (start + want).abs() + 1e-7).all())


@pytest.mark.parametrize("D", [64, 1000, 6144, 20000])
def test_x_as_its_own_residual(D):
    x, w = rand((3, D), torch.bfloat16, 1), rand((D,), torch.float32, 2)
    y, h, rstd = zq.rms_norm(x, w, x)
    check_forward(x, x, w, 1e-6, y, h, rstd)
    keep = x.clone()
    y2, h2, _ = zq.rms_norm(keep, w, keep, hidden=keep)
    assert torch.equal(h2, h) and torch.equal(y2, y)


def test_one_row():
    x, w = rand((700,), torch.float32, 1), rand((700,), torch.float32, 2)
    y, h, rstd = zq.rms_norm(x, w)
    want = x.double() * torch.rsqrt(x.double().square().mean() + 1e-6) * w.double()
    assert y.shape == (700,) and h is x and rstd.shape == (1,)
    assert bool(((y.double() - want).abs() <= 4.1 * U * want.abs()).all())
