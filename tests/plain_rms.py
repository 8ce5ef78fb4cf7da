"""The gradient of the RMS norm in 64 bits, with bounds that follow from the order in which
the kernels add, on inputs where every place of a row matters (no GPU needed)."""
import torch

U = 2.0**-24  # a binary32 rounding
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def places(D):
    """Places of a row: all of a short one; of a long one its ends, the ends of what threads and
    turns hold, and some between."""
    if D <= 40:
        return list(range(D))
    body = D - D % 8  # whole vectors; then one element a thread
    at = {0, 1, 7, 8, D - 1, D - 2, D - 8, D - 9, body - 8, body - 1, body - 9, body, D // 2, D // 3, 2 * D // 3}
    for threads in (16, 32, 64, 128, 192, 256, 512, 1024):
        at |= {8 * threads - 1, 8 * threads, 16 * threads, 24 * threads}
    return sorted(k for k in at | set(range(body, D)) if 0 <= k < D)


def inputs(D, dt, gt, wt, more, dev, offset=0):
    """A row for each of places(D): gradients along the normed row, so that its sum has no
    cancellation, and a third of the sum at that place."""
    at = places(D)
    T = len(at)
    g = torch.Generator().manual_seed(D)

    def held(x, dtype):
        base = torch.zeros(x.numel() + offset, dtype=dtype, device=dev)
        base[offset:].copy_(x.reshape(-1))
        return base[offset:].view(x.shape)

    h = torch.randn(T, D, generator=g)
    dy = 0.01 * h
    rows = torch.arange(T)
    h[rows, at] = 1.0
    dy[rows, at] = 0.005 * D + 0.01
    w = None if wt is None else held(1.0 + 0.1 * torch.rand(D, generator=g), DT[wt])
    dh = held(0.01 * torch.randn(T, D, generator=g), DT[dt]) if more else None
    h = held(h, DT[dt])
    rstd = torch.rsqrt(h.double().square().mean(1) + 1e-6).float()
    return held(dy, DT[gt]), h, w, rstd, dh


def additions(D):
    """Binary32 additions that a term of a row's sum goes through: up to 4 vectors of 8 and a
    single one a thread, 6 exchanges in a wave, 16 waves; above 16,384 places those of one
    vector, the rest in binary64."""
    return 33 + 6 + 15 if D <= 16384 else 8


def row_gradient(dy, h, w, rstd, dh, left_out=()):
    """(dx, what it may be off by) in 64 bits; left_out: places missing from the row's sum."""
    D = h.shape[1]
    dy, h, s = dy.double(), h.double(), rstd.double()[:, None]
    xh, gw = h * s, dy * (1.0 if w is None else w.double())
    term = gw * xh
    # a term: xh, gw, their product; the sum's additions; the division by D
    c_off = (additions(D) + 4) * U * term.abs().sum(1, keepdim=True) / D
    for k in left_out:
        term[:, k] = 0.0
    c = term.sum(1, keepdim=True) / D
    dx = s * (gw - xh * c)
    # gw and xh, the product with c, the difference, the product with rstd; dh's addition
    off = s * (xh.abs() * c_off + 5 * U * (gw.abs() + (xh * c).abs()))
    if dh is not None:
        dx = dx + dh.double()
    return dx, off + 2 * U * dx.abs()


def rows_off(dx, want, off):
    """Which rows of dx are further from `want` than they may be."""
    tiny = torch.finfo(dx.dtype).smallest_normal * half_step(dx.dtype) * 2
    return ((dx.double() - want).abs() > off + 1.01 * half_step(dx.dtype) * want.abs() + tiny).any(1)
