"""The bound on the RMS norm's gradient notices a row's sum that lacks a place, and takes one
in binary32 (no GPU needed)."""
import pytest
import torch

from tests.plain_rms import DT, inputs, places, row_gradient, rows_off

TYPES = [("bf16", "bf16", "f32", True), ("f32", "f32", "f32", False), ("f16", "f32", None, True), ("bf16", "f16", "bf16", True)]


@pytest.mark.parametrize("D", [7, 9, 129, 2051, 8199, 16390, 16391, 40000])
@pytest.mark.parametrize("dt,gt,wt,more", TYPES)
def test_a_missing_place_shows(D, dt, gt, wt, more):
    data = inputs(D, dt, gt, wt, more, "cpu")
    want, off = row_gradient(*data)
    assert not bool(rows_off(want.to(DT[dt]), want, off).any())
    at = places(D)
    tail = range(D - D % 8, D)
    for left_out in ([at[0]], [at[-1]], list(tail), list(range(max(0, D - 8), D)), [at[len(at) // 2]]):
        dx, _ = row_gradient(*data, left_out=left_out)
        bad = rows_off(dx.to(DT[dt]), want, off)
        assert bool(bad[[k in left_out for k in at]].all()), f"without {left_out}"
        if not left_out:
            assert not bool(bad.any())


@pytest.mark.parametrize("D", [129, 2051, 16391])
def test_binary32_is_within(D):
    """Binary32 throughout, summed a vector at a time and then over the vectors by halves."""
    dy, h, w, rstd, dh = inputs(D, "f32", "f32", "f32", False, "cpu")
    xh, gw = h * rstd[:, None], dy * w
    term = torch.nn.functional.pad(gw * xh, (0, -D % 8)).view(len(h), -1, 8)
    c = term[:, :, 0].clone()
    for k in range(1, 8):
        c += term[:, :, k]
    c = torch.nn.functional.pad(c, (0, 4096 - c.shape[1]))
    while c.shape[1] > 1:
        c = c[:, : c.shape[1] // 2] + c[:, c.shape[1] // 2:]
    dx = (gw - xh * (c / D)) * rstd[:, None]
    want, off = row_gradient(dy, h, w, rstd, dh)
    assert not bool(rows_off(dx, want, off).any())
