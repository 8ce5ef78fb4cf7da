"""rms_norm_grad's sum over a row, place by place."""
import pytest
import torch

import paper_2501_04266_amd as zq
from tests.gpu_util import DEV
from tests.plain_rms import DT, inputs, places, row_gradient, rows_off
from tests.test_rms_gradient_bounds import TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [1, 2, 7, 8, 9, 33, 63, 129, 136, 257, 513, 1000, 1025, 1537, 2047, 2048, 2049, 2051, 4096, 4099, 6144,
                               6147, 8192, 8195, 8199, 16384, 16385, 16390, 16391, 20000, 40000])
@pytest.mark.parametrize("dt,gt,wt,more", TYPES)
def test_every_place_counts(D, dt, gt, wt, more):
    """Each row has a third of its sum at a place of its own: ends of vectors, of turns, of the row."""
    for offset in (0, 3):
        data = inputs(D, dt, gt, wt, more, DEV, offset)
        dx, _ = zq.rms_norm_grad(*data)
        bad = rows_off(dx, *row_gradient(*data))
        assert not bool(bad.any()), f"offset {offset}: places {[k for k, b in zip(places(D), bad.tolist()) if b]}"


@pytest.mark.parametrize("D", [16, 32, 48, 64, 96, 528, 544, 1024, 1056, 2064, 2080, 4096, 4128, 6176, 8224])
@pytest.mark.parametrize("dt,gt", [("bf16", "bf16"), ("f16", "f16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "f16")])
def test_addresses_do_not_show(D, dt, gt):
    """Rows of whole lines, of halves of them, and from any element's address: the same bits."""
    for T in (1, 517):
        g = torch.Generator().manual_seed(D + T)
        h, dy, dh = (torch.randn(T, D, generator=g).to(DT[t]).to(DEV) for t in (dt, gt, dt))
        w, rstd = torch.randn(D, generator=g).to(DEV), torch.rsqrt(h.float().square().mean(1) + 1e-6)
        dx, dw = zq.rms_norm_grad(dy, h, w, rstd, dh)

        def moved(x, by):
            base = torch.empty(x.numel() + by, dtype=x.dtype, device=DEV)
            base[by:].copy_(x.view(-1))
            return base[by:].view(x.shape)

        for by in (1, 64 // dx.element_size()):
            out = moved(torch.empty_like(dx), by)
            for args in ((dy, h, dh), (moved(dy, by), moved(h, by), moved(dh, by))):
                again, dw2 = zq.rms_norm_grad(args[0], args[1], w, rstd, args[2], out=out)
                assert again is out and torch.equal(out, dx) and torch.equal(dw2, dw), f"{T} x {D} from {by}"
