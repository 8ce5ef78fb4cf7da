"""rms_norm_grad's sum over a row, place by place."""
import pytest

import paper_2501_04266_amd as zq
from tests.gpu_util import DEV
from tests.plain_rms import inputs, places, row_gradient, rows_off
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
