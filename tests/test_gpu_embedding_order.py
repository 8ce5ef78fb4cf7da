"""The order in which the embedding gradient adds a row's tokens, bit for bit: binary32
additions, tokens ascending; with more than 512 tokens in all, a row that holds a whole
64 positions of the tokens sorted by row (from a multiple of 64 on) is summed up to the
next multiple, by 64s, and these sums in their order."""
import numpy as np
import pytest
import torch

import paper_2501_04266_amd as zq
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu


def total(rows):
    acc = np.zeros(rows.shape[1], np.float32)
    for r in rows:
        acc = acc + r
    return acc


def gradient(ids, dy, V, few):
    order = np.argsort(ids, kind="stable")
    order = order[(ids[order] >= 0) & (ids[order] < V)]
    want = np.zeros((V, dy.shape[1]), np.float32)
    start = np.searchsorted(ids[order], np.arange(V + 1))
    for v in np.unique(ids[order]):
        s, e = int(start[v]), int(start[v + 1])
        if few or -(-s // 64) >= e // 64:
            want[v] = total(dy[order[s:e]])
        else:
            cuts = sorted({s, e, *range(-(-s // 64) * 64, e, 64)})
            want[v] = total(np.stack([total(dy[order[a:b]]) for a, b in zip(cuts, cuts[1:])]))
    return want


@pytest.mark.parametrize("T,V,kind", [(5000, 400, "even"), (5000, 40, "even"), (513, 3, "even"), (512, 60, "even"),
                                      (512, 2, "even"), (20000, 2000, "skewed"), (70000, 1537, "skewed"),
                                      (9000, 70000, "skewed"), (4096, 64, "turns"), (6000, 1, "even")])
def test_order(T, V, kind):
    g = np.random.default_rng(T + V)
    if kind == "turns":  # every lane of a wave another row, then the same
        ids = np.where(np.arange(T) // 64 % 2 == 0, np.arange(T) % 64, np.arange(T) // 128 % 64)
    else:
        ids = (V * (g.random(T) ** (4 if kind == "skewed" else 1))).astype(np.int64)
    ids[g.random(T) < 0.05] = -1
    # magnitudes apart, so that another order rounds otherwise
    dy = (g.standard_normal((T, 9)) * 2.0 ** g.integers(-12, 13, (T, 9))).astype(np.float32)
    got = zq.embedding_grad(torch.from_numpy(ids).to(DEV), torch.from_numpy(dy).to(DEV), V).cpu().numpy()
    want = gradient(ids, dy, V, T <= 512)
    bad = np.argwhere(got.view(np.uint32) != want.view(np.uint32))
    assert len(bad) == 0, f"{len(bad)} differ, first at {bad[0].tolist()}"
