"""The embedding gradient's limits on tokens and rows together: its sort's reads grow
with their product, so a call that would keep the GPU busy for minutes is refused (no
kernel is launched here)."""
import os

import pytest

import paper_2501_04266_amd as zq
from paper_2501_04266_amd import _lib

SIZE, ALIAS = -5, -8
A, B, W = (k << 52 for k in range(1, 4))


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2501_04266_amd import build
        build.build()
    return _lib.lib()


@pytest.mark.parametrize("T,V,taken", [
    (1 << 30, 1 << 20, True), (1 << 30, (1 << 20) + 1, False), (1 << 20, 1 << 30, True), ((1 << 20) + 1, 1 << 30, False),
    (1 << 30, 1 << 30, False), (1 << 22, 1 << 24, True), (512, 1 << 30, True), (0, 1 << 30, True), (1 << 30, 1, True)])
def test_tokens_times_rows(L, T, V, taken):
    assert (L.zq_embedding_grad_bytes(T, V, 1) >= 0) == taken
    # with all else in order but the result on the token ids
    if T:
        assert L.zq_embedding_grad(A, 4, T, B, 2, V, 1, 1.0, 0, A, 0, W, 1 << 51, None) == (ALIAS if taken else SIZE)
    if not taken:
        with pytest.raises(ValueError):
            zq.embedding_grad_bytes(T, V, 1)
