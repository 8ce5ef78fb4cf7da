"""Refusals of the embedding, gradient-norm and INT4-product calls (no kernel is
launched: every check comes before anything is enqueued), with fake device
addresses at the C ABI and CPU tensors at the binding; and the gradient table's
layout, which is made on the host."""
import ctypes
import os

import pytest
import torch

import paper_2501_04266_amd as zq
from paper_2501_04266_amd import _lib

A, B, C, W = 0x7F0000000000, 0x7F0010000000, 0x7F0020000000, 0x7F0030000000
V = 0x7F0040000000
NULL, ALIGN, SIZE, BLOCK, DTYPE, ALIAS = -1, -4, -5, -2, -3, -8


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2501_04266_amd import build
        build.build()
    return _lib.lib()


# (ids, id type, T, table, dtype, V, D, scale, y, dtype, stream)
@pytest.mark.parametrize("args,status", [
    ((A, 4, -1, B, 2, 100, 64, 1.0, C, 2, None), SIZE),
    ((A, 4, 10, B, 2, -1, 64, 1.0, C, 2, None), SIZE),
    ((A, 4, 10, B, 2, 100, -64, 1.0, C, 2, None), SIZE),
    ((A, 4, 10, B, 2, 100, (1 << 24) + 1, 1.0, C, 2, None), SIZE),
    ((A, 4, 1 << 60, B, 2, 100, 64, 1.0, C, 2, None), SIZE),
    ((A, 4, 10, B, 2, 1 << 60, 64, 1.0, C, 2, None), SIZE),
    ((A, 4, 1 << 40, B, 2, 100, 64, 1.0, C + (1 << 50), 2, None), SIZE),   # more workgroups than a launch takes
    ((A, 0, 10, B, 2, 100, 64, 1.0, C, 2, None), DTYPE),
    ((A, 4, 10, B, 3, 100, 64, 1.0, C, 2, None), DTYPE),
    ((A, 4, 10, B, -1, 100, 64, 1.0, C, 2, None), DTYPE),
    ((A, 4, 10, B, 2, 100, 64, 1.0, C, 5, None), DTYPE),
    ((None, 4, 10, B, 2, 100, 64, 1.0, C, 2, None), NULL),
    ((A, 4, 10, None, 2, 100, 64, 1.0, C, 2, None), NULL),
    ((A, 4, 10, B, 2, 100, 64, 1.0, None, 2, None), NULL),
    ((A + 4, 4, 10, B, 2, 100, 64, 1.0, C, 2, None), ALIGN),
    ((A, 4, 10, B + 1, 2, 100, 64, 1.0, C, 2, None), ALIGN),
    ((A, 4, 10, B, 2, 100, 64, 1.0, C + 2, 0, None), ALIGN),
    ((A, 4, 10, B, 2, 100, 64, 1.0, B + 100 * 64 * 2 - 2, 2, None), ALIAS),
    ((A, 4, 10, B, 2, 100, 64, 1.0, A + 72, 2, None), ALIAS),
    ((None, 4, 0, None, 2, 100, 64, 1.0, None, 2, None), 0),
    ((None, 3, 10, None, 2, 100, 0, 1.0, None, 2, None), 0),
])
def test_embedding_argument_errors(L, args, status):
    assert L.zq_embedding(*args) == status


@pytest.mark.parametrize("args,status", [
    ((A, 4, 10, B, W, 100, 64, 100, 1.0, C, 2, None), BLOCK),
    ((A, 4, 10, B, W, 100, 64, 16, 1.0, C, 2, None), BLOCK),
    ((A, 4, 10, B, None, 100, 64, 256, 1.0, C, 2, None), NULL),
    ((A, 4, 10, B, W + 2, 100, 64, 256, 1.0, C, 2, None), ALIGN),
    ((A, 4, 10, B, W, 100, 64, 256, 1.0, W + 96, 2, None), ALIAS),   # 25 scales: 100 bytes
    ((A, 4, 10, B, W, 100, 64, 256, 1.0, B + 6399, 2, None), ALIGN),
    ((A, 4, 10, B, W, 100, 64, 256, 1.0, B + 6398, 2, None), ALIAS),
    ((A, 7, 10, B, W, 100, 64, 256, 1.0, C, 2, None), DTYPE),
    ((A, 4, 0, None, None, 100, 64, 256, 1.0, None, 2, None), 0),
])
def test_int8_embedding_argument_errors(L, args, status):
    assert L.qwz_embedding(*args) == status


def test_embedding_grad_argument_errors(L):
    f = L.zq_embedding_grad
    need = L.zq_embedding_grad_bytes(1000, 50, 64)
    assert need >= 4 * 51 + 4 * 1000   # first positions, the order, and partial sums
    assert L.zq_embedding_grad_bytes(0, 0, 0) == 0 and L.zq_embedding_grad_bytes(100, 50, 64) == 0  # one launch
    for bad in ((-1, 50, 64), (100, -1, 64), (100, 50, -1), ((1 << 30) + 1, 50, 64), (100, (1 << 30) + 1, 64),
                (100, 50, (1 << 24) + 1)):
        assert L.zq_embedding_grad_bytes(*bad) == -1
        T, V, D = bad
        assert f(A, 4, T, B, 2, V, D, 1.0, 0, C, 0, W, 1 << 40, None) == SIZE

    def call(ids=A, it=4, T=1000, dy=B, gt=2, V=50, D=64, acc=0, dw=C, wt=0, ws=W, size=need):
        return f(ids, it, T, dy, gt, V, D, 1.0, acc, dw, wt, ws, size, None)

    assert call(it=2) == DTYPE and call(gt=4) == DTYPE and call(wt=-2) == DTYPE
    assert call(ids=None) == NULL and call(dy=None) == NULL and call(dw=None) == NULL and call(ws=None) == NULL
    assert call(ids=A + 4) == ALIGN and call(dy=B + 1) == ALIGN and call(dw=C + 2) == ALIGN and call(ws=W + 8) == ALIGN
    assert call(size=need - 1) == SIZE
    assert call(dw=B) == ALIAS and call(dw=A + 7996) == ALIAS and call(ws=B) == ALIAS and call(ws=A) == ALIAS
    assert call(ws=C + 64) == ALIAS
    assert call(V=0, dw=None, ws=None) == 0 and call(D=0, dw=None, ws=None) == 0
    assert call(T=0, acc=1, ids=None, dy=None, dw=None, ws=None) == 0
    # few tokens, without a workspace
    assert call(T=100, ws=None, size=0, ids=None) == NULL and call(T=100, ws=None, size=0, dw=B) == ALIAS
    assert call(T=100, ws=None, size=-1) == SIZE


def grad(data=A, n=100, dtype=0, scales=None, out=None, out_dtype=0, block=0):
    return _lib._Grad(data, scales, out, n, dtype, out_dtype, block, 0)


def plan_of(L, *grads):
    plan = _lib._GradPlan()
    return L.zq_grad_plan_make((_lib._Grad * max(1, len(grads)))(*grads), len(grads), ctypes.byref(plan)), plan


@pytest.mark.parametrize("grads,status", [
    ([], 0),
    ([dict(n=0, data=None)], 0),
    ([dict()], 0),
    ([dict(n=-1)], SIZE),
    ([dict(n=1 << 62)], SIZE),
    ([dict(dtype=3)], DTYPE),
    ([dict(dtype=7)], DTYPE),
    ([dict(out=B, out_dtype=5)], DTYPE),
    ([dict(data=None)], NULL),
    ([dict(dtype=5, block=64)], NULL),
    ([dict(dtype=5, block=48, scales=B)], BLOCK),
    ([dict(data=A + 2)], ALIGN),
    ([dict(data=A + 1, dtype=2)], ALIGN),
    ([dict(data=A + 1, dtype=5, block=32, scales=B)], 0),
    ([dict(dtype=5, block=32, scales=B + 2)], ALIGN),
    ([dict(out=B + 2)], ALIGN),
    ([dict(out=B + 2, out_dtype=2)], 0),
    ([dict(out=A)], 0),                                        # in place, said so
    ([dict(out=A, out_dtype=2)], ALIAS),                       # in place as another type
    ([dict(out=A + 396)], ALIAS),
    ([dict(out=A + 400)], 0),
    ([dict(), dict(data=A + 396)], ALIAS),                     # two tensors in place on shared memory
    ([dict(), dict(data=A + 400)], 0),
    ([dict(out=B), dict(out=B + 396)], ALIAS),
    ([dict(out=B), dict(out=C)], 0),                           # one tensor twice, read only
    ([dict(out=B), dict(data=B + 396)], ALIAS),                # an out over another tensor
    ([dict(data=A, n=1000, out=B), dict(data=A + 4, n=1, out=C), dict(data=W, n=1, out=A + 3996)], ALIAS),
    ([dict(data=A, dtype=5, block=32, scales=A + 48)], ALIAS),  # scales, clipped in place, over the codes (50 bytes)
    ([dict(data=A, dtype=5, block=32, scales=A + 52)], 0),
    ([dict(data=A, dtype=5, block=32, scales=B, out=B + 12)], ALIAS),
    ([dict(data=A, dtype=5, block=32, scales=B, out=B + 16)], 0),
])
def test_grad_plan_errors(L, grads, status):
    assert plan_of(L, *[grad(**g) for g in grads])[0] == status


def test_grad_plan_and_call_errors(L):
    assert L.zq_grad_plan_make(None, 1, ctypes.byref(_lib._GradPlan())) == NULL
    assert L.zq_grad_plan_make((_lib._Grad * 1)(grad()), 1, None) == NULL
    assert L.zq_grad_plan_make((_lib._Grad * 1)(grad()), -1, ctypes.byref(_lib._GradPlan())) == SIZE
    rc, plan = plan_of(L, grad(n=10_000), grad(data=B, n=100_000, dtype=5, block=128, scales=C), grad(data=W, n=0))
    assert rc == 0 and plan.count == 3
    assert plan.norm_chunks >= 2 and plan.clip_chunks >= 2
    entries = (_lib._Grad * 3)(grad(n=10_000), grad(data=B, n=100_000, dtype=5, block=128, scales=C), grad(data=W, n=0))
    assert L.zq_grad_plan_table(entries, ctypes.byref(plan), None) == NULL
    assert L.zq_grad_plan_table(None, ctypes.byref(plan), ctypes.create_string_buffer(plan.bytes)) == NULL
    buf = ctypes.create_string_buffer(b"\xa5" * (plan.bytes + 8), plan.bytes + 8)
    assert L.zq_grad_plan_table(entries, ctypes.byref(plan), buf) == 0
    assert buf.raw[plan.bytes:] == b"\xa5" * 8
    p = ctypes.byref(plan)
    assert L.zq_grad_norm(None, A, 1.0, B, None) == NULL and L.zq_grad_norm(p, None, 1.0, B, None) == NULL
    assert L.zq_grad_norm(p, A, 1.0, None, None) == NULL and L.zq_grad_norm(p, A + 8, 1.0, B, None) == ALIGN
    assert L.zq_grad_norm(p, A, 1.0, B + 2, None) == ALIGN
    assert L.zq_grad_clip(None, A, B, 1.0, 1.0, None) == NULL and L.zq_grad_clip(p, None, B, 1.0, 1.0, None) == NULL
    assert L.zq_grad_clip(p, A, None, 1.0, 1.0, None) == NULL and L.zq_grad_clip(p, A + 4, B, 1.0, 1.0, None) == ALIGN
    assert L.zq_grad_clip(p, A, B, -1.0, 1.0, None) == SIZE
    assert L.zq_grad_clip(p, A, B, float("nan"), 1.0, None) == SIZE
    assert L.zq_grad_clip(ctypes.byref(plan_of(L)[1]), A, B, 1.0, 1.0, None) == 0   # no tensors: nothing to do


def test_int4_gemm_argument_errors(L):
    def f(*a):  # (x, xt, packed, scales, M, N, K, block, y, stream)
        return L.zq_int4_dequant_gemm(*a[:-1], None, 0, a[-1])
    assert f(A, 0, B, C, 4, 4, 64, 128, W, None) == DTYPE
    assert f(A, 2, B, C, 4, 4, 96, 128, W, None) == SIZE
    assert f(A, 2, B, C, 4, 4, (1 << 22) + 64, 128, W, None) == SIZE
    assert f(A, 2, B, C, -1, 4, 64, 128, W, None) == SIZE and f(A, 2, B, C, 4, -1, 64, 128, W, None) == SIZE
    assert f(A, 2, B, C, 4, 1 << 60, 64, 128, W, None) == SIZE and f(A, 2, B, C, 1 << 60, 4, 64, 128, W, None) == SIZE
    assert f(A, 2, B, C, 4, 4, 64, 100, W, None) == BLOCK
    assert f(None, 2, B, C, 4, 4, 64, 128, W, None) == NULL and f(A, 2, None, C, 4, 4, 64, 128, W, None) == NULL
    assert f(A, 2, B, None, 4, 4, 64, 128, W, None) == NULL and f(A, 2, B, C, 4, 4, 64, 128, None, None) == NULL
    assert f(A + 8, 2, B, C, 4, 4, 64, 128, W, None) == ALIGN and f(A, 2, B + 8, C, 4, 4, 64, 128, W, None) == ALIGN
    assert f(A, 2, B, C + 2, 4, 4, 64, 128, W, None) == ALIGN and f(A, 1, B, C, 4, 4, 64, 128, W + 2, None) == ALIGN
    assert f(A, 2, B, C, 4, 4, 64, 128, A + 508, None) == ALIAS and f(A, 2, B, C, 4, 4, 64, 128, B + 124, None) == ALIAS
    assert f(A, 2, B, C, 4, 4, 64, 128, C + 4, None) == ALIAS
    assert f(None, 2, None, None, 0, 4, 64, 128, None, None) == 0 and f(None, 2, None, None, 4, 0, 64, 128, None, None) == 0


def test_int4_gemm_workspace(L):
    f, need = L.zq_int4_dequant_gemm, L.zq_int4_dequant_gemm_bytes(8, 32, 24576)
    assert need > 0 and need % (4 * 8 * 32) == 0 and L.zq_int4_dequant_gemm_bytes(8, 32, 64) == 0
    args = (A, 2, B, C, 8, 32, 24576, 128, W)
    assert f(*args, None, 0, None) == SIZE and f(*args, V, need - 1, None) == SIZE and f(*args, None, need, None) == NULL
    assert f(*args, V + 2, need, None) == ALIGN and f(*args, A, need, None) == ALIAS and f(*args, W, need, None) == ALIAS
    for bad in ((-1, 4, 64), (4, -1, 64), (4, 4, 65), (4, 4, -64), (1 << 40, 4, 64), (4, 1 << 60, 64)):
        assert L.zq_int4_dequant_gemm_bytes(*bad) == -1
    assert L.zq_int4_dequant_gemm_bytes(0, 4, 64) == 0 and L.zq_int4_dequant_gemm_bytes(4, 0, 64) == 0


def test_binding_refusals():
    ids = torch.zeros(6, dtype=torch.int64)
    table = torch.zeros((10, 8))
    with pytest.raises(TypeError):
        zq.embedding(ids.float(), table)
    with pytest.raises(TypeError):
        zq.embedding(ids, table.double())
    with pytest.raises(ValueError):
        zq.embedding(ids, table.view(-1))
    with pytest.raises(ValueError):
        zq.embedding(ids, table, out=torch.zeros(47))
    with pytest.raises(TypeError):
        zq.embedding(ids, table)                      # not on a GPU
    with pytest.raises(ValueError):
        zq.qwz_embedding(ids, torch.zeros(79, dtype=torch.int8), torch.zeros(1), 10, 8)
    with pytest.raises(ValueError):
        zq.qwz_embedding(ids, torch.zeros(80, dtype=torch.int8), torch.zeros(2), 10, 8, block=32)
    with pytest.raises(TypeError):
        zq.qwz_embedding(ids, torch.zeros(80, dtype=torch.uint8), torch.zeros(1), 10, 8)
    dy = torch.zeros((6, 8))
    with pytest.raises(ValueError):
        zq.embedding_grad(ids, torch.zeros((5, 8)), 10)
    with pytest.raises(ValueError):
        zq.embedding_grad(ids, dy, 10, accumulate=True)
    with pytest.raises(ValueError):
        zq.embedding_grad(ids, dy, 10, out=torch.zeros((9, 8)))
    with pytest.raises(ValueError):
        zq.embedding_grad(ids, dy, -1)
    with pytest.raises(ValueError):
        zq.embedding_grad(ids.repeat(200), dy.repeat(200, 1), 10, out=table, workspace=torch.zeros(10, dtype=torch.uint8))
    with pytest.raises(TypeError):
        zq.embedding_grad(ids, dy, 10, out=table, workspace=torch.zeros(1000))
    with pytest.raises(TypeError):
        zq.grad_table([torch.zeros(5, dtype=torch.int32)])
    with pytest.raises(ValueError):
        zq.grad_table([dy], [None, None])
    with pytest.raises(ValueError):
        zq.grad_table([(torch.zeros(4, dtype=torch.uint8), torch.zeros(1), 9, 32)])
    with pytest.raises(ValueError):
        zq.grad_table([(torch.zeros(40, dtype=torch.uint8), torch.zeros(2), 70, 32)])
    with pytest.raises(TypeError):
        zq.grad_table([dy])                           # not on a GPU
    x = torch.zeros((2, 64), dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        zq.int4_dequant_gemm(x.float(), torch.zeros(64, dtype=torch.uint8), torch.zeros(4), 2, 32)
    with pytest.raises(ValueError):
        zq.int4_dequant_gemm(x, torch.zeros(63, dtype=torch.uint8), torch.zeros(4), 2, 32)
    with pytest.raises(ValueError):
        zq.int4_dequant_gemm(x, torch.zeros(64, dtype=torch.uint8), torch.zeros(3), 2, 32)
    with pytest.raises(ValueError):
        zq.int4_dequant_gemm(x, torch.zeros(64, dtype=torch.uint8), torch.zeros(4), 2, 32, y=torch.zeros(3))
    with pytest.raises(ValueError):
        zq.int4_dequant_gemm(x[0], torch.zeros(64, dtype=torch.uint8), torch.zeros(4), 2, 32)
