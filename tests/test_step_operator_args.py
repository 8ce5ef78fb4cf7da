"""The optimizer's step, the RMS norm and the policy loss refuse what they do not take
(CPU; no kernel is launched): the C calls with made-up addresses, which nothing
dereferences, and the binding with tensors of the wrong kind."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

import paper_2501_04266_amd as zq
from paper_2501_04266_amd import _lib

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
vp = ctypes.c_void_p
NULL, BLOCK, DTYPE, ALIGN, SIZE, ALIAS = -1, -2, -3, -4, -5, -8
F32, F16, BF16, I32, I64, INT4, INT8, F8 = range(8)
A, B, C, D, E, G, H, W = (k << 44 for k in range(1, 9))


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2501_04266_amd import build
        build.build()
    return _lib.lib()


def test_layouts_of_the_binding(tmp_path):
    exe = str(tmp_path / "layouts")
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"),
                    os.path.join(HERE, "c", "more_layouts.c"), "-o", exe], check=True)
    said = subprocess.run([exe], capture_output=True, text=True, check=True).stdout.splitlines()
    header = {f[0]: tuple(int(v) for v in f[1:]) for f in (line.split() for line in said)}
    mirror = {name: (getattr(_lib, name),) for name in ("ZQ_INT8", "ZQ_F8")}
    for name, cls in (("zq_adamw", _lib._AdamW), ("zq_adamw_plan", _lib._AdamWPlan), ("zq_adamw_args", _lib._AdamWArgs),
                      ("zq_policy", _lib._Policy)):
        mirror[name] = (ctypes.sizeof(cls),)
        for field, _ in cls._fields_:
            d = getattr(cls, field)
            mirror[f"{name}.{field}"] = (d.offset, d.size)
    assert mirror == header


# ---------------------------------------------------------------- the optimizer's step

def tensor(**other):
    e = dict(param=A, grad=B, m=C, v=D, n=1000, weight_decay=0.1, lr_scale=1.0, param_dtype=F32, grad_dtype=BF16,
             state_dtype=F32)
    e.update(other)
    return _lib._AdamW(**e)


def made(L, *entries, count=None):
    plan = _lib._AdamWPlan()
    array = (_lib._AdamW * max(1, len(entries)))(*entries)
    return L.zq_adamw_plan_make(array, len(entries) if count is None else count, ctypes.byref(plan)), plan


INT4_GRAD = dict(grad_dtype=INT4, grad_scales=E, grad_block=128)
STATE8 = dict(state_dtype=F8, m_scales=G, v_scales=H, state_block=256)
OUT8 = dict(out=W, out_dtype=INT8, out_scales=W + (1 << 40), out_block=64)


@pytest.mark.parametrize("other,status", [
    ({}, 0), (INT4_GRAD, 0), (STATE8, 0), (OUT8, 0), (dict(out=W, out_dtype=F16), 0),
    (dict(n=-1), SIZE), (dict(n=1 << 62), SIZE), (dict(weight_decay=math.nan), SIZE), (dict(lr_scale=math.inf), SIZE),
    (dict(param_dtype=3), DTYPE), (dict(grad_dtype=INT8), DTYPE), (dict(state_dtype=BF16), DTYPE),
    (dict(out=W, out_dtype=INT4), DTYPE),
    ({**INT4_GRAD, "grad_block": 48}, BLOCK), ({**STATE8, "state_block": 16}, BLOCK), ({**OUT8, "out_block": 0}, BLOCK),
    (dict(param=None), NULL), (dict(grad=None), NULL), (dict(m=None), NULL), (dict(v=None), NULL),
    ({**INT4_GRAD, "grad_scales": None}, NULL), ({**STATE8, "m_scales": None}, NULL), ({**STATE8, "v_scales": None}, NULL),
    ({**OUT8, "out_scales": None}, NULL),
    (dict(param=A + 2), ALIGN), (dict(grad=B + 1), ALIGN), (dict(m=C + 2), ALIGN), (dict(v=D + 1), ALIGN),
    ({**INT4_GRAD, "grad": B + 1}, 0), ({**INT4_GRAD, "grad_scales": E + 2}, ALIGN),
    ({**STATE8, "m": C + 1, "v": D + 3}, 0), ({**STATE8, "v_scales": H + 1}, ALIGN),
    ({**OUT8, "out": W + 1}, 0), ({**OUT8, "out_scales": W + (1 << 40) + 2}, ALIGN), (dict(out=W + 1, out_dtype=BF16), ALIGN),
    # 1,000 elements: 4,000 bytes of param, m and v, 2,000 of the gradient
    (dict(param=B + 1996), ALIAS), (dict(param=B + 2000), 0), (dict(m=A + 3996), ALIAS), (dict(v=C), ALIAS),
    (dict(out=A, out_dtype=F32), ALIAS), (dict(out=B, out_dtype=BF16), ALIAS),
    ({**STATE8, "m_scales": G, "v_scales": G + 12}, ALIAS), ({**STATE8, "v_scales": G + 16}, 0),
    ({**INT4_GRAD, "grad": A + 3900}, ALIAS), ({**INT4_GRAD, "grad_scales": C + 4}, ALIAS),
    ({**OUT8, "out_scales": D}, ALIAS),
    (dict(n=0, param=None, grad=None, m=None, v=None), 0),
])
def test_tensors(L, other, status):
    assert made(L, tensor(**other))[0] == status


def test_tables(L):
    rc, plan = made(L, tensor(), tensor(param=A + 4000, grad=B, m=C + 4000, v=D + 4000, n=9000))
    assert rc == 0 and plan.count == 2 and plan.pieces == 1 + 9 and plan.block_pieces == 0  # of 1,024; a gradient may be read twice
    assert plan.bytes == 64 + 2 * 112 + 4 * 10
    rc, plan = made(L, tensor(), tensor(param=A + 4000, grad=B, m=C + 4000, v=D + 4000, n=9000, **STATE8))
    assert rc == 0 and plan.pieces == 1 and plan.block_pieces == 3 and plan.bytes == 64 + 2 * 112 + 4 * 4  # of 4,096
    assert made(L, tensor(), tensor())[0] == ALIAS  # a parameter twice
    assert made(L, count=-1)[0] == SIZE and made(L)[0] == 0
    assert L.zq_adamw_plan_make(None, 1, ctypes.byref(plan)) == NULL and L.zq_adamw_plan_make(None, 0, None) == NULL
    # 2^31 pieces and more
    assert made(L, tensor(n=1 << 43, m=1 << 50, v=1 << 51, param=1 << 52, grad=1 << 53))[0] == SIZE
    assert L.zq_adamw_plan_table(None, None, None) == NULL


@pytest.mark.parametrize("args,more,status", [
    (dict(step=0), {}, SIZE), (dict(step=-3), {}, SIZE), (dict(beta1=1.0), {}, SIZE), (dict(beta1=-0.1), {}, SIZE),
    (dict(beta2=1.5), {}, SIZE), (dict(beta2=math.nan), {}, SIZE), (dict(eps=-1e-8), {}, SIZE),
    (dict(lr=math.inf), {}, SIZE), (dict(lr=math.nan), {}, SIZE),
    (dict(max_norm=-1.0), dict(norm=B), SIZE), (dict(max_norm=math.nan), dict(norm=B), SIZE),
    ({}, dict(table=A + 8), ALIGN), ({}, dict(step=B + 4), ALIGN), ({}, dict(lr=B + 2), ALIGN), ({}, dict(norm=B + 1), ALIGN),
    ({}, dict(table=None), NULL),
    # nothing to do: checked all the same
    ({}, {}, 0), (dict(max_norm=-1.0), {}, 0), (dict(step=0), dict(step=B), 0), (dict(lr=math.nan), dict(lr=B), 0),
])
def test_numbers_of_a_step(L, args, more, status):
    a = _lib._AdamWArgs(**{**dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, max_norm=1.0, scale=1.0), **args})
    at = {**dict(table=A, step=None, lr=None, norm=None), **more}
    empty = _lib._AdamWPlan(64, 0, 0, 0, 0)
    assert L.zq_adamw_step(ctypes.byref(empty), vp(at["table"]), ctypes.byref(a), vp(at["step"]), vp(at["lr"]),
                           vp(at["norm"]), None) == status
    assert L.zq_adamw_step(None, vp(A), ctypes.byref(a), None, None, None, None) == NULL
    assert L.zq_adamw_step(ctypes.byref(empty), vp(A), None, None, None, None, None) == NULL


def test_binding_of_the_step():
    p, s = [torch.zeros(100)], [torch.zeros(100)]
    with pytest.raises(TypeError, match="GPU"):
        zq.adamw_table(p, s, s, s)
    with pytest.raises(ValueError, match="grads"):
        zq.adamw_table(p, [], s, s)
    with pytest.raises(ValueError, match="outs"):
        zq.adamw_table(p, s, s, s, [])
    with pytest.raises(ValueError, match="weight_decay"):
        zq.adamw_table(p, s, s, s, weight_decay=[0.1, 0.2])
    with pytest.raises(TypeError, match="dtype"):
        zq.adamw_table([torch.zeros(100, dtype=torch.int32)], s, s, s)
    with pytest.raises(TypeError, match="AdamWTable"):
        zq.adamw_step(p, 1, 0.1)
    with pytest.raises(ValueError, match="bits"):
        zq.adamw_states(p, 16)
    table = zq.AdamWTable([p, s, s, s, [None]], _lib._AdamWPlan(), torch.zeros(64, dtype=torch.uint8))
    with pytest.raises(ValueError, match="max_norm"):
        zq.adamw_step(table, 1, 0.1, norm=torch.zeros(()))
    with pytest.raises(TypeError, match="step"):
        zq.adamw_step(table, torch.zeros(1), 0.1)
    with pytest.raises(TypeError, match="lr"):
        zq.adamw_step(table, 1, torch.zeros(1, dtype=torch.float64))
    with pytest.raises(TypeError, match="GPU"):
        zq.adamw_step(table, 1, torch.zeros(1))
    m, v = zq.adamw_states(p, 8, 32)
    assert m[0][0].dtype == torch.float8_e4m3fn and v[0][0].dtype == torch.float8_e5m2 and m[0][1].shape == (4,)


@pytest.mark.parametrize("change", ["short grad", "long grad", "int4 count", "moments unlike", "blocks unlike", "state type",
                                    "short scales", "short out"])
def test_binding_of_a_tensor(monkeypatch, change):
    """Sizes and types are checked before anything else is done."""
    monkeypatch.setattr(_lib, "_dev", lambda t, name: 16)
    n = 100
    g, m, v, o = torch.zeros(n), torch.zeros(n), torch.zeros(n), None
    m8 = (torch.zeros(n, dtype=torch.uint8).view(torch.float8_e4m3fn), torch.zeros(2), 64)
    v8 = (torch.zeros(n, dtype=torch.uint8).view(torch.float8_e5m2), torch.zeros(2), 64)
    if change == "short grad":
        g = torch.zeros(99)
    elif change == "long grad":
        g = torch.zeros(101)
    elif change == "int4 count":
        g = (torch.zeros(50, dtype=torch.uint8), torch.zeros(1), 99, 128)
    elif change == "moments unlike":
        m = m8
    elif change == "blocks unlike":
        m, v = m8, (v8[0], torch.zeros(4), 32)
    elif change == "state type":
        m, v = m8, (m8[0], v8[1], 64)
    elif change == "short scales":
        m, v = (m8[0], torch.zeros(1), 64), v8
    else:
        o = (torch.zeros(99, dtype=torch.int8), torch.zeros(2), 64)
    with pytest.raises((ValueError, TypeError)):
        zq.adamw_table([torch.zeros(n)], [g], [m], [v], [o])


# ---------------------------------------------------------------- RMS norm

def norm(L, int8=False, **other):
    a = dict(x=A, residual=B, xt=BF16, weight=C, wt=F32, T=10, D=64, eps=1e-6, h=D, y=E, yt=BF16, scales=G, block=32, rstd=H)
    a.update(other)
    head = [vp(a["x"]), vp(a["residual"]), a["xt"], vp(a["weight"]), a["wt"], a["T"], a["D"], a["eps"], vp(a["h"]), vp(a["y"])]
    if int8:
        return L.qwz_rms_norm(*head, vp(a["scales"]), a["block"], vp(a["rstd"]), None)
    return L.zq_rms_norm(*head, a["yt"], vp(a["rstd"]), None)


@pytest.mark.parametrize("other,status", [
    (dict(T=0), 0), (dict(T=0, x=None, y=None), 0), (dict(T=-1), SIZE), (dict(D=0), SIZE), (dict(D=(1 << 24) + 64), SIZE),
    (dict(T=1 << 31), SIZE), (dict(eps=-1.0), SIZE), (dict(eps=math.nan), SIZE), (dict(xt=3), DTYPE), (dict(wt=-1), DTYPE),
    (dict(x=None), NULL), (dict(y=None), NULL), (dict(h=None), NULL),
    (dict(x=A + 1), ALIGN), (dict(residual=B + 1), ALIGN), (dict(weight=C + 2), ALIGN), (dict(h=D + 1), ALIGN), (dict(rstd=H + 2), ALIGN),
    # 1,280 bytes of x, residual and h, 256 of weight, 40 of rstd
    (dict(y=A + 1278), ALIAS), (dict(y=B), ALIAS), (dict(y=C + 252), ALIAS), (dict(y=D), ALIAS), (dict(rstd=A), ALIAS),
    (dict(rstd=E), ALIAS), (dict(h=A + 2), ALIAS), (dict(h=B - 2), ALIAS), (dict(h=C), ALIAS), (dict(h=E), ALIAS),
])
@pytest.mark.parametrize("int8", [False, True])
def test_norm(L, other, status, int8):
    assert norm(L, int8, **other) == status


def test_norm_of_either_kind(L):
    assert norm(L, yt=INT8) == DTYPE and norm(L, y=E + 1) == ALIGN
    assert norm(L, True, block=48) == BLOCK and norm(L, True, D=80) == SIZE and norm(L, True, scales=None) == NULL
    assert norm(L, True, scales=G + 2) == ALIGN and norm(L, True, scales=E + 600) == ALIAS and norm(L, True, scales=A) == ALIAS
    assert norm(L, True, T=0, y=None, scales=None) == 0


def grad(L, **other):
    a = dict(dy=A, gt=BF16, h=B, xt=BF16, weight=C, wt=F32, rstd=D, dh=E, T=10, D=64, dx=G, accumulate=0, dw=H, dwt=F32, ws=W)
    a.update(other)
    a.setdefault("bytes", max(0, L.zq_rms_norm_grad_bytes(a["T"], a["D"])))
    return L.zq_rms_norm_grad(vp(a["dy"]), a["gt"], vp(a["h"]), a["xt"], vp(a["weight"]), a["wt"], vp(a["rstd"]), vp(a["dh"]),
                              a["T"], a["D"], vp(a["dx"]), a["accumulate"], vp(a["dw"]), a["dwt"], vp(a["ws"]), a["bytes"], None)


@pytest.mark.parametrize("other,status", [
    (dict(gt=3), DTYPE), (dict(xt=7), DTYPE), (dict(wt=4), DTYPE), (dict(dwt=5), DTYPE),
    (dict(T=-1), SIZE), (dict(D=0), SIZE), (dict(D=(1 << 24) + 1), SIZE), (dict(bytes=100), SIZE),
    (dict(dy=None), NULL), (dict(h=None), NULL), (dict(rstd=None), NULL), (dict(dx=None), NULL), (dict(ws=None), NULL),
    (dict(dy=A + 1), ALIGN), (dict(h=B + 1), ALIGN), (dict(weight=C + 1), ALIGN), (dict(rstd=D + 1), ALIGN),
    (dict(dh=E + 1), ALIGN), (dict(dx=G + 1), ALIGN), (dict(dw=H + 2), ALIGN), (dict(ws=W + 8), ALIGN),
    (dict(dx=A), ALIAS), (dict(dx=B + 1278), ALIAS), (dict(dx=E + 2), ALIAS), (dict(dw=C), ALIAS), (dict(dw=G), ALIAS),
    (dict(ws=A), ALIAS), (dict(ws=G), ALIAS), (dict(dx=D), ALIAS),
    (dict(T=0, dw=None), 0), (dict(T=0, accumulate=1), 0),
])
def test_norm_gradient(L, other, status):
    assert grad(L, **other) == status


def test_norm_gradient_bytes(L):
    f = L.zq_rms_norm_grad_bytes
    assert f(-1, 64) == f(4, 0) == f(4, (1 << 24) + 1) == f(1 << 31, 64) == -1
    for T in (0, 1, 5, 511, 4000, 1 << 20):
        for d in (1, 64, 512, 513, 6144, 8193, 16385, 1 << 24):
            assert 4 * d <= f(T, d) <= max(4 * d, 1 << 24) and f(T, d) % (4 * d) == 0 and f(T, d) // (4 * d) <= max(1, T)
    with pytest.raises(ValueError):
        zq.rms_norm_grad_bytes(-1, 4)


class OnGpu(torch.Tensor):
    is_cuda = True


def gpu(t):
    return t.as_subclass(OnGpu)


def test_norm_of_host_tensors():
    x, w, r = torch.zeros(4, 64), torch.ones(64), torch.zeros(4)
    for call in (lambda: zq.rms_norm(x, w), lambda: zq.qwz_rms_norm(x, w, block=32), lambda: zq.rms_norm_grad(x, x, w, r)):
        with pytest.raises(TypeError, match="GPU"):
            call()


def test_binding_of_the_norm(monkeypatch):
    monkeypatch.setattr(_lib, "_here", lambda **t: None)
    monkeypatch.setattr(_lib, "_stream", lambda s: None)
    x, w = gpu(torch.zeros(4, 64)), gpu(torch.ones(64))
    for call in (lambda **k: zq.rms_norm(x, w, **k), lambda **k: zq.qwz_rms_norm(x, w, block=32, **k)):
        with pytest.raises(ValueError, match="residual"):
            call(hidden=x)
        with pytest.raises(TypeError, match="dtype"):
            call(residual=x.half())
        with pytest.raises(ValueError, match="shape"):
            call(residual=gpu(torch.zeros(64, 4)))
        with pytest.raises(ValueError, match="rstd"):
            call(rstd=gpu(torch.zeros(3)))
    with pytest.raises(TypeError, match="out_dtype"):
        zq.rms_norm(x, w, out_dtype=torch.float64, rstd=gpu(torch.zeros(4)))
    with pytest.raises(ValueError, match="weight"):
        zq.rms_norm(x, gpu(torch.ones(65)))
    with pytest.raises(ValueError, match="shape"):
        zq.rms_norm(gpu(torch.zeros(())), None)
    with pytest.raises(ValueError, match="contiguous"):
        zq.rms_norm(gpu(torch.zeros(64, 4)).t(), w)
    with pytest.raises(ValueError, match="dy"):
        zq.rms_norm_grad(x, gpu(torch.zeros(5, 64)), w, gpu(torch.zeros(5)))
    with pytest.raises(ValueError, match="rstd"):
        zq.rms_norm_grad(x, x, w, gpu(torch.zeros(3)))
    with pytest.raises(ValueError, match="dweight"):
        zq.rms_norm_grad(x, x, w, gpu(torch.zeros(4)), out=gpu(torch.zeros(4, 64)), dweight=gpu(torch.zeros(65)))
    with pytest.raises(ValueError, match="accumulate"):
        zq.rms_norm_grad(x, x, w, gpu(torch.zeros(4)), out=gpu(torch.zeros(4, 64)), accumulate=True)
    with pytest.raises(ValueError, match="workspace"):
        zq.rms_norm_grad(x, x, w, gpu(torch.zeros(4)), out=gpu(torch.zeros(4, 64)), dweight=gpu(torch.zeros(64)),
                         workspace=gpu(torch.zeros(8, dtype=torch.uint8)))


# ---------------------------------------------------------------- the loss

def loss(L, policy=None, **other):
    a = dict(logits=A, lt=BF16, T=10, V=100, ld=104, ids=B, it=I64, sums=C, logp=D, grad=E, gt=BF16, ldg=104, ws=W, bytes=320)
    a.update(other)
    p = dict(old_logp=G, advantages=G + 4096, weights=G + 8192, ref_logp=H, clip_low=0.2, clip_high=0.2, kl=0.1, scale=1.0,
             grad_scale=1.0)
    p.update(policy or {})
    return L.zq_policy_loss(vp(a["logits"]), a["lt"], a["T"], a["V"], a["ld"], vp(a["ids"]), a["it"],
                            ctypes.byref(_lib._Policy(**p)), vp(a["sums"]), vp(a["logp"]), vp(a["grad"]), a["gt"], a["ldg"],
                            vp(a["ws"]), a["bytes"], None)


@pytest.mark.parametrize("other,policy,status", [
    (dict(lt=3), {}, DTYPE), (dict(it=0), {}, DTYPE), (dict(gt=INT8), {}, DTYPE),
    (dict(T=-1), {}, SIZE), (dict(T=(1 << 30) + 1), {}, SIZE), (dict(V=0), {}, SIZE), (dict(V=(1 << 24) + 1, ld=1 << 25), {}, SIZE),
    (dict(ld=99), {}, SIZE), (dict(ldg=99), {}, SIZE), (dict(ld=(1 << 59) // 10 + 1), {}, SIZE), (dict(ldg=(1 << 59) // 10 + 1), {}, SIZE), (dict(bytes=319), {}, SIZE),
    ({}, dict(scale=0.0), SIZE), ({}, dict(scale=-1.0), SIZE), ({}, dict(scale=math.inf), SIZE), ({}, dict(scale=math.nan), SIZE),
    ({}, dict(clip_low=-0.1), SIZE), ({}, dict(clip_low=1.1), SIZE), ({}, dict(clip_high=-0.1), SIZE), ({}, dict(clip_high=math.nan), SIZE),
    ({}, dict(kl=-1.0), SIZE), ({}, dict(kl=math.inf), SIZE), ({}, dict(grad_scale=math.nan), SIZE),
    (dict(logits=None), {}, NULL), (dict(ids=None), {}, NULL), (dict(sums=None), {}, NULL), (dict(ws=None), {}, NULL),
    ({}, dict(old_logp=None), NULL), ({}, dict(advantages=None), NULL), ({}, dict(ref_logp=None), NULL),
    (dict(logits=A + 1), {}, ALIGN), (dict(ids=B + 4), {}, ALIGN), (dict(sums=C + 2), {}, ALIGN), (dict(logp=D + 1), {}, ALIGN),
    (dict(grad=E + 1), {}, ALIGN), (dict(ws=W + 8), {}, ALIGN), ({}, dict(weights=G + 8193), ALIGN),
    # rows of 100 elements 104 apart: 9 * 208 + 200 bytes
    (dict(grad=A + 2070), {}, ALIAS), (dict(grad=A, ldg=128), {}, ALIAS), (dict(grad=A, gt=F16), {}, ALIAS), (dict(grad=A + 2), {}, ALIAS),
    (dict(logp=B), {}, ALIAS), (dict(sums=D), {}, ALIAS), (dict(ws=E), {}, ALIAS), (dict(sums=G + 32), {}, ALIAS), (dict(logp=H), {}, ALIAS),
])
def test_loss(L, other, policy, status):
    assert loss(L, policy, **other) == status


def test_loss_bytes_and_null_policy(L):
    assert L.zq_policy_loss_bytes(-1) == L.zq_policy_loss_bytes((1 << 30) + 1) == -1 and L.zq_policy_loss_bytes(7) == 224
    assert L.zq_policy_loss(vp(A), 2, 1, 4, 4, vp(B), 4, None, vp(C), None, None, 0, 0, vp(W), 32, None) == NULL
    with pytest.raises(ValueError):
        zq.policy_loss_bytes(-1)


@pytest.mark.parametrize("a,status", [
    ((A, 2, 0, 100, 100, B, 4, 1.0, D), 0), ((A, 5, 4, 100, 100, B, 4, 1.0, D), DTYPE), ((A, 2, 4, 100, 100, B, 2, 1.0, D), DTYPE),
    ((A, 2, -4, 100, 100, B, 4, 1.0, D), SIZE), ((A, 2, 4, 100, 98, B, 4, 1.0, D), SIZE), ((A, 2, 4, 100, 100, B, 4, 0.0, D), SIZE),
    ((None, 2, 4, 100, 100, B, 4, 1.0, D), NULL), ((A, 2, 4, 100, 100, None, 4, 1.0, D), NULL), ((A, 2, 4, 100, 100, B, 4, 1.0, None), NULL),
    ((A + 1, 2, 4, 100, 100, B, 4, 1.0, D), ALIGN), ((A, 2, 4, 100, 100, B + 2, 3, 1.0, D), ALIGN), ((A, 2, 4, 100, 100, B, 4, 1.0, D + 2), ALIGN),
    ((A, 2, 4, 100, 100, B, 4, 1.0, A + 796), ALIAS), ((A, 2, 4, 100, 100, B, 4, 1.0, B + 28), ALIAS),
])
def test_token_logp(L, a, status):
    assert L.zq_token_logp(vp(a[0]), *a[1:5], vp(a[5]), *a[6:8], vp(a[8]), None) == status


def test_binding_of_the_loss():
    z, ids, row = torch.zeros(4, 9), torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    with pytest.raises(TypeError, match="GPU"):
        zq.token_logp(z, ids)
    with pytest.raises(TypeError, match="dtype"):
        zq.token_logp(z.double(), ids)
    with pytest.raises(ValueError, match="shape"):
        zq.token_logp(torch.zeros(()), ids)
    with pytest.raises(TypeError, match="GPU"):
        zq.policy_loss(z, ids, row, row)


def test_binding_of_rows(monkeypatch):
    """Rows, ids and per-token values have to agree in number, logits in their layout."""
    z, ids, row = gpu(torch.zeros(4, 9)), gpu(torch.zeros(4, dtype=torch.int64)), gpu(torch.zeros(4))
    monkeypatch.setattr(_lib, "_here", lambda **t: None)
    monkeypatch.setattr(_lib, "_stream", lambda s: None)
    for bad in (gpu(torch.zeros(9, 4)).t(), gpu(torch.zeros(4, 18))[:, ::2], gpu(torch.zeros(1, 9)).expand(4, 9)):
        with pytest.raises(ValueError, match="contiguous"):
            zq.token_logp(bad, ids)
    with pytest.raises(ValueError, match="ids"):
        zq.token_logp(z, gpu(torch.zeros(5, dtype=torch.int64)))
    with pytest.raises(TypeError, match="ids"):
        zq.token_logp(z, row)
    for k in range(2):
        args = [row, row]
        args[k] = gpu(torch.zeros(5))
        with pytest.raises(ValueError, match="needed"):
            zq.policy_loss(z, ids, *args)
    with pytest.raises(ValueError, match="weights"):
        zq.policy_loss(z, ids, row, row, gpu(torch.zeros(3)))
    with pytest.raises(TypeError, match="ref_logp"):
        zq.policy_loss(z, ids, row, row, None, row.double(), kl=0.1)
    with pytest.raises(TypeError, match="grad_dtype"):
        zq.policy_loss(z, ids, row, row, grad_dtype=torch.int8)
    with pytest.raises(ValueError, match="grad"):
        zq.policy_loss(z, ids, row, row, grad=gpu(torch.zeros(4, 8)))
    with pytest.raises(ValueError, match="grad"):
        zq.policy_loss(z, ids, row, row, grad=gpu(torch.zeros(3, 9)))


def test_another_device_is_refused(monkeypatch):
    class Elsewhere(torch.Tensor):
        def get_device(self):
            return 1

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    with pytest.raises(ValueError, match="current device"):
        _lib._here(x=torch.zeros(1).as_subclass(Elsewhere))
