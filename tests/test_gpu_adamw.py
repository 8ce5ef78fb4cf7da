"""adamw_step on the GPU: every bit against the definition in binary32 on the host, and
the distance to it in binary64."""
import itertools
import math

import numpy as np
import pytest
import torch

import paper_2501_04266_amd as zq
from tests import plain_adamw as plain
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu
F = np.float32
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
STEP = dict(lr=3e-3, b1=0.9, b2=0.99, eps=1e-8)


def bits_of(t):
    """A tensor's bits on the host."""
    t = t.detach().contiguous()
    return t.view({1: torch.uint8, 2: torch.int16, 4: torch.int32, 8: torch.int64}[t.element_size()]).cpu().numpy()


def guarded(n, dtype, fill=None, offset=0, dev=DEV):
    """A tensor of n elements within a larger one of bytes 0xA5, at an element offset."""
    size = torch.empty(0, dtype=dtype).element_size()
    base = torch.full(((n + offset + 37) * size,), 0xA5, dtype=torch.uint8, device=dev).view(dtype)
    t = base[offset:offset + n]
    if fill is not None:
        t.copy_(fill)
    return t, base


def guards_kept(t, base):
    at = (t.data_ptr() - base.data_ptr()) // base.element_size()
    around = torch.cat([base[:at].reshape(-1).view(torch.uint8), base[at + t.numel():].reshape(-1).view(torch.uint8)])
    return bool((around == 0xA5).all())


class Tensor:
    """One parameter with its gradient, moments and copy, on the GPU and the host."""

    def __init__(self, rng, n, param="f32", grad="bf16", state=32, out=None, block=64, offset=0, spread=1.0, wd=0.1):
        self.n, self.block, self.wd, self.out_kind = n, block, wd, out
        x = torch.from_numpy((rng.standard_normal(n) * 0.02).astype(F))
        self.p, self.p_base = guarded(n, DT[param], x, offset)
        scale = np.exp(rng.uniform(-spread, spread, n)) * 1e-3
        g = torch.from_numpy((rng.standard_normal(n) * scale).astype(F))
        if grad == "int4":
            packed, scales = zq.qgz_quantize(g.to(DEV), block) if n else (torch.empty(0, dtype=torch.uint8, device=DEV), torch.empty(0, device=DEV))
            keep, _ = guarded(packed.numel(), torch.uint8, packed, offset)
            self.grad = (keep, scales, n, block)
            q = keep.cpu().numpy().astype(np.int64)
            codes = np.stack([q & 15, q >> 4], 1).reshape(-1)[:n]
            self.q, self.q_scales = np.where(codes > 7, codes - 16, codes).astype(F), scales.cpu().numpy()
        else:
            self.grad, _ = guarded(n, DT[grad], g, offset)
        m = (rng.standard_normal(n) * scale).astype(F)
        v = (rng.standard_normal(n) * scale).astype(F) ** 2
        self.state = state
        if state == 32:
            self.m, self.m_base = guarded(n, torch.float32, torch.from_numpy(m), offset)
            self.v, self.v_base = guarded(n, torch.float32, torch.from_numpy(v), offset)
            self.entries = self.m, self.v
        else:
            half = np.full(n, 0x8000)
            self.m8, self.v8 = [], []
            for x, signed, dtype, keep in ((m, True, torch.float8_e4m3fn, self.m8), (v, False, torch.float8_e5m2, self.v8)):
                codes, scales = plain.encode8(x, half, block, signed) if n else (np.zeros(0, np.uint8), np.zeros(0, F))
                c, c_base = guarded(n, torch.uint8, torch.from_numpy(codes), offset)
                s, s_base = guarded(len(scales), torch.float32, torch.from_numpy(scales), offset)
                keep += [c.view(dtype), c_base, s, s_base]
            self.entries = (self.m8[0], self.m8[2], block), (self.v8[0], self.v8[2], block)
        self.out = self.out_base = None
        if out == "int8":
            codes, self.out_base = guarded(n, torch.int8, None, offset)
            scales, self.outs_base = guarded(zq.num_scales(n, block), torch.float32, None, offset)
            self.out = (codes, scales, block)
        elif out:
            self.out, self.out_base = guarded(n, DT[out], None, offset)

    def host(self):
        """(p, m, v) as binary32 on the host."""
        p = self.p.float().cpu().numpy()
        if self.state == 32:
            return p, self.m.cpu().numpy(), self.v.cpu().numpy()
        return (p, *[plain.decode8(k[0].view(torch.uint8).cpu().numpy(), k[2].cpu().numpy(), self.block, s)
                     for k, s in ((self.m8, True), (self.v8, False))])

    def gradient(self, c):
        if isinstance(self.grad, tuple):
            return self.q * plain.spread((self.q_scales * c).astype(F), self.block, self.n)
        return self.grad.float().cpu().numpy() * c


def table_of(ts, **more):
    return zq.adamw_table([t.p for t in ts], [t.grad for t in ts], [t.entries[0] for t in ts],
                          [t.entries[1] for t in ts], [t.out for t in ts], weight_decay=[t.wd for t in ts], **more)


def check_step(ts, before, t, lr=STEP["lr"], norm=None, max_norm=None, scale=1.0, lr_scale=1.0, what=""):
    """The tensors after step t from what `before` holds of them."""
    args = (t, lr, STEP["b1"], STEP["b2"], STEP["eps"])
    c = plain.clip_factor(scale, norm, max_norm)
    for k, (x, (p0, m0, v0)) in enumerate(zip(ts, before)):
        g = x.gradient(c).astype(F)
        p, m, v = plain.step32(p0, g, m0, v0, *args, x.wd, lr_scale)
        exact, off = plain.step64(p0, x.gradient(F(1)).astype(np.float64) * float(c), m0, v0, *args, x.wd, lr_scale)
        for name, one, ref, tol in zip("pmv", (p, m, v), exact, off):
            # gradients as INT4 values carry one more rounding (of the scale times c)
            assert (np.abs(one - ref) <= tol * 1.2 + 1e-44).all(), f"{what} tensor {k}: {name} against 64 bits"
        want = torch.from_numpy(p).to(x.p.dtype)
        assert np.array_equal(bits_of(x.p), bits_of(want)), f"{what} tensor {k} ({x.n} elements): weight"
        if x.state == 32:
            assert np.array_equal(bits_of(x.m), bits_of(torch.from_numpy(m))), f"{what} tensor {k}: m"
            assert np.array_equal(bits_of(x.v), bits_of(torch.from_numpy(v))), f"{what} tensor {k}: v"
            assert guards_kept(x.m, x.m_base) and guards_kept(x.v, x.v_base), what
        elif x.n:
            w = plain.drawn(t, k, 0, x.n)
            for keep, y, drawn, signed in ((x.m8, m, w & np.uint64(0xFFFF), True), (x.v8, v, w >> np.uint64(16), False)):
                codes, scales = plain.encode8(y, drawn, x.block, signed)
                assert np.array_equal(bits_of(keep[2]), bits_of(torch.from_numpy(scales))), f"{what} tensor {k}: scales"
                assert np.array_equal(bits_of(keep[0]), codes), f"{what} tensor {k}: codes (signed: {signed})"
                assert guards_kept(keep[0].view(torch.uint8), keep[1]) and guards_kept(keep[2], keep[3]), what
        assert guards_kept(x.p, x.p_base), f"{what} tensor {k}: memory around the weight"
        if x.out_kind == "int8" and x.n:
            codes, scales = zq.qwz_quantize(x.p.clone(), x.block)
            assert np.array_equal(bits_of(x.out[0]), bits_of(codes)), f"{what} tensor {k}: INT8 codes"
            assert np.array_equal(bits_of(x.out[1]), bits_of(scales)), f"{what} tensor {k}: INT8 scales"
            assert guards_kept(x.out[0], x.out_base) and guards_kept(x.out[1], x.outs_base), what
        elif x.out_kind and x.n:
            assert np.array_equal(bits_of(x.out), bits_of(x.p.to(x.out.dtype))), f"{what} tensor {k}: copy"
            assert guards_kept(x.out, x.out_base), what


def step(ts, t, table=None, **more):
    zq.adamw_step(table or table_of(ts), t, STEP["lr"], (STEP["b1"], STEP["b2"]), STEP["eps"], **more)
    torch.cuda.synchronize()


SIZES = [0, 1, 2, 3, 5, 31, 63, 64, 65, 255, 257, 1023, 1024, 1025, 4095, 4096, 4097, 8191, 12291]


@pytest.mark.parametrize("state,out,block", [(32, None, 64), (32, "bf16", 64), (32, "int8", 32), (8, "int8", 128),
                                             (8, None, 1024), (8, "f16", 512), (32, "int8", 1024), (8, "f32", 256)])
@pytest.mark.parametrize("offset", [0, 1, 3])
def test_sizes(state, out, block, offset):
    """Every size at once, at any element address; three steps."""
    rng = np.random.default_rng(block + offset)
    ts = [Tensor(rng, n, grad=g, state=state, out=out, block=block, offset=offset)
          for n, g in zip(SIZES, itertools.cycle(["bf16", "int4", "f32", "f16"]))]
    table = table_of(ts)
    for t in (1, 2, 3):
        before = [x.host() for x in ts]
        step(ts, t, table)
        check_step(ts, before, t, what=f"step {t}")


@pytest.mark.parametrize("param,grad,state", itertools.product(["f32", "f16", "bf16"], ["f32", "f16", "bf16", "int4"], [32, 8]))
def test_types(param, grad, state):
    rng = np.random.default_rng(7)
    for out in (None, "f32", "f16", "bf16", "int8"):
        ts = [Tensor(rng, n, param, grad, state, out) for n in (4096 * 2 + 70, 63)]
        before = [x.host() for x in ts]
        step(ts, 5)
        check_step(ts, before, 5, what=f"{out}")


@pytest.mark.parametrize("norm,max_norm,scale", [(0.25, 1.0, 1.0), (7.5, 1.0, 1.0), (7.5, 1.0, 2.0**-10), (0.0, 0.0, 1.0), (3.0, 0.0, 1.0)])
def test_clipping(norm, max_norm, scale):
    rng = np.random.default_rng(3)
    ts = [Tensor(rng, 5000, grad=g, state=s) for g, s in (("bf16", 32), ("int4", 8), ("f32", 8))]
    before = [x.host() for x in ts]
    step(ts, 2, norm=torch.tensor(norm, device=DEV), max_norm=max_norm, scale=scale)
    check_step(ts, before, 2, norm=norm, max_norm=max_norm, scale=scale)


@pytest.mark.parametrize("norm", [math.inf, -math.inf, math.nan])
def test_norm_not_finite_leaves_everything(norm):
    rng = np.random.default_rng(3)
    ts = [Tensor(rng, 5000, state=s, out=o) for s, o in ((32, "bf16"), (8, "int8"))]
    held = [b.clone() for x in ts for b in (x.p_base, x.out_base)] + [b.clone() for k in (ts[1].m8, ts[1].v8) for b in k]
    m = ts[0].m.clone()
    step(ts, 2, norm=torch.tensor(norm, device=DEV), max_norm=1.0)
    now = [b for x in ts for b in (x.p_base, x.out_base)] + [b for k in (ts[1].m8, ts[1].v8) for b in k]
    assert all(np.array_equal(bits_of(a), bits_of(b)) for a, b in zip(held, now))
    assert np.array_equal(bits_of(m), bits_of(ts[0].m))


def test_as_clipping_and_then_a_step():
    """norm and max_norm give the bits of grad_clip into binary32 and a step from that."""
    rng = np.random.default_rng(11)
    n = 30000
    a, b = (Tensor(np.random.default_rng(2), n, grad="int4", state=8) for _ in range(2))
    grads = zq.grad_table([a.grad], [torch.empty(n, device=DEV)])
    norm = zq.grad_norm(grads)
    step([a], 4, norm=norm, max_norm=0.1)
    clipped = zq.grad_clip(grads, norm, 0.1)[0]
    zq.adamw_step(zq.adamw_table([b.p], [clipped], [b.entries[0]], [b.entries[1]], weight_decay=b.wd), 4, STEP["lr"],
                  (STEP["b1"], STEP["b2"]), STEP["eps"])
    assert np.array_equal(bits_of(a.p), bits_of(b.p))
    assert np.array_equal(bits_of(a.m8[0]), bits_of(b.m8[0])) and np.array_equal(bits_of(a.v8[0]), bits_of(b.v8[0]))
    del rng


def test_fresh_states_and_zero_gradients():
    for bits in (32, 8):
        p = [torch.randn(3000, generator=torch.Generator().manual_seed(1)).to(DEV), torch.randn(70, device=DEV)]
        start = [x.clone() for x in p]
        m, v = zq.adamw_states(p, bits, 64)
        table = zq.adamw_table(p, [torch.zeros_like(x) for x in p], m, v, weight_decay=0.5)
        zq.adamw_step(table, 1, 0.1)
        # 0 / (0 + eps) = 0: only the decay
        decay = F(1.0 - 0.1 * 0.5)
        for x, s in zip(p, start):
            assert np.array_equal(x.cpu().numpy(), s.cpu().numpy() * decay)
        for e in (*m, *v):
            for x in (e if bits == 32 else e[0].view(torch.uint8), e if bits == 32 else e[1]):
                assert not bool(x.any())


def test_lr_scale_per_tensor():
    rng = np.random.default_rng(5)
    ts = [Tensor(rng, 700, state=s) for s in (32, 8)]
    before = [x.host() for x in ts]
    step(ts, 3, table_of(ts, lr_scale=0.125))
    check_step(ts, before, 3, lr_scale=0.125)


def test_wide_blocks_of_uneven_magnitudes():
    """Gradients over many orders of magnitude in a block, and values at the codes' ends."""
    rng = np.random.default_rng(9)
    ts = [Tensor(rng, 9000, grad="f32", state=8, block=b, spread=s) for b, s in ((32, 6.0), (256, 12.0), (1024, 20.0))]
    table = table_of(ts)
    for t in (1, 2):
        before = [x.host() for x in ts]
        step(ts, t, table)
        check_step(ts, before, t)


def test_rounding_keeps_small_changes_on_average():
    """v under a decay of 0.999 with no gradient: nearest rounding to 2 bits would keep it
    for ever; the mean over many elements follows 0.999^t.  Each step moves a value by a
    share p of a code step s <= 1/4 of it with variance p s^2 <= 0.001 s: after 200 steps
    of relative variance 200 * 0.001 / 4 = 0.05 at most, 40,000 elements' mean is within
    5 * sqrt(0.05 / 40000) = 0.0056 of its expectation."""
    n = 40000
    p = [torch.zeros(n, device=DEV)]
    m, v = zq.adamw_states(p, 8, 64)
    rng = np.random.default_rng(1)
    values = (rng.uniform(0.3, 1.0, n)).astype(F)
    codes, scales = plain.encode8(values, np.full(n, 0x8000), 64, False)
    v[0][0].view(torch.uint8).copy_(torch.from_numpy(codes))
    v[0][1].copy_(torch.from_numpy(scales))
    start = plain.decode8(codes, scales, 64, False).astype(np.float64).mean()
    table = zq.adamw_table(p, [torch.zeros(n, device=DEV)], m, v)
    for t in range(1, 201):
        zq.adamw_step(table, t, 0.0, (0.9, 0.999))
    end = plain.decode8(v[0][0].view(torch.uint8).cpu().numpy(), v[0][1].cpu().numpy(), 64, False).astype(np.float64).mean()
    assert abs(end / start / 0.999**200 - 1) < 0.0056 + 1e-3


def test_step_and_rate_on_the_device_in_a_graph():
    """A captured step reads the count and the rate when it runs; replays with eager work
    between them give the eager steps' bits."""
    rng_seed, n = 21, 20000
    a, b = ([Tensor(np.random.default_rng(rng_seed), n, state=s, out=o, grad=g)
             for s, o, g in ((32, "bf16", "bf16"), (8, "int8", "int4"))] for _ in range(2))
    ta, tb = table_of(a), table_of(b)
    count, rate = torch.zeros(1, dtype=torch.int64, device=DEV), torch.zeros(1, device=DEV)
    norm = torch.full((), 0.5, device=DEV)
    more = dict(norm=norm, max_norm=0.25)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        count.add_(1)
        zq.adamw_step(ta, count, rate, (STEP["b1"], STEP["b2"]), STEP["eps"], **more)
    for t, lr in ((1, 1e-3), (2, 5e-4), (3, 2.5e-4), (4, 1e-4)):
        rate.fill_(lr)
        graph.replay()
        zq.adamw_step(tb, t, float(F(lr)), (STEP["b1"], STEP["b2"]), STEP["eps"], **more)
        torch.cuda.synchronize()
        for x, y in zip(a, b):
            assert np.array_equal(bits_of(x.p_base), bits_of(y.p_base)), f"step {t}"
            assert np.array_equal(bits_of(x.out_base), bits_of(y.out_base)), f"step {t}"
        assert np.array_equal(bits_of(a[1].m8[0]), bits_of(b[1].m8[0])), f"step {t}"
        assert np.array_equal(bits_of(a[1].v8[0]), bits_of(b[1].v8[0])), f"step {t}"
    assert int(count) == 4


def test_on_another_stream():
    a, b = ([Tensor(np.random.default_rng(4), 100000, state=8, grad="int4")] for _ in range(2))
    ta, tb = table_of(a), table_of(b)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    zq.adamw_step(ta, 1, 1e-3, stream=side)
    zq.adamw_step(tb, 1, 1e-3)
    torch.cuda.synchronize()
    assert np.array_equal(bits_of(a[0].p), bits_of(b[0].p)) and np.array_equal(bits_of(a[0].m8[0]), bits_of(b[0].m8[0]))


def test_many_small_tensors():
    rng = np.random.default_rng(8)
    ts = [Tensor(rng, int(n), grad=g, state=8 if i % 2 else 32, block=32)
          for i, (n, g) in enumerate(zip(rng.integers(1, 40, 500), itertools.cycle(["f32", "int4"])))]
    before = [x.host() for x in ts]
    step(ts, 9)
    check_step(ts, before, 9)


def test_no_tensors():
    zq.adamw_step(zq.adamw_table([], [], [], []), 1, 1e-3)


def test_elements_beyond_2_32():
    """The end of a tensor of more than 2^32 elements: addresses, and the bits drawn there."""
    n, tail, block = 2**32 + 4096 * 2 + 70, 9000, 256
    first = n - tail
    p = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    grad = torch.zeros((n + 1) // 2, dtype=torch.uint8, device=DEV)
    gs = torch.full((zq.num_scales(n, block),), 1e-3, device=DEV)
    rng = np.random.default_rng(3)
    grad[first // 2:] = torch.from_numpy(rng.integers(0, 256, (n + 1) // 2 - first // 2, dtype=np.uint8)).to(DEV)
    m, v = zq.adamw_states([p], 8, block)
    p[first:] = torch.from_numpy((rng.standard_normal(tail) * 0.02).astype(F)).to(DEV)
    p0 = p[first:].float().cpu().numpy()
    q = grad[first // 2:].cpu().numpy().astype(np.int64)
    q = np.stack([q & 15, q >> 4], 1).reshape(-1)[first % 2:][:tail]
    g = np.where(q > 7, q - 16, q).astype(F) * F(1e-3)
    zq.adamw_step(zq.adamw_table([p], [(grad, gs, n, block)], m, v), 6, STEP["lr"], (STEP["b1"], STEP["b2"]), STEP["eps"])
    zero = np.zeros(tail, F)
    want, m1, v1 = plain.step32(p0, g, zero, zero, 6, STEP["lr"], STEP["b1"], STEP["b2"], STEP["eps"], 0.0)
    assert np.array_equal(bits_of(p[first:]), bits_of(torch.from_numpy(want).bfloat16()))
    at = first + -first % block  # whole blocks from here on, all beyond 2^32
    assert at > 2**32 - 4096 and n - at > 2 * 4096
    at = max(at, 2**32)
    k = at - first
    w = plain.drawn(6, 0, at, n - at)
    for keep, y, drawn, signed in ((m[0], m1, w & np.uint64(0xFFFF), True), (v[0], v1, w >> np.uint64(16), False)):
        codes, scales = plain.encode8(y[k:], drawn, block, signed)
        assert np.array_equal(bits_of(keep[0].view(torch.uint8)[at:]), codes)
        assert np.array_equal(bits_of(keep[1][at // block:]), bits_of(torch.from_numpy(scales)))
    assert not bool(p[:first].any())


def test_step_or_rate_alone_on_the_device():
    count, rate = torch.full((1,), 4, dtype=torch.int64, device=DEV), torch.full((1,), 1e-3, device=DEV)
    lr = float(rate)
    for step_arg, lr_arg in ((4, lr), (count, lr), (4, rate), (count, rate)):
        ts = [Tensor(np.random.default_rng(6), n, state=s) for n, s in ((3000, 32), (700, 8))]
        before = [x.host() for x in ts]
        zq.adamw_step(table_of(ts), step_arg, lr_arg, (STEP["b1"], STEP["b2"]), STEP["eps"])
        check_step(ts, before, 4, lr=lr)


def test_one_gradient_for_two_weights():
    """A gradient is only read, so two weights may share it."""
    a, b = (Tensor(np.random.default_rng(s), 5000, state=32) for s in (1, 2))
    b.grad = a.grad
    before = [a.host(), b.host()]
    step([a, b], 2)
    check_step([a, b], before, 2)
