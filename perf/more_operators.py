"""Timed workloads of the rest of a rank's training step: the optimizer's update, the
norm between layers with its gradient, and the loss at the output head.

A case's "op" says which operator it makes a pass through:

  adamw      one AdamW step over many tensors: gradients dense or as the INT4 shards
             that a reduce level leaves, clipped by a norm that is on the GPU; moments in
             32 or 8 bits; beside the weight in place, a copy of it in 16 bits or in the
             INT8 format that is gathered next
  rms        root-mean-square norm of rows after the residual's addition, its output
             dense or in the INT8 format
  rms_grad   its gradient: the rows', the weight's
  logp       log-probabilities of chosen tokens from logits
  policy     the clipped policy loss with a KL term from logits, and the logits' gradient

Sizes are those of the package's own workloads where it has them (hidden 2048 and 6144,
one layer 12 h^2 elements, gradient shards of 1/8, a vocabulary of 50,000); token counts
are generic.  8-bit moments are float8 codes with a binary32 scale a block and are
returned as that; an INT8 output is returned dequantised.  `draw` spreads over the same
ranges.
"""
import math
import random

import torch

# run() in plain torch, or through the package's calls
own = False

DEV = "cuda"
_DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "f16": 2, "bf16": 2}
H_13B, H_20B, VOCAB = 2048, 6144, 50000
SHARD_20B = 12 * H_20B * H_20B // 8
LR, BETA1, BETA2, EPS, DECAY = 3e-4, 0.9, 0.95, 1e-8, 0.1


def listed():
    return [
        # one layer of a small model, tensor by tensor: the latency of a step
        {"name": "adamw-small", "op": "adamw", "tensors": "layers", "count": 1, "h": 256, "param": "f32", "state": 32,
         "out": "bf16", "clip": True},
        # an unsharded model of 24 layers in mixed precision, clipped
        {"name": "adamw-model", "op": "adamw", "tensors": "layers", "count": 24, "h": H_13B, "param": "f32", "state": 32,
         "out": "bf16", "clip": True},
        # a rank's shards of 8 layers: INT4 gradients, 8-bit moments, the INT8 weight that is gathered next
        {"name": "adamw-shards", "op": "adamw", "tensors": "shards", "count": 8, "n": SHARD_20B, "block": 128,
         "param": "f32", "state": 8, "state_block": 256, "out": "int8", "out_block": 256, "clip": True},
        # tensors of any size and gradient type, weights in 16 bits alone, 8-bit moments in small blocks
        {"name": "adamw-ragged", "op": "adamw", "tensors": "mixed", "count": 150, "n": 3000000, "sizes": 5, "block": 64,
         "param": "bf16", "state": 8, "state_block": 64, "out": "", "clip": False},
        # generation: one token's row
        {"name": "rms-token", "op": "rms", "T": 1, "D": H_20B, "dtype": "bf16", "weight": "bf16", "residual": True,
         "out": "bf16", "block": 0},
        # a training micro-batch of 8 x 2048 tokens
        {"name": "rms-batch", "op": "rms", "T": 16384, "D": H_20B, "dtype": "bf16", "weight": "f32", "residual": True,
         "out": "bf16", "block": 0},
        # a smaller model's, the output in the INT8 format
        {"name": "rms-int8", "op": "rms", "T": 8192, "D": H_13B, "dtype": "bf16", "weight": "f32", "residual": True,
         "out": "int8", "block": 128},
        # the micro-batch's gradient, the residual stream's own gradient added
        {"name": "rms-grad", "op": "rms_grad", "T": 16384, "D": H_20B, "dtype": "bf16", "weight": "f32", "residual": True},
        # odd sizes everywhere, no residual
        {"name": "rms-grad-ragged", "op": "rms_grad", "T": 5003, "D": 2051, "dtype": "f16", "weight": "f32",
         "residual": False},
        # generation: the log-probabilities of 8 sequences' sampled tokens, logits as the output head writes them
        {"name": "logp-few", "op": "logp", "T": 8, "V": VOCAB, "logits": "f32", "scale": 1.0, "pad": 0.0},
        # a training micro-batch's loss and gradient
        {"name": "policy-batch", "op": "policy", "T": 8192, "V": VOCAB, "logits": "bf16", "grad": "bf16", "scale": 1.0,
         "kl": 0.05, "pad": 0.1},
        # a vocabulary that no tile divides, sampled at a temperature, binary32 logits
        {"name": "policy-ragged", "op": "policy", "T": 3001, "V": 16411, "logits": "f32", "grad": "f32", "scale": 1.25,
         "kl": 0.0, "pad": 0.0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A row length: a multiple of 64 mostly, sometimes of 8, sometimes any number."""
    step = rng.choice([128, 128, 128, 8, 1])
    n = _log(rng, lo, hi)
    return max(lo, n // step * step + (64 if step == 128 and n < 6000 else 0))


def draw(rng):
    op = rng.choice(["adamw", "adamw", "rms", "rms_grad", "logp", "policy"])
    if op == "adamw":
        tensors = rng.choice(["layers", "shards", "mixed"])
        case = {"op": op, "tensors": tensors, "param": rng.choice(["f32", "f32", "bf16", "f16"]),
                "state": rng.choice([32, 8]), "out": rng.choice(["", "bf16", "f16", "int8"]), "clip": rng.random() < 0.7}
        most = 4 * 12 * H_13B * H_13B
        if tensors == "layers":
            case["h"] = rng.choice([256, 512, 1024, 1536, 2048])
            case["count"] = _log(rng, 1, min(24, most // (12 * case["h"] ** 2)))
        else:
            case["count"] = _log(rng, 1, 8) if tensors == "shards" else _log(rng, 1, 150)
            case["n"] = _log(rng, 1000, most // case["count"])
            case["block"] = rng.choice([64, 128, 256])
            case["sizes"] = rng.randrange(1 << 30)
        if case["state"] == 8:
            case["state_block"] = rng.choice([32, 64, 128, 256, 512])
        if case["out"] == "int8":
            case["out_block"] = rng.choice([64, 128, 256, 1024])
        return case
    if op == "rms":
        int8 = rng.random() < 0.4
        block = rng.choice([32, 64, 128]) if int8 else 0
        D = _log(rng, 1, 8192 // block) * block if int8 else _width(rng, 16, 16384)
        return {"op": op, "T": _log(rng, 1, min(65536, 16384 * H_20B // D)), "D": D,
                "dtype": rng.choice(["bf16", "bf16", "f16", "f32"]), "weight": rng.choice(["f32", "bf16"]),
                "residual": rng.random() < 0.7, "out": "int8" if int8 else rng.choice(["bf16", "f16", "f32"]),
                "block": block}
    if op == "rms_grad":
        D = _width(rng, 16, 16384)
        return {"op": op, "T": _log(rng, 1, min(65536, 16384 * H_20B // D)), "D": D,
                "dtype": rng.choice(["bf16", "bf16", "f16", "f32"]), "weight": rng.choice(["f32", "bf16"]),
                "residual": rng.random() < 0.7}
    V = rng.choice([_log(rng, 1000, 131072), _log(rng, 1000, 131072) // 64 * 64])
    case = {"op": op, "T": _log(rng, 1, 4096 * VOCAB // V if op == "policy" else 2048 * VOCAB // V), "V": V,
            "logits": rng.choice(["bf16", "bf16", "f16", "f32"]), "scale": rng.choice([1.0, 1.0, 1.25, 0.5]),
            "pad": rng.choice([0.0, 0.1])}
    if op == "policy":
        case.update(grad=case["logits"], kl=rng.choice([0.0, 0.05]))
    return case


# ---------------------------------------------------------------- inputs

def _gen(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    return gen


def _randn(n, std, gen, dtype="f32"):
    return (torch.randn(n, generator=gen, device=DEV) * std).to(_DT[dtype])


def _blocks(x, block):
    """x as rows of one block each, the last one padded with zeros."""
    short = -x.numel() % block
    return (torch.nn.functional.pad(x, (0, short)) if short else x).view(-1, block)


def _encode(x, block, qmax):
    """Symmetric absmax codes (int8, one an element) and scales."""
    b = _blocks(x, block)
    a = b.abs().amax(1)
    top = torch.full_like(a, qmax)
    codes = torch.round(b * torch.where(a > 0, top / a, torch.zeros_like(a))[:, None]).to(torch.int8)
    return codes.view(-1)[: x.numel()].contiguous(), a / top


def _pack(codes):
    """Two codes a byte, the first in the low half."""
    if codes.numel() % 2:
        codes = torch.nn.functional.pad(codes, (0, 1))
    pair = codes.view(torch.uint8).view(-1, 2)
    return (pair[:, 0] & 15) | (pair[:, 1] << 4)


def _specs(case):
    """(gradient's dtype, elements) of each tensor of an adamw case."""
    if case["tensors"] == "layers":
        h = case["h"]
        matrices = [("bf16", n) for n in (3 * h * h, h * h, 4 * h * h, 4 * h * h)]
        vectors = [("f32", n) for n in (3 * h, h, 4 * h, h, h, h, h, h)]
        return (matrices + vectors) * case["count"]
    if "sizes" not in case:
        return [("int4", case["n"])] * case["count"]
    rng = random.Random(case["sizes"])
    sizes = [_log(rng, max(1, case["n"] // 1000), case["n"]) for _ in range(case["count"])]
    if case["tensors"] == "shards":
        return [("int4", n) for n in sizes]
    return [(rng.choice(["bf16", "f16", "f32", "int4"]), n) for n in sizes]


def _decays(case):
    """Weight decay of each tensor: none for vectors."""
    if case["tensors"] == "layers":
        return ([DECAY] * 4 + [0.0] * 8) * case["count"]
    return [DECAY] * len(_specs(case))


def _adamw_inputs(case, gen):
    """The training program's flat buffers and each tensor's part of them."""
    sizes = [n for _, n in _specs(case)]
    total, i = sum(sizes), {"step": 100}
    i["param"] = _randn(total, 0.02, gen, case["param"])
    grads, squares = [], torch.zeros((), dtype=torch.float64, device=DEV)
    for dtype, n in _specs(case):
        if dtype == "int4":
            codes, scales = _encode(_randn(n, 1e-3, gen), case["block"], 7.0)
            squares += (_blocks(codes.float(), case["block"]).square().sum(1).double() * scales.double().square()).sum()
            grads.append((_pack(codes), scales, n, case["block"]))
        else:
            grads.append(_randn(n, 1e-3, gen, dtype))
            squares += grads[-1].float().square().sum(dtype=torch.float64)
    i["grads"], i["norm"] = grads, squares.sqrt().float()
    m = _randn(total, 3e-4, gen)
    v = _randn(total, 1e-3, gen).square_()
    if case["state"] == 32:
        i["m"], i["v"] = m, v
        i["ms"], i["vs"] = list(m.split(sizes)), list(v.split(sizes))
    else:
        block = case["state_block"]
        counts = [-(-n // block) for n in sizes]
        for name, x, dtype, top in (("m", m, torch.float8_e4m3fn, 448.0), ("v", v, torch.float8_e5m2, 57344.0)):
            codes = torch.empty(total, dtype=dtype, device=DEV)
            scales = torch.empty(sum(counts), dtype=torch.float32, device=DEV)
            parts = list(zip(codes.split(sizes), scales.split(counts)))
            for (c, s), part in zip(parts, x.split(sizes)):
                b = _blocks(part, block)
                s.copy_(b.abs().amax(1) * (1.0 / top))
                c.copy_((b / s[:, None].clamp(min=1e-30)).clamp(-top, top).view(-1)[: part.numel()].to(dtype))
            i[name], i[name + "_scales"] = codes, scales
            i[name + "s"] = [(c, s, block) for c, s in parts]
    i["params"] = list(i["param"].split(sizes))
    if case["out"] == "int8":
        # one buffer of whole blocks: a tensor's part starts with a block
        block = case["out_block"]
        counts = [-(-n // block) for n in sizes]
        i["out"] = torch.zeros(sum(counts) * block, dtype=torch.int8, device=DEV)
        i["out_scales"] = torch.zeros(sum(counts), dtype=torch.float32, device=DEV)
        parts = zip(i["out"].split([c * block for c in counts]), i["out_scales"].split(counts))
        i["outs"] = [(codes[:n], scales, block) for n, (codes, scales) in zip(sizes, parts)]
        i["out_values"] = torch.empty(sum(counts) * block, dtype=torch.bfloat16, device=DEV)
    elif case["out"]:
        i["out"] = torch.zeros(total, dtype=_DT[case["out"]], device=DEV)
        i["outs"] = list(i["out"].split(sizes))
    else:
        i["outs"] = None
    return i


def _inputs(case, seed):
    gen, op = _gen(seed), case["op"]
    if op == "adamw":
        return _adamw_inputs(case, gen)
    T = case["T"]
    if op in ("rms", "rms_grad"):
        D, dtype = case["D"], case["dtype"]
        weight = (1.0 + 0.1 * _randn(D, 1.0, gen)).to(_DT[case["weight"]])
        x = _randn(T * D, 1.0, gen, dtype).view(T, D)
        if op == "rms":
            return {"weight": weight, "x": x,
                    "residual": _randn(T * D, 2.0, gen, dtype).view(T, D) if case["residual"] else None}
        # as the forward pass left them: the rows that were normed, and 1 / rms of each
        return {"weight": weight, "h": x, "rstd": torch.rsqrt(x.double().square().mean(1) + 1e-5).float(),
                "dy": _randn(T * D, 1e-3, gen, dtype).view(T, D),
                "dh": _randn(T * D, 1e-3, gen, dtype).view(T, D) if case["residual"] else None}
    V = case["V"]
    logits = _randn(T * V, 2.0, gen, case["logits"]).view(T, V)
    ids = (torch.exp(torch.rand(T, generator=gen, device=DEV, dtype=torch.float64) * math.log(V + 1)).long() - 1).clamp_(0, V - 1)
    # the sampled token is one that the model finds likely
    at = torch.arange(T, device=DEV)
    logits[at, ids] = (logits[at, ids].float() + 10.0 * torch.rand(T, generator=gen, device=DEV)).to(_DT[case["logits"]])
    pad = torch.rand(T, generator=gen, device=DEV) < case["pad"]
    i = {"logits": logits, "ids": torch.where(pad, torch.full_like(ids, -1), ids)}
    if op == "policy":
        z = logits.float() * case["scale"]
        logp = z[at, ids] - torch.logsumexp(z, 1)
        del z
        i["old_logp"] = logp + 0.15 * _randn(T, 1.0, gen)
        i["ref_logp"] = logp + 0.3 * _randn(T, 1.0, gen) if case["kl"] else None
        i["advantages"] = _randn(T, 1.0, gen)
        i["weights"] = torch.where(pad, torch.zeros(T, device=DEV), torch.full((T,), 1.0 / T, device=DEV))
    return i


# ---------------------------------------------------------------- the calls

def prepare(case, seed):
    state = _inputs(case, seed)
    state["case"] = case
    if own and case["op"] == "adamw":
        # built once for the buffers of a training run
        import paper_2501_04266_amd as zq
        state["table"] = zq.adamw_table(state["params"], state["grads"], state["ms"], state["vs"], state["outs"],
                                        weight_decay=_decays(case))
    return state


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _adamw_outputs(state):
    got = [state[k] for k in ("param", "m", "v", "m_scales", "v_scales") if k in state]
    if state["case"]["out"] == "int8":
        return got + [state["out_values"], state["out_scales"]]
    return got + [state["out"]] if state["case"]["out"] else got


def _run_own(state):
    import paper_2501_04266_amd as zq
    case = state["case"]
    op = case["op"]
    if op == "adamw":
        state["step"] += 1
        zq.adamw_step(state["table"], state["step"], LR, (BETA1, BETA2), EPS,
                      norm=state["norm"] if case["clip"] else None, max_norm=1.0)
        if case["out"] == "int8":
            zq.qwz_dequantize(state["out"], state["out_scales"], case["out_block"], y=state["out_values"])
        return _adamw_outputs(state)
    if op == "rms":
        if case["out"] == "int8":
            codes, scales, h, rstd = zq.qwz_rms_norm(state["x"], state["weight"], state["residual"], eps=1e-5,
                                                     block=case["block"])
            y = zq.qwz_dequantize(codes, scales, case["block"], torch.bfloat16).view(case["T"], case["D"])
            return [y, scales, rstd] + ([h] if case["residual"] else [])
        y, h, rstd = zq.rms_norm(state["x"], state["weight"], state["residual"], eps=1e-5,
                                 out_dtype=_DT[case["out"]])
        return [y, rstd] + ([h] if case["residual"] else [])
    if op == "rms_grad":
        return zq.rms_norm_grad(state["dy"], state["h"], state["weight"], state["rstd"], state["dh"])
    if op == "logp":
        return zq.token_logp(state["logits"], state["ids"], scale=case["scale"])
    return zq.policy_loss(state["logits"], state["ids"], state["old_logp"], state["advantages"], state["weights"],
                          state["ref_logp"], clip=(0.2, 0.2), kl=case["kl"], scale=case["scale"],
                          grad_dtype=_DT[case["grad"]])


# ---------------------------------------------------------------- in plain torch

def _mix(x):
    """32 bits of x (held in 64) to 32 bits that look like drawn ones."""
    low = 0xFFFFFFFF
    x = x ^ (x >> 16)
    x = x * 0x6A09E667 & low
    x = x ^ (x >> 15)
    x = x * 0x3B67AE85 & low
    return x ^ (x >> 16)


def _mix_int(x):
    return int(_mix(torch.tensor(x & 0xFFFFFFFF, dtype=torch.int64)))


def _drawn(step, tensor, n):
    """The rounding bits of a tensor's elements: a function of the step, the tensor's place in the list and theirs in it."""
    key = _mix_int(_mix_int(step) + tensor * 0x9E3779B9)
    return _mix(torch.arange(n, device=DEV) ^ key)  # n < 2^32


def _decode8(part):
    codes, scales, block = part
    return (_blocks(codes.view(torch.uint8), block).view(codes.dtype).float() * scales[:, None]).view(-1)[: codes.numel()]


def _encode8(x, part, bits):
    """x into float8 codes and scales: e4m3 with a sign or e5m2 without, rounded up with the chance of the part cut off."""
    codes, scales, block = part
    signed = codes.dtype == torch.float8_e4m3fn
    top, shift, unit, last = (448.0, 20, 2.0**-120, 126) if signed else (57344.0, 21, 2.0**-112, 123)
    b = _blocks(x, block)
    a = b.abs().amax(1)
    full = torch.full_like(a, top)
    fits = a >= 2.0**-110
    scales.copy_(torch.where(fits, a / full, torch.zeros_like(a)))
    r = torch.where(fits, full / torch.where(fits, a, full), torch.zeros_like(a))
    y = ((b.abs() * r[:, None]) * unit).view(-1)[: x.numel()]
    cut = (bits & 0xFFFF) * 16 + 8 if signed else (bits >> 16) * 32 + 16
    code = ((y.view(torch.int32).long() + cut) >> shift).clamp(max=last)
    if signed:
        code = code + 128 * (x < 0).long()
    codes.view(torch.uint8).copy_(code.to(torch.uint8))


def _plain_adamw(state):
    case = state["case"]
    state["step"] += 1
    step = state["step"]
    om1, om2 = torch.tensor([1.0 - BETA1, 1.0 - BETA2], dtype=torch.float64).float().tolist()
    b1, b2, eps = torch.tensor([BETA1, BETA2, EPS], dtype=torch.float64).float().tolist()
    root = float(torch.tensor(1.0 / math.sqrt(1.0 - BETA2**step), dtype=torch.float64).float())
    alpha = float(torch.tensor(LR / (1.0 - BETA1**step), dtype=torch.float64).float())
    c = torch.ones((), device=DEV)
    if case["clip"]:
        c = torch.clamp(torch.ones((), device=DEV) / (state["norm"] + 1e-6), max=1.0)
    for k, (p, grad, m8, v8, wd) in enumerate(zip(state["params"], state["grads"], state["ms"], state["vs"],
                                                  _decays(case))):
        n = p.numel()
        if isinstance(grad, tuple):
            packed, scales, _, block = grad
            low, high = (packed << 4).view(torch.int8) >> 4, packed.view(torch.int8) >> 4
            q = torch.stack((low, high), 1).view(-1)[:n].float()
            g = (_blocks(q, block) * (scales * c)[:, None]).view(-1)[:n]
        else:
            g = grad.float() * c
        m, v = (m8, v8) if case["state"] == 32 else (_decode8(m8), _decode8(v8))
        m = m * b1 + g * om1
        v = v * b2 + (g * g) * om2
        decay = float(torch.tensor(1.0 - LR * wd, dtype=torch.float64).float())
        new = p.float() * decay - (m / (v.sqrt() * root + eps)) * alpha
        p.copy_(new)
        if case["state"] == 32:
            m8.copy_(m)
            v8.copy_(v)
        else:
            bits = _drawn(step, k, n)
            _encode8(m, m8, bits)
            _encode8(v, v8, bits)
        if case["out"] == "int8":
            codes, scales, block = state["outs"][k]
            q, s = _encode(p.float(), block, 127.0)
            codes.copy_(q)
            scales.copy_(s)
        elif case["out"]:
            state["outs"][k].copy_(p)
    if case["out"] == "int8":
        state["out_values"].copy_((_blocks(state["out"].float(), case["out_block"])
                                   * state["out_scales"][:, None]).view(-1))
    return _adamw_outputs(state)


def _plain_rms(state):
    case = state["case"]
    h = state["x"]
    if case["residual"]:
        h = (h.float() + state["residual"].float()).to(h.dtype)
    x = h.float()
    # a sum of thousands of squares, and INT8 codes next to it: in 64 bits
    rstd = torch.rsqrt(x.double().square().mean(1) + 1e-5).float()
    y = (x * rstd[:, None]) * state["weight"].float()
    if case["out"] != "int8":
        return [y.to(_DT[case["out"]]), rstd] + ([h] if case["residual"] else [])
    codes, scales = _encode(y.view(-1), case["block"], 127.0)
    y = (_blocks(codes.float(), case["block"]) * scales[:, None]).view(y.shape).bfloat16()
    return [y, scales, rstd] + ([h] if case["residual"] else [])


def _plain_rms_grad(state):
    h, dy, rstd = state["h"].float(), state["dy"].float(), state["rstd"][:, None]
    xh = h * rstd
    dxh = dy * state["weight"].float()
    dx = (dxh - xh * (dxh * xh).mean(1, keepdim=True)) * rstd
    if state["dh"] is not None:
        dx = dx + state["dh"].float()
    return dx.to(state["h"].dtype), (dy * xh).sum(0)


def _plain_policy(state):
    case = state["case"]
    logits, ids, scale = state["logits"], state["ids"], case["scale"]
    real = ids >= 0
    at = ids.clamp(min=0)[:, None]
    z = logits.float()
    top = z.amax(1, keepdim=True)
    p = torch.exp((z - top) * scale)
    total = p.sum(1, dtype=torch.float64)
    # clipping asks on which side of a border the ratio is: its logarithm in 64 bits
    logp = (z.gather(1, at) - top).view(-1).double() * scale - torch.log(total)
    zero = torch.zeros((), dtype=torch.float64, device=DEV)
    if case["op"] == "logp":
        return torch.where(real, logp, zero).float()
    A, w = state["advantages"].double(), torch.where(real, state["weights"].double(), zero)
    ratio = torch.exp(logp - state["old_logp"].double())
    clipped = torch.where(A > 0, ratio > 1.2, (A < 0) & (ratio < 0.8))
    pg = -torch.minimum(ratio * A, ratio.clamp(0.8, 1.2) * A)
    slope = torch.where(clipped, zero, -A * ratio)
    kl = zero.expand_as(pg)
    if case["kl"]:
        d = state["ref_logp"].double() - logp
        kl = torch.exp(d) - d - 1.0
        slope = slope + case["kl"] * (1.0 - torch.exp(d))
    sums = torch.stack(((w * (pg + case["kl"] * kl)).sum(), (w * pg).sum(), (w * kl).sum(), (w * clipped).sum()))
    g = (w * slope * scale).float()[:, None]
    p *= -(g / total.float()[:, None])
    p.scatter_add_(1, at, g)
    return sums.float(), torch.where(real, logp, zero).float(), p.to(_DT[case["grad"]])


def _run_plain(state):
    op = state["case"]["op"]
    if op == "adamw":
        return _plain_adamw(state)
    if op == "rms":
        return _plain_rms(state)
    if op == "rms_grad":
        return _plain_rms_grad(state)
    return _plain_policy(state)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    op = case["op"]
    if op == "adamw":
        size = flops = 0.0
        for dtype, n in _specs(case):
            size += n * (0.5 + 4.0 / case["block"] if dtype == "int4" else _SIZE[dtype])
            size += n * 2 * _SIZE[case["param"]]
            size += n * (16.0 if case["state"] == 32 else 2 * (2.0 + 8.0 / case["state_block"]))
            if case["out"] == "int8":  # written, read and written dequantised
                size += n * (2 * (1.0 + 4.0 / case["out_block"]) + 2.0)
            elif case["out"]:
                size += n * _SIZE[case["out"]]
            flops += 14.0 * n
        return {"bytes": float(size), "flops": float(flops)}
    T = case["T"]
    if op in ("rms", "rms_grad"):
        D, e = case["D"], _SIZE[case["dtype"]]
        weight = D * _SIZE[case["weight"]]
        if op == "rms":
            size = T * D * e * (3 if case["residual"] else 1) + 4.0 * T + weight
            if case["out"] == "int8":  # written, read and written dequantised
                size += T * D * (2 * (1.0 + 4.0 / case["block"]) + 2.0)
            else:
                size += T * D * _SIZE[case["out"]]
            return {"bytes": float(size), "flops": 6.0 * T * D}
        size = T * D * e * (4 if case["residual"] else 3) + 4.0 * T + weight + 4.0 * D
        return {"bytes": float(size), "flops": 10.0 * T * D}
    rows, V, e = T * (1.0 - case["pad"]), case["V"], _SIZE[case["logits"]]
    if op == "logp":
        return {"bytes": float(rows * V * e + 12.0 * T), "flops": 4.0 * rows * V}
    return {"bytes": float(rows * V * e + T * V * _SIZE[case["grad"]] + 28.0 * T + 16.0), "flops": 7.0 * rows * V}


# ---------------------------------------------------------------- in 64 bits

def _signed(packed, n):
    """The INT4 codes as doubles: two's complement halves of each byte."""
    out = torch.empty(packed.numel() * 2, dtype=torch.float64, device=DEV)
    for half in (0, 1):
        u = (packed.to(torch.int32) >> (4 * half)) & 15
        out[half::2] = (u - 16 * (u > 7)).double()
    return out[:n]


def _spread(scales, block, n):
    return scales.double().repeat_interleave(block)[:n]


def _int8_values(y, block):
    """y (whole blocks, or a last short one) as its INT8 codes and scales stand for it, and the scales."""
    n = y.numel()
    a = torch.cat((y.abs(), y.new_zeros(-n % block))).view(-1, block).max(1).values
    step = (a / 127.0).repeat_interleave(block)[:n]
    return torch.where(step > 0, torch.round(y / step.clamp(min=1e-300)), torch.zeros_like(y)) * step, a / 127.0


def _exact_adamw(case, i):
    t = i["step"] + 1
    c = min(1.0, 1.0 / (float(i["norm"]) + 1e-6)) if case["clip"] else 1.0
    got = []
    for p, g, m, v, wd in zip(i["params"], i["grads"], i["ms"], i["vs"], _decays(case)):
        n = p.numel()
        g = c * (_signed(g[0], n) * _spread(g[1], g[3], n) if isinstance(g, tuple) else g.double())
        if case["state"] == 32:
            m, v = m.double(), v.double()
        else:
            m, v = (x.double() * _spread(s, b, n) for x, s, b in (m, v))
        m = BETA1 * m + (1.0 - BETA1) * g
        v = BETA2 * v + (1.0 - BETA2) * g**2
        step = LR * (m / (1.0 - BETA1**t)) / (torch.sqrt(v / (1.0 - BETA2**t)) + EPS)
        got.append((p.double() * (1.0 - LR * wd) - step, m, v))
    param, m, v = (torch.cat(x) for x in zip(*got))
    # 8-bit moments are rounded by drawn bits: no value of theirs but the drawn one
    answer = [param, m, v] if case["state"] == 32 else [param, None, None, None, None]
    if case["out"] == "int8":
        whole = [torch.nn.functional.pad(x[0].to(_DT[case["param"]]).double(), (0, -x[0].numel() % case["out_block"]))
                 for x in got]
        return answer + list(_int8_values(torch.cat(whole), case["out_block"]))
    return answer + [param] if case["out"] else answer


def exact(case, seed):
    i, op = _inputs(case, seed), case["op"]
    if op == "adamw":
        return _exact_adamw(case, i)
    if op == "rms":
        h = i["x"].double()
        if case["residual"]:
            h = (h + i["residual"].double()).to(i["x"].dtype).double()
        rms = torch.sqrt((h * h).sum(1) / case["D"] + 1e-5)
        y = h / rms[:, None] * i["weight"].double()
        tail = [h] if case["residual"] else []
        if case["out"] != "int8":
            return [y, 1.0 / rms] + tail
        values, scales = _int8_values(y.reshape(-1), case["block"])
        return [values.view(y.shape), scales, 1.0 / rms] + tail
    if op == "rms_grad":
        D, rows = case["D"], []
        dw = torch.zeros(D, dtype=torch.float64, device=DEV)
        w = i["weight"].double()
        for part in torch.arange(case["T"], device=DEV).split(2048):
            h, dy, s = i["h"][part].double(), i["dy"][part].double(), i["rstd"][part].double()[:, None]
            dw += (dy * h * s).sum(0)
            along = (dy * w * h).sum(1, keepdim=True)
            dx = s * dy * w - s**3 * h * along / D
            rows.append(dx + i["dh"][part].double() if case["residual"] else dx)
        return torch.cat(rows), dw
    ids, scale = i["ids"], case["scale"]
    T, V = i["logits"].shape
    logps = torch.zeros(T, dtype=torch.float64, device=DEV)
    grad = torch.zeros(T, V, dtype=torch.float64, device=DEV) if op == "policy" else None
    sums = torch.zeros(4, dtype=torch.float64, device=DEV)
    for part in (ids >= 0).nonzero().view(-1).split(1024):
        rows = torch.log_softmax(i["logits"][part].double() * scale, 1)
        a = ids[part]
        lp = rows.take_along_dim(a[:, None], 1)[:, 0]
        logps[part] = lp
        if op == "logp":
            continue
        A, w, old = (i[k][part].double() for k in ("advantages", "weights", "old_logp"))
        ratio = (lp - old).exp()
        free, held = ratio * A, torch.clip(ratio, 0.8, 1.2) * A
        clipped = free > held
        pg = -torch.where(clipped, held, free)
        slope = torch.where(clipped, torch.zeros_like(A), -free)
        kl = torch.zeros_like(A)
        if case["kl"]:
            more = i["ref_logp"][part].double() - lp
            kl = torch.expm1(more) - more
            slope = slope - case["kl"] * torch.expm1(more)
        sums += torch.stack([(w * x).sum() for x in (pg + case["kl"] * kl, pg, kl, clipped.double())])
        hot = torch.zeros_like(rows)
        hot[torch.arange(a.numel(), device=DEV), a] = 1.0
        grad[part] = (w * slope * scale)[:, None] * (hot - rows.exp())
    return logps if op == "logp" else (sums, logps, grad)
