"""Timed workloads of the operators around the compression path: the embedding
layer, gradient norm and clipping, and products with INT4 weights.

A case's "op" says which operator it makes a pass through:

  embedding   rows of the embedding table by token id, scaled: the table as INT8
              codes and scales (as gathered), or dense
  gradient    the embedding table's gradient from the rows' gradients: dense, rows of
              tokens that do not occur are zero
  norm        the norm of all gradients of a rank: dense tensors, or the INT4 shards
              that a reduce level leaves
  clip        the norm, then the gradients scaled down to a largest norm into the
              flat buffer that the optimizer reads
  product     products of a few tokens with weights held as INT4 codes and block scales

Sizes are those of the package's own workloads where it has them (hidden 2048 and 6144,
one layer 12 h^2 elements, gradient shards of 1/8); vocabularies and token counts are
generic.  Token ids are drawn with a frequency of about 1 / rank, as in text; padding
is id -1 (a row of zeros, no gradient).  `draw` spreads over the same ranges.
"""
import math
import random

import torch

# run() in plain torch, or through the package's calls
own = False

DEV = "cuda"
_DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "f16": 2, "bf16": 2}
H_13B, H_20B = 2048, 6144
SHARD_20B = 12 * H_20B * H_20B // 8


def listed():
    return [
        # generation: the next token's row, the table as gathered; a call's latency
        {"name": "embed-token", "op": "embedding", "T": 1, "V": 50000, "D": H_20B, "table": "int8", "block": 256,
         "out": "bf16", "scale": 1.0, "pad": 0.0},
        # a training micro-batch of 8 x 2048 tokens, rows scaled by sqrt(D), some of them padding
        {"name": "embed-batch", "op": "embedding", "T": 16384, "V": 50000, "D": H_20B, "table": "bf16", "block": 0,
         "out": "bf16", "scale": 78.5, "pad": 0.05},
        # a short sequence through a small model's table
        {"name": "grad-short", "op": "gradient", "T": 512, "V": 8000, "D": 1024, "dtype": "f32", "out": "f32",
         "scale": 1.0, "pad": 0.0},
        # the micro-batch's gradient of the whole table, the fp32 buffer that is compressed next
        {"name": "grad-batch", "op": "gradient", "T": 16384, "V": 50000, "D": H_20B, "dtype": "bf16", "out": "f32",
         "scale": 78.5, "pad": 0.05},
        # many more tokens than rows, odd sizes everywhere: rows start at any 2-byte address
        {"name": "grad-ragged", "op": "gradient", "T": 40001, "V": 16411, "D": 2051, "dtype": "f16", "out": "f32",
         "scale": 1.0, "pad": 0.0},
        # the INT4 gradient shards of 16 layers after their last reduce level
        {"name": "norm-shards", "op": "norm", "tensors": "shards", "count": 16, "n": SHARD_20B, "block": 128},
        # an unsharded model of 24 layers, tensor by tensor: matrices bf16, vectors f32
        {"name": "norm-model", "op": "norm", "tensors": "layers", "count": 24, "h": H_13B},
        # one layer's tensors clipped into the optimizer's fp32 gradients
        {"name": "clip-layer", "op": "clip", "tensors": "layers", "count": 1, "h": H_13B, "out": "f32",
         "unscale": 1.0},
        # one INT4 shard, clipped as it is dequantised; gradients carry a loss scale of 1024
        {"name": "clip-shard", "op": "clip", "tensors": "shards", "count": 1, "n": SHARD_20B, "block": 128,
         "out": "f32", "unscale": 1.0 / 1024},
        # generation: one token through the four products of a layer
        {"name": "token-layer", "op": "product", "M": 1, "shapes": "18432x6144,6144x6144,24576x6144,6144x24576",
         "block": 128, "dtype": "bf16"},
        # 16 sequences a step through a smaller layer, finer scales
        {"name": "batch-layer", "op": "product", "M": 16, "shapes": "6144x2048,2048x2048,8192x2048,2048x8192",
         "block": 64, "dtype": "f16"},
        # the output head for a few sequences: a vocabulary that no tile divides
        {"name": "head-5", "op": "product", "M": 5, "shapes": "50001x6144", "block": 128, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A row length: a multiple of 64 mostly, sometimes of 8, sometimes any number."""
    step = rng.choice([128, 128, 128, 8, 1])
    n = _log(rng, lo, hi)
    return max(lo, n // step * step + (64 if step == 128 and n < 6000 else 0))


def draw(rng):
    op = rng.choice(["embedding", "gradient", "norm", "clip", "product"])
    if op == "embedding":
        D, table = _width(rng, 64, 8192), rng.choice(["int8", "int8", "bf16", "f16", "f32"])
        T = _log(rng, 1, min(32768, 16384 * H_20B // D))
        return {"op": op, "T": T, "V": _log(rng, 1000, 131072), "D": D, "table": table,
                "block": rng.choice([64, 128, 256]) if table == "int8" else 0,
                "out": rng.choice(["bf16", "f16", "f32"]), "scale": rng.choice([1.0, math.sqrt(D)]),
                "pad": rng.choice([0.0, 0.0, 0.1])}
    if op == "gradient":
        D = _width(rng, 64, 8192)
        T = _log(rng, 1, min(65536, 16384 * H_20B // D))
        return {"op": op, "T": T, "V": _log(rng, 1000, min(131072, 50000 * H_20B // D)), "D": D,
                "dtype": rng.choice(["bf16", "bf16", "f16", "f32"]), "out": rng.choice(["f32", "f32", "bf16"]),
                "scale": rng.choice([1.0, math.sqrt(D)]), "pad": rng.choice([0.0, 0.0, 0.1])}
    if op in ("norm", "clip"):
        tensors = rng.choice(["shards", "layers", "mixed"])
        case = {"op": op, "tensors": tensors}
        most = 24 * 12 * H_13B * H_13B if op == "norm" else 4 * 12 * H_13B * H_13B
        if tensors == "layers":
            case["h"] = rng.choice([1536, 2048])
            case["count"] = rng.randint(1, most // (12 * case["h"] ** 2))
        else:
            case["count"] = _log(rng, 1, 16) if tensors == "shards" else _log(rng, 1, 400)
            case["n"] = _log(rng, 1000, most // case["count"])
            case["block"] = rng.choice([64, 128, 256])
            case["sizes"] = rng.randrange(1 << 30)
        if op == "clip":
            case.update(out=rng.choice(["f32", "f32", "bf16"]), unscale=rng.choice([1.0, 1.0 / 1024]))
        return case
    K = _log(rng, 8, 384) * 64
    N = _log(rng, 1000, min(65536, 49152 * H_20B // K))
    if rng.random() < 0.6:  # else an output width that no tile divides
        N = N // 64 * 64
    return {"op": op, "M": _log(rng, 1, 64), "shapes": f"{N}x{K}", "block": rng.choice([32, 64, 128, 128, 256]),
            "dtype": rng.choice(["bf16", "bf16", "f16"])}


# ---------------------------------------------------------------- inputs

def _gen(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    return gen


def _randn(n, std, gen, dtype="f32"):
    return (torch.randn(n, generator=gen, device=DEV) * std).to(_DT[dtype])


def _ids(case, gen):
    """Token ids, rank r about as often as 1 / (r + 1), a share of them padding."""
    T, V = case["T"], case["V"]
    u = torch.rand(T, generator=gen, device=DEV, dtype=torch.float64)
    ids = (torch.exp(u * math.log(V + 1)).long() - 1).clamp_(0, V - 1)
    pad = torch.rand(T, generator=gen, device=DEV) < case["pad"]
    return torch.where(pad, torch.full_like(ids, -1), ids)


def _blocks(x, block):
    """x as rows of one block each, the last one padded with zeros."""
    short = -x.numel() % block
    return (torch.nn.functional.pad(x, (0, short)) if short else x).view(-1, block)


def _encode(x, block, qmax):
    """Symmetric absmax codes (int8, one an element) and scales."""
    b = _blocks(x, block)
    a = b.abs().amax(1)
    codes = torch.round(b * torch.where(a > 0, qmax / a, torch.zeros_like(a))[:, None]).to(torch.int8)
    return codes.view(-1)[: x.numel()].contiguous(), a / qmax


def _pack(codes):
    """Two codes a byte, the first in the low half."""
    if codes.numel() % 2:
        codes = torch.nn.functional.pad(codes, (0, 1))
    pair = codes.view(torch.uint8).view(-1, 2)
    return (pair[:, 0] & 15) | (pair[:, 1] << 4)


def _unpack(packed, n):
    low = (packed << 4).view(torch.int8) >> 4
    high = packed.view(torch.int8) >> 4
    return torch.stack((low, high), 1).view(-1)[:n]


def _specs(case):
    """(dtype, elements) of each gradient tensor of a norm or clip case."""
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


def _gradients(case, gen):
    """The gradient tensors: dense ones, or (packed codes, scales, elements, block)."""
    std, got = 1e-3 / case.get("unscale", 1.0), []
    for dtype, n in _specs(case):
        if dtype == "int4":
            codes, scales = _encode(_randn(n, std, gen), case["block"], 7.0)
            got.append((_pack(codes), scales, n, case["block"]))
        else:
            got.append(_randn(n, std, gen, dtype))
    return got


def _shapes(case):
    return [tuple(int(v) for v in s.split("x")) for s in case["shapes"].split(",")]


def _inputs(case, seed):
    gen, op = _gen(seed), case["op"]
    if op == "embedding":
        V, D = case["V"], case["D"]
        ids = _ids(case, gen)
        if case["table"] != "int8":
            return {"ids": ids, "table": _randn(V * D, 0.02, gen, case["table"]).view(V, D)}
        codes, scales = _encode(_randn(V * D, 0.02, gen), case["block"], 127.0)
        return {"ids": ids, "codes": codes, "scales": scales}
    if op == "gradient":
        ids = _ids(case, gen)
        return {"ids": ids, "dy": _randn(case["T"] * case["D"], 1e-3, gen, case["dtype"]).view(case["T"], case["D"])}
    if op in ("norm", "clip"):
        return {"grads": _gradients(case, gen)}
    products = []
    for N, K in _shapes(case):
        x = _randn(case["M"] * K, 1.0, gen, case["dtype"]).view(case["M"], K)
        codes, scales = _encode(_randn(N * K, 0.02, gen), case["block"], 7.0)
        products.append((x, _pack(codes), scales, N))
    return {"products": products}


# ---------------------------------------------------------------- the calls

def prepare(case, seed):
    state = _inputs(case, seed)
    state["case"] = case
    if case["op"] == "clip":
        # the optimizer's gradients: one flat buffer, a tensor's part after the other's
        sizes = [n for _, n in _specs(case)]
        state["flat"] = torch.empty(sum(sizes), dtype=_DT[case["out"]], device=DEV)
        state["outs"] = list(state["flat"].split(sizes))
    if own and case["op"] in ("norm", "clip"):
        # built once for the gradient buffers of a training run
        import paper_2501_04266_amd as zq
        state["table"] = zq.grad_table(state["grads"], state.get("outs"))
    return state


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    import paper_2501_04266_amd as zq
    case = state["case"]
    op = case["op"]
    if op == "embedding":
        if case["table"] != "int8":
            return zq.embedding(state["ids"], state["table"], scale=case["scale"], out_dtype=_DT[case["out"]])
        return zq.qwz_embedding(state["ids"], state["codes"], state["scales"], case["V"], case["D"], case["block"],
                                scale=case["scale"], out_dtype=_DT[case["out"]])
    if op == "gradient":
        return zq.embedding_grad(state["ids"], state["dy"], case["V"], scale=case["scale"],
                                 out_dtype=_DT[case["out"]])
    if op == "norm":
        return zq.grad_norm(state["table"])
    if op == "clip":
        norm = zq.grad_norm(state["table"], scale=case["unscale"])
        zq.grad_clip(state["table"], norm, 1.0, scale=case["unscale"])
        return norm, state["flat"]
    return [zq.int4_dequant_gemm(x, packed, scales, N, case["block"]) for x, packed, scales, N in state["products"]]


def _plain_dequant(packed, scales, n, block):
    return (_blocks(_unpack(packed, n).float(), block) * scales[:, None]).view(-1)[:n]


def _plain_norm(grads, scale):
    total = torch.zeros((), dtype=torch.float32, device=DEV)
    for g in grads:
        g = _plain_dequant(*g) if isinstance(g, tuple) else g.float()
        total = total + (g * g).sum()
    return torch.sqrt(total) * scale


def _run_plain(state):
    case = state["case"]
    op = case["op"]
    if op == "embedding":
        ids, D = state["ids"], case["D"]
        at = ids.clamp(min=0)
        if case["table"] == "int8":
            flat = at[:, None] * D + torch.arange(D, device=DEV)
            rows = state["codes"].view(-1, D)[at].float() * state["scales"][flat // case["block"]]
        else:
            rows = state["table"][at].float()
        rows = torch.where(ids[:, None] < 0, torch.zeros((), device=DEV), rows * case["scale"])
        return rows.to(_DT[case["out"]])
    if op == "gradient":
        ids = state["ids"]
        # padding goes to a row of its own, which is cut off
        dw = torch.zeros(case["V"] + 1, case["D"], dtype=torch.float32, device=DEV)
        dw.index_add_(0, torch.where(ids < 0, torch.full_like(ids, case["V"]), ids), state["dy"].float())
        return (dw[: case["V"]] * case["scale"]).to(_DT[case["out"]])
    if op == "norm":
        return _plain_norm(state["grads"], 1.0)
    if op == "clip":
        norm = _plain_norm(state["grads"], case["unscale"])
        c = torch.clamp(1.0 / (norm + 1e-6), max=1.0) * case["unscale"]
        for g, out in zip(state["grads"], state["outs"]):
            out.copy_((_plain_dequant(*g) if isinstance(g, tuple) else g.float()) * c)
        return norm, state["flat"]
    outs = []
    for x, packed, scales, N in state["products"]:
        K = x.shape[1]
        w = _plain_dequant(packed, scales, N * K, case["block"]).view(N, K)
        outs.append(x.float() @ w.t())
    return outs


# ---------------------------------------------------------------- what a pass cannot do without

def _distinct(case):
    """Expected number of distinct rows that the ids name."""
    r = torch.arange(1, case["V"] + 1, dtype=torch.float64)
    p = torch.log1p(1.0 / r) / math.log(case["V"] + 1) * (1.0 - case["pad"])
    return float((1.0 - (1.0 - p) ** case["T"]).sum())


def work(case):
    op = case["op"]
    if op == "embedding":
        T, D = case["T"], case["D"]
        row = D * (1 + 4.0 / case["block"]) if case["table"] == "int8" else D * _SIZE[case["table"]]
        size = 8.0 * T + _distinct(case) * row + T * D * _SIZE[case["out"]]
        flops = T * D * (2.0 if case["table"] == "int8" else 1.0)
    elif op == "gradient":
        T, D = case["T"], case["D"]
        size = T * (8.0 + (1.0 - case["pad"]) * D * _SIZE[case["dtype"]]) + case["V"] * D * _SIZE[case["out"]]
        flops = (1.0 - case["pad"]) * T * D + case["V"] * D
    elif op in ("norm", "clip"):
        size = flops = 0.0
        for dtype, n in _specs(case):
            size += n * (0.5 + 4.0 / case["block"] if dtype == "int4" else _SIZE[dtype])
            flops += 2.0 * n
            if op == "clip":
                size += n * _SIZE[case["out"]]
                flops += n
        size += 4.0
    else:
        size = flops = 0.0
        for N, K in _shapes(case):
            size += N * K * (0.5 + 4.0 / case["block"]) + 2.0 * case["M"] * K + 4.0 * case["M"] * N
            flops += 2.0 * case["M"] * N * K
    return {"bytes": float(size), "flops": float(flops)}


# ---------------------------------------------------------------- in 64 bits

def _signed(packed, n):
    """The INT4 codes as doubles: two's complement halves of each byte."""
    out = torch.empty(packed.numel() * 2, dtype=torch.float64, device=DEV)
    for half in (0, 1):
        u = (packed.to(torch.int32) >> (4 * half)) & 15
        out[half::2] = (u - 16 * (u > 7)).double()
    return out[:n]


def _values64(packed, scales, n, block):
    return _signed(packed, n) * scales.double().repeat_interleave(block)[:n]


def _norm64(grads):
    total = 0.0
    for g in grads:
        if isinstance(g, tuple):
            g = _values64(*g)
        for part in g.split(1 << 26):
            total += float(part.double().square().sum())
    return math.sqrt(total)


def exact(case, seed):
    i, op = _inputs(case, seed), case["op"]
    if op == "embedding":
        ids, D, V = i["ids"], case["D"], case["V"]
        y = torch.zeros(case["T"], D, dtype=torch.float64, device=DEV)
        real = (ids >= 0).nonzero().view(-1)
        if case["table"] == "int8":
            cols = torch.arange(D, device=DEV)
            for part in real.split(4096):
                flat = (ids[part] * D).view(-1, 1) + cols
                y[part] = (torch.take(i["codes"], flat).double() * torch.take(i["scales"], flat // case["block"]).double()
                           * case["scale"])
        else:
            y[real] = i["table"].index_select(0, ids[real]).double() * case["scale"]
        return y
    if op == "gradient":
        # token by token in the order of the ids: running sums, and their differences where the id changes
        ids, dy = i["ids"], i["dy"]
        order = torch.argsort(ids, stable=True)
        order = order[ids[order] >= 0]
        dw = torch.zeros(case["V"], case["D"], dtype=torch.float64, device=DEV)
        if order.numel() == 0:
            return dw
        rows, counts = torch.unique_consecutive(ids[order], return_counts=True)
        ends = counts.cumsum(0) - 1
        for cols in torch.arange(case["D"], device=DEV).split(1024):
            run_ = dy[order][:, cols].double().cumsum(0)[ends]
            run_[1:] -= run_[:-1].clone()
            dw[rows[:, None], cols[None, :]] = run_ * case["scale"]
        return dw
    if op == "norm":
        return torch.tensor(_norm64(i["grads"]), dtype=torch.float64, device=DEV)
    if op == "clip":
        norm = _norm64(i["grads"]) * case["unscale"]
        c = min(1.0, 1.0 / (norm + 1e-6)) * case["unscale"]
        return torch.tensor(norm, dtype=torch.float64, device=DEV), torch.cat(
            [(_values64(*g) if isinstance(g, tuple) else g.double()) * c for g in i["grads"]])
    outs = []
    for x, packed, scales, N in i["products"]:
        K, parts = x.shape[1], []
        # some rows of the weight at a time, an even number, so that they start at a byte and (K % block == 0) a block
        step = 4096
        for n0 in range(0, N, step):
            n1 = min(N, n0 + step)
            codes = _signed(packed[n0 * K // 2: n1 * K // 2], (n1 - n0) * K)
            at = torch.arange(n0 * K, n1 * K, device=DEV) // case["block"]
            w = (codes * scales[at].double()).view(n1 - n0, K)
            parts.append(torch.mm(x.double(), w.t().contiguous()))
        outs.append(torch.cat(parts, 1))
    return outs
