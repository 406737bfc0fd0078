"""The performance cases of the query encoder's operators: what stands between tokens and the vectors that the index
is asked with, and the gradients that train it.

A case is a dict of plain values.  Its "op" says which calls one pass makes:
  embed         pqt_embed: scaled rows of an embedding table for n tokens
  embed_grad    pqt_embed_gradient: the table's gradient, summed over the places of every token
  norm          pqt_layer_norm: layer norm of every row
  norm_grad     pqt_layer_norm_gradient: the gradients of the input, the weight and the bias
  project       pqt_block_quantize + pqt_block_product: y = x W^T + bias, both in 8-bit blocks of 128
  project_step  the same as a training step: y, the input's and the weight's gradient
V rows of a table, d values of a row, n tokens or outputs, rows / m positions, k inputs of a product.
"pad": the rows of the inputs lie that many values further apart than they are long.
"""
import math

import numpy as np
import torch

own = False                      # False: the plain forms; True: the library's calls
DEVICE = torch.device("cuda", 0)
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 128
TOP = 448.0                      # largest e4m3 value
EPS = 1e-5


def listed():
    return [
        # one short query's tokens: latency is what counts
        {"name": "embed-query", "op": "embed", "n": 7, "V": 32768, "d": 1024, "type": "bf16", "out": "bf16", "ids": 64, "padding": 0.0, "pad": 0},
        # the tokens of a batch of passages, padded to one length, on their way into the index
        {"name": "embed-corpus", "op": "embed", "n": 100_003, "V": 100_000, "d": 1024, "type": "bf16", "out": "f32", "ids": 64, "padding": 0.05, "pad": 0},
        # a fine-tuning step on a few sentences, small table
        {"name": "embed-grad-few", "op": "embed_grad", "n": 333, "V": 8192, "d": 512, "type": "f32", "out": "f32", "ids": 64, "padding": 0.05, "pad": 0},
        # a training step's batch of tokens with natural frequencies: a few tokens hold much of it
        {"name": "embed-grad-batch", "op": "embed_grad", "n": 131_071, "V": 65_536, "d": 1024, "type": "bf16", "out": "f32", "ids": 64, "padding": 0.05, "pad": 0},
        # the benchmark's 10,000 queries of 128 floats, normalised before they are asked
        {"name": "norm-queries", "op": "norm", "rows": 10_000, "d": 128, "type": "f32", "out": "f32", "pad": 0},
        # a batch of 960 values a row inside a wider buffer, odd number of rows
        {"name": "norm-batch", "op": "norm", "rows": 65_537, "d": 960, "type": "bf16", "out": "bf16", "pad": 64},
        # backward of a batch of sentences
        {"name": "norm-grad-batch", "op": "norm_grad", "rows": 4097, "d": 1000, "type": "bf16", "out": "bf16", "pad": 0},
        # backward of a training step's batch at a wide model
        {"name": "norm-grad-wide", "op": "norm_grad", "rows": 16_384, "d": 4096, "type": "bf16", "out": "bf16", "pad": 0},
        # one position projected while a user waits: the weights are what is read
        {"name": "project-one", "op": "project", "m": 1, "k": 4096, "n": 4096, "type": "bf16", "out": "bf16", "bias": True, "pad": 0},
        # the benchmark's 10,000 queries brought to the index's 128 dimensions, as the floats that it takes
        {"name": "project-queries", "op": "project", "m": 10_000, "k": 1000, "n": 128, "type": "bf16", "out": "f32", "bias": True, "pad": 0},
        # a wide layer over a batch of passages
        {"name": "project-layer", "op": "project", "m": 16_384, "k": 4096, "n": 4096, "type": "bf16", "out": "bf16", "bias": False, "pad": 0},
        # a training step of a projection to 960 dimensions, ragged sizes
        {"name": "project-step", "op": "project_step", "m": 8191, "k": 2000, "n": 960, "type": "bf16", "out": "bf16", "bias": False, "pad": 0},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _length(rng, lo, hi):
    """A row's length: a power of two as most models have it, a multiple of 40, or odd."""
    v = _log_int(rng, lo, hi)
    return rng.choice((2 ** int(math.log2(v)), max(40, v // 40 * 40), v | 1))


def draw(rng):
    op = rng.choice(("embed", "embed_grad", "norm", "norm_grad", "project", "project", "project_step"))
    case = {"op": op, "type": rng.choice(("bf16", "bf16", "f32", "f16"))}
    case["out"] = rng.choice((case["type"], "f32")) if op in ("embed", "norm", "project") else "f32" if op == "embed_grad" else case["type"]
    case["pad"] = rng.choice((0, 0, 0, 8, 64, 5))
    if op in ("embed", "embed_grad"):
        case["d"] = _length(rng, 32, 4096)
        case["n"] = _log_int(rng, 1, min(131_071, 100_000_000 // case["d"]))
        case["V"] = _log_int(rng, 1000, min(131_071, 67_000_000 // case["d"]))
        case["ids"] = rng.choice((32, 64))
        case["padding"] = rng.choice((0.0, 0.05, 0.3))
        return case
    if op in ("norm", "norm_grad"):
        case["d"] = _length(rng, 32, 16_384)
        case["rows"] = _log_int(rng, 1, min(100_000, 33_000_000 // case["d"]))
        return case
    case["k"] = _length(rng, 64, 8192)
    case["n"] = _length(rng, 32, 8192)
    products = 250_000_000_000 if op == "project" else 15_000_000_000
    most = min(16_384, 60_000_000 // max(case["k"], case["n"]), products // (case["k"] * case["n"]))
    case["m"] = _log_int(rng, 1 if op == "project" else 64, max(64, most))
    case["bias"] = op == "project" and rng.random() < 0.5
    return case


# ---- inputs --------------------------------------------------------------------------------------------------------
def _normal(g, rows, cols, dtype, pad=0, scale=1.0):
    """Rows of activations: a few dimensions are many times as large as the others, as layers have them."""
    size = torch.exp(0.4 * torch.randn(cols, generator=g, device=DEVICE))
    size = torch.where(torch.rand(cols, generator=g, device=DEVICE) < 0.005, 20 * size, size) * scale
    wide = torch.empty(rows, cols + pad, dtype=dtype, device=DEVICE)
    step = max(1, (1 << 27) // (cols + pad))
    for s in range(0, rows, step):
        wide[s:s + step, :cols] = (torch.randn(min(step, rows - s), cols, generator=g, device=DEVICE) * size).to(dtype)
    wide[:, cols:] = 0
    return wide[:, :cols]


def _tokens(g, case):
    """Token ids with the frequencies of words (the r-th most frequent about 1 / r of the first), in any order of ids;
    -1 marks the places that pad a batch to one length."""
    n, V = case["n"], case["V"]
    rank = torch.exp(torch.rand(n, generator=g, device=DEVICE, dtype=torch.float64) * math.log(V + 1.0)).long() - 1
    ids = torch.randperm(V, generator=g, device=DEVICE)[rank.clamp_(0, V - 1)]
    ids = torch.where(torch.rand(n, generator=g, device=DEVICE) < case["padding"], torch.full_like(ids, -1), ids)
    return ids.to(torch.int32 if case["ids"] == 32 else torch.int64)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    op, dt, pad = case["op"], TYPES[case["type"]], case["pad"]
    s = {"case": case}
    if op == "embed":
        s["table"] = _normal(g, case["V"], case["d"], dt, pad, 0.02)
        s["tokens"] = _tokens(g, case)
        s["scale"] = math.sqrt(case["d"])
    elif op == "embed_grad":
        s["grad"] = _normal(g, case["n"], case["d"], dt, pad, 0.01)
        s["tokens"] = _tokens(g, case)
        s["scale"] = math.sqrt(case["d"])
    elif op in ("norm", "norm_grad"):
        x = _normal(g, case["rows"], case["d"], dt, pad)
        x += torch.randn(case["d"], generator=g, device=DEVICE).to(dt)
        s["x"] = x
        s["weight"] = (1 + 0.1 * torch.randn(case["d"], generator=g, device=DEVICE)).to(dt)
        s["bias"] = (0.1 * torch.randn(case["d"], generator=g, device=DEVICE)).to(dt)
        if op == "norm_grad":
            s["grad"] = _normal(g, case["rows"], case["d"], dt, pad, 0.01)
            s["mean"], s["rstd"] = _statistics(x)         # kept by the forward pass
    else:
        s["x"] = _normal(g, case["m"], case["k"], dt, pad)
        # the weights are cut into blocks once, when they are loaded or updated
        w = _normal(g, case["n"], case["k"], dt, 0, 1 / math.sqrt(case["k"]))
        s["w"] = _cut(w)
        s["bias"] = torch.randn(case["n"], generator=g, device=DEVICE) if case["bias"] else None
        if op == "project_step":
            s["wt"] = _cut(w.t())
            s["grad"] = _normal(g, case["m"], case["n"], dt, pad, 0.01)
    return s


# ---- the plain forms -----------------------------------------------------------------------------------------------
def _power(e):
    return ((e + 127) << 23).view(torch.float32)


def _cut(x):
    """8-bit blocks of 128 values along each row: (codes padded to whole blocks, scale bytes, values of a row)."""
    rows, k = x.shape
    blocks = -(-k // BLOCK)
    f = torch.zeros(rows, blocks * BLOCK, device=x.device)
    f[:, :k] = x
    f = f.view(rows, blocks, BLOCK)
    top = torch.where(torch.isfinite(f), f.abs(), 0.0).amax(2)
    part, e = torch.frexp(top / TOP)
    e = torch.where(part > 0.5, e, e - 1).clamp_(min=-126).to(torch.int32)
    codes = (f * _power(-e)[:, :, None]).to(torch.float8_e4m3fn).view(rows, blocks * BLOCK)
    return codes, (e + 127).to(torch.uint8), k


def _stand_for(blocks):
    """The values that 8-bit blocks stand for."""
    codes, scales, k = blocks
    f = codes.float().view(codes.shape[0], -1, BLOCK) * _power(scales.to(torch.int32) - 127)[:, :, None]
    return f.view(codes.shape[0], -1)[:, :k]


def _statistics(x):
    f = x.float()
    mean = f.mean(1)
    return mean, torch.rsqrt((f - mean[:, None]).square().mean(1) + EPS)


def _plain(s):
    case, op = s["case"], s["case"]["op"]
    out = TYPES[case["out"]]
    if op == "embed":
        tok = s["tokens"].long()
        y = s["table"][tok.clamp(min=0)].float() * s["scale"]
        return torch.where((tok >= 0)[:, None], y, 0.0).to(out)
    if op == "embed_grad":
        tok = s["tokens"].long()
        total = torch.zeros(case["V"] + 1, case["d"], device=DEVICE)           # the last row takes the padding
        total.index_add_(0, torch.where(tok >= 0, tok, case["V"]), s["grad"].float())
        return (total[:case["V"]] * s["scale"]).to(out)
    if op == "norm":
        mean, rstd = _statistics(s["x"])
        y = (s["x"].float() - mean[:, None]) * rstd[:, None] * s["weight"].float() + s["bias"].float()
        return y.to(out), mean, rstd
    if op == "norm_grad":
        grad = s["grad"].float()
        h = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        gw = grad * s["weight"].float()
        dx = s["rstd"][:, None] * (gw - gw.mean(1, keepdim=True) - h * (gw * h).mean(1, keepdim=True))
        return dx.to(out), (grad * h).sum(0), grad.sum(0)
    y = _stand_for(_cut(s["x"])) @ _stand_for(s["w"]).t()
    if s["bias"] is not None:
        y = y + s["bias"]
    if op == "project":
        return y.to(out)
    dx = _stand_for(_cut(s["grad"])) @ _stand_for(s["wt"]).t()
    dw = _stand_for(_cut(s["grad"].t())) @ _stand_for(_cut(s["x"].t())).t()
    return y.to(out), dx.to(out), dw


def run(s):
    if not own:
        return _plain(s)
    import paper_1702_05911_amd as pqt
    case, op = s["case"], s["case"]["op"]
    out = TYPES[case["out"]]
    if op == "embed":
        return pqt.pqt_embed(s["table"], s["tokens"], s["scale"], out_dtype=out)
    if op == "embed_grad":
        return pqt.pqt_embed_gradient(s["grad"], s["tokens"], case["V"], s["scale"], out_dtype=out)
    if op == "norm":
        return pqt.pqt_layer_norm(s["x"], s["weight"], s["bias"], EPS, out_dtype=out)
    if op == "norm_grad":
        return pqt.pqt_layer_norm_gradient(s["grad"], s["x"], s["weight"], s["mean"], s["rstd"])
    w = pqt.Blocks(*s["w"])
    if op == "project":
        return pqt.pqt_block_product(pqt.pqt_block_quantize(s["x"]), w, bias=s["bias"], out_dtype=out)
    x, xt = pqt.pqt_block_quantize(s["x"], columns=True)
    grad, gradt = pqt.pqt_block_quantize(s["grad"], columns=True)
    return (pqt.pqt_block_product(x, w, out_dtype=out), pqt.pqt_block_product(grad, pqt.Blocks(*s["wt"]), out_dtype=out),
            pqt.pqt_block_product(gradt, xt, out_dtype=torch.float32))


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def _distinct(n, V, padding):
    """Expected number of distinct tokens among n."""
    r = np.arange(1, V + 1, dtype=np.float64)
    p = np.log1p(1 / r) / math.log(V + 1.0)
    return float(np.sum(1 - np.exp(n * (1 - padding) * np.log1p(-p))))


def work(case):
    op, t, o = case["op"], SIZES[case["type"]], SIZES[case["out"]]
    if op == "embed":
        n, d = case["n"], case["d"]
        return {"bytes": n * case["ids"] / 8 + _distinct(n, case["V"], case["padding"]) * d * t + n * d * o, "flops": n * d}
    if op == "embed_grad":
        n, d = case["n"], case["d"]
        return {"bytes": n * case["ids"] / 8 + n * (1 - case["padding"]) * d * t + case["V"] * d * o, "flops": n * d}
    if op == "norm":
        rows, d = case["rows"], case["d"]
        return {"bytes": rows * d * (t + o) + 8 * rows + 2 * d * t, "flops": 8 * rows * d}
    if op == "norm_grad":
        rows, d = case["rows"], case["d"]
        return {"bytes": rows * d * (2 * t + o) + 8 * rows + d * (t + 8), "flops": 14 * rows * d}
    m, n, k = case["m"], case["n"], case["k"]
    weights = n * k * (1 + 1 / BLOCK)
    if op == "project":
        return {"bytes": m * k * t + weights + m * n * o + (4 * n if case["bias"] else 0), "flops": 2 * m * n * k}
    return {"bytes": m * (k + n) * t + 2 * weights + m * (n + k) * o + 4 * n * k, "flops": 6 * m * n * k}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------
def _blocks64(x):
    """Row by row, in blocks of 128: the nearest number of four significant bits (three below 2^-6) under the block's scale, the
    smallest power of two that brings its largest value to at most 448."""
    x = x.double()
    short = -x.shape[1] % 128
    x = torch.cat([x, x.new_zeros(x.shape[0], short)], 1) if short else x
    parts = x.unflatten(1, (-1, 128))
    largest = parts.abs().amax(2, keepdim=True)
    bits = torch.ceil(torch.log2(torch.clamp(largest, min=1e-60) / 448))
    bits = torch.where(448 * torch.exp2(bits - 1) >= largest, bits - 1, bits)          # the logarithm may be an ulp off
    bits = torch.where(448 * torch.exp2(bits) < largest, bits + 1, bits).clamp(min=-126)
    v = parts / torch.exp2(bits)
    octave = torch.frexp(v)[1].double() - 1
    unit = torch.exp2(octave.clamp(min=-6) - 3)
    v = torch.round(v / unit) * unit * torch.exp2(bits)
    return v.flatten(1)[:, :x.shape[1] - short]


def _values64(kept):
    codes, scales, k = kept
    return (codes.double() * torch.exp2(scales.double() - 127).repeat_interleave(128, 1))[:, :k]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "embed":
        y = s["table"].double()[s["tokens"].long()] * s["scale"]            # -1 reads the last row: cleared below
        y[s["tokens"] < 0] = 0
        return y
    if op == "embed_grad":
        keep = s["tokens"] >= 0
        ids, rows = s["tokens"][keep].long(), s["grad"][keep].double()
        return rows.new_zeros(case["V"], case["d"]).index_put_((ids,), rows, accumulate=True) * s["scale"]
    if op in ("norm", "norm_grad"):
        x, w, b = s["x"].double(), s["weight"].double(), s["bias"].double()
        mean = x.sum(1, keepdim=True) / case["d"]
        sigma = (((x - mean) ** 2).sum(1, keepdim=True) / case["d"] + EPS).sqrt()
        if op == "norm":
            return (x - mean) / sigma * w + b, mean[:, 0], 1 / sigma[:, 0]
        grad = s["grad"].double()
        mean, rstd = s["mean"].double()[:, None], s["rstd"].double()[:, None]    # the forward pass's own
        h = (x - mean) * rstd
        gw = grad * w
        return rstd * (gw - gw.sum(1, keepdim=True) / case["d"] - h * ((gw * h).sum(1, keepdim=True) / case["d"])), (grad * h).sum(0), grad.sum(0)
    x, w = _blocks64(s["x"]), _values64(s["w"])
    y = x @ w.t()
    if s["bias"] is not None:
        y += s["bias"].double()
    if op == "project":
        return y
    grad = s["grad"]
    return y, _blocks64(grad) @ _values64(s["wt"]).t(), _blocks64(grad.t()) @ _blocks64(s["x"].t()).t()
