"""The performance cases of the query encoder's layers: root-mean-square norm with the residual's addition, into 8-bit blocks or not, and
attention among the tokens of every text with a learned bias by the bucket of their distance; each with its gradient.

A case is a dict of plain values.  Its "op" says which calls one pass makes:
  norm          pqt_rms_norm: h = x + residual, y = h / rms(h) * weight
  norm_project  pqt_rms_norm into 8-bit blocks of 128, and pqt_block_product on them: the projection behind the norm
  norm_grad     pqt_rms_norm_gradient: the gradient of h, with what arrives along the residual's way, and the weight's
  attend        pqt_attention: softmax(scale q k^T + bias) v for every head of every text
  attend_grad   pqt_attention_gradient: the gradients of q, k, v and of the bias
rows of d values for the norms, n outputs of the projection.  Attention: `texts` of up to `longest` tokens (the lengths are spread evenly below
that; of sixteen or more one is empty and one has a single token), one behind the other, or padded to one length; `behind` rows after the last one that no text
has; `heads` of d values, `kv` of them for keys and values; `buckets` of distances up to `far` (0: no bias).
"pad": the rows of the inputs lie that many values further apart than they are long.
"""
import math

import torch

own = False                      # False: the plain forms; True: the library's calls
DEVICE = torch.device("cuda", 0)
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 128
TOP = 448.0                      # largest e4m3 value
EPS = 1e-6
FAR = 128                        # distances from there on share the last buckets


def _texts(name, op, texts, longest, heads, kv, d, kind, buckets=32, padded=False, behind=0, pad=0):
    return {"name": name, "op": op, "texts": texts, "longest": longest, "heads": heads, "kv": kv, "d": d, "type": kind, "buckets": buckets, "padded": padded,
            "behind": behind, "pad": pad}


def listed():
    return [
        # one short query's tokens between two sub-layers: latency is what counts
        {"name": "norm-query", "op": "norm", "rows": 7, "d": 1024, "type": "bf16", "residual": True, "pad": 0},
        # the tokens of a batch of passages on their way into the index, inside a wider buffer
        {"name": "norm-corpus", "op": "norm", "rows": 100_003, "d": 960, "type": "bf16", "residual": True, "pad": 64},
        # the last norm of a batch of passages and the projection to the index's 128 dimensions
        {"name": "norm-project", "op": "norm_project", "rows": 16_385, "d": 2000, "n": 128, "type": "bf16", "residual": True, "pad": 0},
        # backward of a fine-tuning step on a few sentences
        {"name": "norm-grad-few", "op": "norm_grad", "rows": 333, "d": 512, "type": "f32", "residual": True, "pad": 0},
        # backward of a training step's batch
        {"name": "norm-grad-batch", "op": "norm_grad", "rows": 32_768, "d": 2048, "type": "bf16", "residual": True, "pad": 0},
        # one short query: latency
        _texts("attend-query", "attend", 1, 7, 16, 16, 64, "bf16"),
        # a batch of short queries, one behind the other, in a buffer with room for more
        _texts("attend-queries", "attend", 4096, 32, 16, 16, 64, "bf16", behind=100),
        # passages on their way into the index, padded to one length
        _texts("attend-passages", "attend", 512, 256, 12, 12, 64, "bf16", padded=True),
        # one long document, shared key heads
        _texts("attend-document", "attend", 1, 8191, 16, 4, 128, "bf16"),
        # a fine-tuning step on a few sentences in fp32
        _texts("attend-grad-few", "attend_grad", 8, 48, 8, 8, 64, "f32"),
        # a training step on passages
        _texts("attend-grad-passages", "attend_grad", 64, 512, 16, 16, 64, "bf16"),
        # a training step on documents, shared key heads of 80 values
        _texts("attend-grad-documents", "attend_grad", 2, 4001, 8, 2, 80, "f16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _row(rng, lo, hi):
    """A row's length: a power of two as most models have it, a multiple of 40, or odd."""
    v = _log_int(rng, lo, hi)
    return rng.choice((2 ** int(math.log2(v)), max(40, v // 40 * 40), v | 1))


def draw(rng):
    op = rng.choice(("norm", "norm_project", "norm_grad", "attend", "attend", "attend", "attend_grad", "attend_grad"))
    case = {"op": op, "type": rng.choice(("bf16", "bf16", "f32", "f16")), "pad": rng.choice((0, 0, 0, 8, 64, 5))}
    if op in ("norm", "norm_project", "norm_grad"):
        case["d"] = _row(rng, 32, 8192)
        case["rows"] = _log_int(rng, 1, min(100_000, 90_000_000 // case["d"]))
        case["residual"] = rng.random() < 0.75
        if op == "norm_project":
            case["n"] = rng.choice((96, 128, 960, _log_int(rng, 32, 1024)))
            case["rows"] = min(case["rows"], 16_385)
        return case
    case["d"] = rng.choice((32, 64, 64, 80, 128, _log_int(rng, 8, 128)))
    case["heads"] = rng.choice((1, 4, 8, 12, 16))
    case["kv"] = rng.choice([k for k in (case["heads"], case["heads"], case["heads"] // 2, case["heads"] // 4, 1) if k and case["heads"] % k == 0])
    case["buckets"] = rng.choice((0, 32, 32, 64, 20))
    case["longest"] = _log_int(rng, 1, 8191 if op == "attend" else 4001)
    # what the plain forms hold: a square of numbers for every head of every text
    square = case["heads"] * case["longest"] ** 2 * (4 if case["type"] == "f32" else 1)
    most = min(4096, max(1, 400_000_000 // square), 131_072 // case["longest"])
    case["texts"] = _log_int(rng, 1, max(1, most))
    case["padded"] = rng.random() < 0.4
    case["behind"] = 0 if case["padded"] else rng.choice((0, 0, 1, 100))
    return case


# ---- inputs --------------------------------------------------------------------------------------------------------
def _normal(g, rows, cols, dtype, pad=0, scale=1.0, few=0.005):
    """Rows of activations: dimensions of different sizes, of which a few are many times as large as the others, as layers have them."""
    size = torch.exp(0.4 * torch.randn(cols, generator=g, device=DEVICE))
    size = torch.where(torch.rand(cols, generator=g, device=DEVICE) < few, 20 * size, size) * scale
    wide = torch.empty(rows, cols + pad, dtype=dtype, device=DEVICE)
    step = max(1, (1 << 27) // (cols + pad))
    for s in range(0, rows, step):
        wide[s:s + step, :cols] = (torch.randn(min(step, rows - s), cols, generator=g, device=DEVICE) * size).to(dtype)
    wide[:, cols:] = 0
    return wide[:, :cols]


def _lengths(case):
    texts, longest = case["texts"], case["longest"]
    out = [max(1, round(longest * (0.15 + 0.85 * (s + 1) / texts))) for s in range(texts)]
    if texts >= 16:
        out[0], out[1] = 0, 1
    return out


def _bucket(distance, buckets, far):
    """The usual buckets of distances: half of them for keys behind the query; of each half one for every distance below its half, then ever wider ones up to
    `far`.  Whole numbers only: the border of step t lies where (distance / near)^rest reaches (far / near)^t."""
    half = buckets // 2
    away, near = abs(distance), half // 2
    rest = half - near
    if away < near or near == 0:
        own_bucket = min(away, half - 1)
    else:
        t = 0
        while t < rest - 1 and away ** rest * near ** (t + 1) >= far ** (t + 1) * near ** rest:
            t += 1
        own_bucket = near + t
    return own_bucket + (half if distance > 0 else 0)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    op, dt, pad, d = case["op"], TYPES[case["type"]], case["pad"], case["d"]
    s = {"case": case}
    if op in ("norm", "norm_project", "norm_grad"):
        x = _normal(g, case["rows"], d, dt, pad)
        s["weight"] = (1 + 0.1 * torch.randn(d, generator=g, device=DEVICE)).to(dt)
        if op == "norm_grad":
            s["h"] = x                                       # kept by the forward pass, as rstd is
            s["rstd"] = torch.rsqrt(x.float().square().mean(1) + EPS)
            s["grad"] = _normal(g, case["rows"], d, dt, pad, 0.01)
            s["through"] = _normal(g, case["rows"], d, dt, pad, 0.01) if case["residual"] else None
            return s
        s["x"] = x
        s["residual"] = _normal(g, case["rows"], d, dt, pad, 4.0) if case["residual"] else None
        if op == "norm_project":
            s["w"] = _cut(_normal(g, case["n"], d, dt, 0, 1 / math.sqrt(d)))       # the weights are cut into blocks once
        return s
    heads, kv, texts, longest = case["heads"], case["kv"], case["texts"], case["longest"]
    lengths = torch.tensor(_lengths(case), device=DEVICE)[torch.randperm(texts, generator=g, device=DEVICE)]
    if case["padded"]:
        s["starts"] = torch.arange(texts + 1, device=DEVICE) * longest
        s["lengths"] = lengths
        n = texts * longest
    else:
        s["starts"] = torch.cat([lengths.new_zeros(1), lengths.cumsum(0)])
        s["lengths"] = None
        n = sum(_lengths(case)) + case["behind"]
    qkv = _normal(g, n, (heads + 2 * kv) * d, dt, pad, 1.0, 0.0)                   # a fused projection's result
    s["q"], s["k"], s["v"] = qkv[:, :heads * d], qkv[:, heads * d:(heads + kv) * d], qkv[:, (heads + kv) * d:]
    s["scale"] = 1 / math.sqrt(d)
    s["bias"] = s["distances"] = None
    if case["buckets"]:
        s["bias"] = torch.randn(heads, case["buckets"], generator=g, device=DEVICE)
        s["distances"] = torch.tensor([_bucket(t, case["buckets"], FAR) for t in range(-FAR, FAR + 1)], dtype=torch.int32, device=DEVICE)
    if op == "attend_grad":
        s["out"], s["lse"] = _attend(s)                      # kept by the forward pass
        s["grad"] = _normal(g, n, heads * d, dt, pad, 0.01)
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


def _places(s):
    """(row of every place of every text, whether a token is there): texts x longest."""
    case = s["case"]
    at = torch.arange(case["longest"], device=DEVICE)
    lengths = s["lengths"] if s["lengths"] is not None else s["starts"][1:] - s["starts"][:-1]
    there = at[None, :] < lengths[:, None]
    return torch.where(there, s["starts"][:-1, None] + at[None, :], 0), there


def _split(x, rows, there, heads):
    """texts x heads x longest x d in fp32, zeros where no token is."""
    f = torch.where(there[:, :, None], x[rows].float(), 0.0)
    return f.unflatten(2, (heads, -1)).transpose(1, 2).contiguous()


def _join(y, rows, there, n):
    """The reverse of _split: n rows, zeros where no token is."""
    out = torch.zeros(n, y.shape[1] * y.shape[3], device=DEVICE)
    out[rows[there]] = y.transpose(1, 2).flatten(2)[there]
    return out


def _bucket_of_places(s):
    at = torch.arange(s["case"]["longest"], device=DEVICE)
    return s["distances"][(at[None, :] - at[:, None]).clamp(-FAR, FAR) + FAR].long()


def _logits(s, q, k, there):
    """Scaled products of the queries and keys plus the bias, -inf where no key is."""
    z = (q @ k.transpose(2, 3)).mul_(s["scale"])
    if s["bias"] is not None:
        z += s["bias"][:, _bucket_of_places(s)]
    return z.masked_fill_(~there[:, None, None, :], -math.inf)


def _attend(s):
    case, n = s["case"], s["q"].shape[0]
    heads, group = case["heads"], case["heads"] // case["kv"]
    rows, there = _places(s)
    k = _split(s["k"], rows, there, case["kv"]).repeat_interleave(group, 1)
    v = _split(s["v"], rows, there, case["kv"]).repeat_interleave(group, 1)
    z = _logits(s, _split(s["q"], rows, there, heads), k, there)
    top = z.amax(3, keepdim=True).clamp_(min=-1e30)                       # (texts without tokens)
    z = z.sub_(top).exp_()
    total = z.sum(3, keepdim=True)
    out = _join((z @ v) / total.clamp(min=1e-30), rows, there, n)
    lse = torch.full((heads, n), -math.inf, device=DEVICE)
    lse[:, rows[there]] = (top + total.log())[..., 0].transpose(1, 2)[there].t()
    return out.to(s["q"].dtype), lse


def _attend_gradient(s):
    case, n, dt = s["case"], s["q"].shape[0], s["q"].dtype
    heads, kv = case["heads"], case["kv"]
    group = heads // kv
    rows, there = _places(s)
    q, grad = _split(s["q"], rows, there, heads), _split(s["grad"], rows, there, heads)
    k = _split(s["k"], rows, there, kv).repeat_interleave(group, 1)
    v = _split(s["v"], rows, there, kv).repeat_interleave(group, 1)
    lse = torch.where(there[:, None, :], s["lse"][:, rows].transpose(0, 1), math.inf)[..., None]        # places without a token: no weights
    p = _logits(s, q, k, there).sub_(lse).exp_()
    dv = (p.transpose(2, 3) @ grad).unflatten(1, (kv, group)).sum(2)
    delta = (grad * _split(s["out"], rows, there, heads)).sum(3, keepdim=True)
    dz = (grad @ v.transpose(2, 3)).sub_(delta).mul_(p)
    del p
    dq = (dz @ k).mul_(s["scale"])
    dk = (dz.transpose(2, 3) @ q).mul_(s["scale"]).unflatten(1, (kv, group)).sum(2)
    results = _join(dq, rows, there, n).to(dt), _join(dk, rows, there, n).to(dt), _join(dv, rows, there, n).to(dt)
    if s["bias"] is None:
        return results
    # sums along the diagonals: rows in reverse order, one place further to the right each
    longest = case["longest"]
    wide = torch.zeros(heads, longest, 2 * longest, dtype=torch.float64, device=DEVICE)
    wide[:, :, :longest] = dz.sum(0, dtype=torch.float64).flip(1)
    along = wide.flatten(1)[:, :longest * (2 * longest - 1)].unflatten(1, (longest, -1)).sum(1)
    bucket = s["distances"][torch.arange(1 - longest, longest, device=DEVICE).clamp(-FAR, FAR) + FAR].long()
    return results + (torch.zeros(heads, case["buckets"], dtype=torch.float64, device=DEVICE).index_add_(1, bucket, along).float(),)


def _plain(s):
    op = s["case"]["op"]
    if op == "attend":
        return _attend(s)
    if op == "attend_grad":
        return _attend_gradient(s)
    w = s["weight"].float()
    if op == "norm_grad":
        h, grad, rstd = s["h"].float(), s["grad"].float(), s["rstd"][:, None]
        z = h * rstd
        gw = grad * w
        dh = rstd * (gw - z * (gw * z).mean(1, keepdim=True))
        if s["through"] is not None:
            dh = dh + s["through"].float()
        return dh.to(s["h"].dtype), (grad * z).sum(0)
    h = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(s["x"].dtype)
    f = h.float()
    rstd = torch.rsqrt(f.square().mean(1) + EPS)
    y = f * rstd[:, None] * w
    if op == "norm":
        return y.to(h.dtype), h, rstd
    return (_stand_for(_cut(y)) @ _stand_for(s["w"]).t()).to(h.dtype), h, rstd


def run(s):
    if not own:
        return _plain(s)
    import paper_1702_05911_amd as pqt
    op = s["case"]["op"]
    if op == "norm":
        return pqt.pqt_rms_norm(s["x"], s["weight"], s["residual"], EPS)
    if op == "norm_project":
        y, h, rstd = pqt.pqt_rms_norm(s["x"], s["weight"], s["residual"], EPS, blocks=True)
        return pqt.pqt_block_product(y, pqt.Blocks(*s["w"]), out_dtype=h.dtype), h, rstd
    if op == "norm_grad":
        return pqt.pqt_rms_norm_gradient(s["grad"], s["h"], s["weight"], s["rstd"], s["through"])
    layout = dict(heads=s["case"]["heads"], scale=s["scale"], bias=s["bias"], distances=s["distances"], lengths=s["lengths"])
    if op == "attend":
        return pqt.pqt_attention(s["q"], s["k"], s["v"], s["starts"], **layout)
    dq, dk, dv, dbias = pqt.pqt_attention_gradient(s["grad"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["starts"], **layout)
    return (dq, dk, dv) if dbias is None else (dq, dk, dv, dbias)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def work(case):
    op, t, d = case["op"], SIZES[case["type"]], case["d"]
    if op in ("norm", "norm_project", "norm_grad"):
        rows = case["rows"]
        if op == "norm_grad":
            return {"bytes": rows * d * t * (4 if case["residual"] else 3) + 4 * rows + d * (t + 4), "flops": 12 * rows * d}
        kept = 2 if case["residual"] else 0                  # the residual read, h written
        if op == "norm":
            return {"bytes": rows * d * t * (2 + kept) + 4 * rows + d * t, "flops": 6 * rows * d}
        n = case["n"]
        return {"bytes": rows * d * t * (1 + kept) + 4 * rows + d * t + n * d * (1 + 1 / BLOCK) + rows * n * t, "flops": 2 * rows * d * n + 6 * rows * d}
    lengths = _lengths(case)
    tokens, pairs = sum(lengths), sum(x * x for x in lengths)
    n = case["texts"] * case["longest"] if case["padded"] else tokens + case["behind"]
    heads, kv = case["heads"], case["kv"]
    if op == "attend":
        return {"bytes": tokens * d * t * (heads + 2 * kv) + n * heads * (d * t + 4), "flops": 4 * pairs * d * heads}
    return {"bytes": tokens * (d * t * (3 * heads + 2 * kv) + 4 * heads) + n * d * t * (heads + 2 * kv), "flops": 10 * pairs * d * heads}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------
def _blocks64(x):
    """Row by row, in blocks of 128: the nearest number of four significant bits (three below 2^-6) under the block's scale, the
    smallest power of two that brings its largest value to at most 448."""
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


def _attend64(s, gradient):
    """Head by head over texts padded to the longest one; a place without a token is a key that no query sees and a query that nobody asks for."""
    case, n, d, longest = s["case"], s["q"].shape[0], s["case"]["d"], s["case"]["longest"]
    first = s["starts"][:-1]
    length = s["starts"].diff() if s["lengths"] is None else s["lengths"]
    place = torch.arange(longest, device=DEVICE)
    token = place < length[:, None]
    row = (first[:, None] + place)[token]
    away = place - place[:, None]
    group = case["heads"] // case["kv"]

    def rows_of(x, head):
        y = torch.zeros(len(first), longest, d, dtype=torch.float64, device=DEVICE)
        y[token] = x[row, head * d:(head + 1) * d].double()
        return y

    def put(to, head, y):
        to[row, head * d:(head + 1) * d] += y[token]

    zeros = lambda heads: torch.zeros(n, heads * d, dtype=torch.float64, device=DEVICE)  # noqa: E731
    out, dq, dk, dv = zeros(case["heads"]), zeros(case["heads"]), zeros(case["kv"]), zeros(case["kv"])
    lse = torch.full((case["heads"], n), -math.inf, dtype=torch.float64, device=DEVICE)
    dbias = torch.zeros(case["heads"], max(1, case["buckets"]), dtype=torch.float64, device=DEVICE)
    for head in range(case["heads"]):
        q, k, v = rows_of(s["q"], head), rows_of(s["k"], head // group), rows_of(s["v"], head // group)
        z = torch.bmm(q, k.transpose(1, 2).contiguous()) * s["scale"]
        if s["bias"] is not None:
            bucket = s["distances"].long()[away.clamp(-FAR, FAR) + FAR]
            z += s["bias"][head].double()[bucket]
        z[~token[:, None, :].expand_as(z)] = -math.inf
        if not gradient:
            share = torch.logsumexp(z, 2)
            p = torch.exp(z - share.clamp(min=-1e300)[:, :, None])
            put(out, head, torch.bmm(p, v))
            lse[head, row] = share[token]
            continue
        kept = torch.full((len(first), longest), math.inf, dtype=torch.float64, device=DEVICE)
        kept[token] = s["lse"][head, row].double()
        p = torch.exp(z - kept[:, :, None])
        g = rows_of(s["grad"], head)
        ds = p * (torch.bmm(g, v.transpose(1, 2).contiguous()) - (g * rows_of(s["out"], head)).sum(2, keepdim=True))
        put(dq, head, torch.bmm(ds, k) * s["scale"])
        put(dk, head // group, torch.bmm(ds.transpose(1, 2).contiguous(), q) * s["scale"])
        put(dv, head // group, torch.bmm(p.transpose(1, 2).contiguous(), g))
        if s["bias"] is not None:
            over = ds.sum(0)
            for b in range(case["buckets"]):
                dbias[head, b] = over[bucket == b].sum()
    if not gradient:
        return out, lse
    return (dq, dk, dv) if s["bias"] is None else (dq, dk, dv, dbias)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("attend", "attend_grad"):
        return _attend64(s, op == "attend_grad")
    w = s["weight"].double()
    if op == "norm_grad":
        h, grad, rstd = s["h"].double(), s["grad"].double(), s["rstd"].double()[:, None]      # the forward pass's own
        inner = (grad * w * h).sum(1, keepdim=True) / case["d"]
        dh = rstd * grad * w - h * rstd ** 3 * inner
        if s["through"] is not None:
            dh += s["through"].double()
        return dh, (grad * h * rstd).sum(0)
    h = s["x"].double()
    if s["residual"] is not None:
        h = (h + s["residual"].double()).to(s["x"].dtype).double()          # the norm is that of the sum as it is kept
    rms = (h.square().sum(1, keepdim=True) / case["d"] + EPS).sqrt()
    y = h / rms * w
    if op == "norm_project":
        y = _blocks64(y) @ _values64(s["w"]).t()
    return y, h, 1 / rms[:, 0]
