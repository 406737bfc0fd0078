"""The query encoder's layers against their definitions in 64 bits: root-mean-square norm with the residual's addition and its gradient, attention with
a bias by the bucket of distances and its gradient.

Tolerances follow from the arithmetic, U = 2^-24 the unit of fp32: a sum of c terms in any order is off by at most c U times the sum of their magnitudes, a
stored result, and a weight that is rounded to be multiplied, by its type's unit; an exponential by what its argument is off.  The references run in float64."""
import math
import os
import types

import pytest
import torch

from paper_1702_05911_amd import buildlib

if not os.path.exists(buildlib.OUTPUT):
    buildlib.build_library()
import paper_1702_05911_amd.binding as pqt  # noqa: E402

gpu = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}
INF = float("inf")


def dev():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: no silent fallback")
    return torch.device("cuda", 0)


def normal(shape, dtype, seed, pad=0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    wide = torch.zeros(shape[0], shape[1] + pad, dtype=dtype)
    wide[:, :shape[1]] = (torch.randn(shape, generator=g) * scale).to(dtype)
    return wide.to(dev())[:, :shape[1]]


def within(got, want, tol, what):
    """|got - want| <= tol + the rounding of the stored type, element by element; infinities are equal, and stand for what the type does not hold."""
    t = got.dtype
    got, want = got.double(), want.to(got.device)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    tol = tol + want.abs() * UNIT[t] * (1 + 2.0 ** -6) + LEAST[t]
    beyond = (want.abs() + tol > torch.finfo(t).max) & got.isinf() & (got * want > 0)
    bad = ~(((got - want).abs() <= tol) | (got == want) | beyond)
    if bad.any():
        i = tuple(int(v) for v in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} values off, first at {i}: {got[i]} for {want[i]}, tolerance {tol[i]}")


def guarded(rows, cols, dtype, pad=3):
    """An output inside a wider buffer, and a check that nothing outside it was written."""
    wide = torch.full((rows + 2, cols + 2 * pad), 7.0, dtype=dtype, device=dev())
    view = wide[1:1 + rows, pad:pad + cols]

    def check():
        keep = wide.clone()
        keep[1:1 + rows, pad:pad + cols] = 7.0
        assert bool((keep == 7.0).all()), "written outside the output"
    return view, check


# ---- root-mean-square norm -------------------------------------------------------------------------------------------
NORM = [  # rows, D, type, y's type, weight's type, residual, pad
    (1, 1, "f32", "f32", "f32", True, 0), (1, 7, "bf16", "bf16", "bf16", False, 3), (7, 1024, "bf16", "bf16", "bf16", True, 0), (333, 63, "f16", "f32", "f32", True, 1),
    (64, 64, "f32", "bf16", "f16", False, 0), (129, 65, "bf16", "f32", "bf16", True, 5), (5, 127, "f16", "f16", "f16", True, 0), (40, 257, "f32", "f32", None, True, 8),
    (301, 960, "bf16", "bf16", "f32", True, 64), (17, 2048, "f16", "bf16", "bf16", True, 0), (9, 2049, "bf16", "f16", None, False, 3), (5, 4097, "f32", "f16", "f32", True, 0),
    (3, 8200, "bf16", "bf16", "bf16", True, 1), (2, 16385, "f32", "f32", "f32", True, 0), (2, 32768, "bf16", "f32", "f32", True, 0), (4099, 40, "bf16", "bf16", "bf16", True, 0)]


def norm_inputs(rows, D, kind, weight, residual, pad):
    x, r = normal((rows, D), TYPES[kind], rows + D, pad), normal((rows, D), TYPES[kind], rows + D + 1, pad, 3.0) if residual else None
    w = (1 + 0.3 * normal((1, D), torch.float32, D + 5)[0]).to(TYPES[weight]).contiguous() if weight else None
    return x, r, w


def norm_reference(h, w, eps):
    """(y, relative error of y before it is stored, rstd): the sum of D squares and eps is off by (D + 2) U of itself, its root by half of that and a unit."""
    D = h.shape[1]
    h = h.double()
    rstd = 1 / (h.square().mean(1) + eps).sqrt()
    y = h * rstd[:, None]
    return y * w.double() if w is not None else y, (D / 2 + 8) * U, rstd


@gpu
@pytest.mark.parametrize("rows,D,kind,out,weight,residual,pad", NORM)
def test_rms_norm(rows, D, kind, out, weight, residual, pad):
    x, r, w = norm_inputs(rows, D, kind, weight, residual, pad)
    view, check = guarded(rows, D, TYPES[out])
    y, h, rstd = pqt.pqt_rms_norm(x, w, r, 1e-6, out=view)
    assert y is view and (h is x if r is None else h.is_contiguous())
    if r is not None:
        assert torch.equal(h, (x.float() + r.float()).to(x.dtype))
    want, rel, want_rstd = norm_reference(h, w, 1e-6)
    within(y, want, want.abs() * rel, "y")
    within(rstd, want_rstd, want_rstd * rel, "rstd")
    check()
    again = pqt.pqt_rms_norm(x, w, r, 1e-6, out_dtype=TYPES[out])
    assert torch.equal(again[0], y) and torch.equal(again[2], rstd)
    # in blocks: each value is the nearest e4m3 number under the smallest power of two with its block's largest at most 448
    blocks, h2, rstd2 = pqt.pqt_rms_norm(x, w, r, 1e-6, blocks=True)
    assert torch.equal(h2, h)
    within(rstd2, want_rstd, want_rstd * rel, "rstd beside blocks")
    kb = -(-D // 128)
    assert blocks.codes.shape == (rows, kb * 128) and blocks.scales.shape == (rows, kb) and blocks.cols == D
    scale = torch.exp2(blocks.scales.double() - 127)
    values = blocks.codes.double().view(rows, kb, 128) * scale[:, :, None]
    padded = torch.zeros(rows, kb * 128, dtype=torch.float64, device=dev())
    padded[:, :D] = want
    padded = padded.view(rows, kb, 128)
    top = padded.abs().amax(2)
    assert bool((top <= 448 * scale * (1 + rel)).all()) and bool(((top > 224 * scale * (1 - rel)) | (blocks.scales == 1)).all())
    step = torch.maximum(padded.abs() * 2.0 ** -4, scale[:, :, None] * 2.0 ** -10)              # half a step: four significant bits, or 2^-9 below 2^-6
    assert bool(((values - padded).abs() <= step * (1 + 16 * rel) + padded.abs() * rel).all())
    assert not bool(blocks.codes.view(torch.uint8).view(rows, -1)[:, D:].any())


@gpu
def test_rms_norm_special_rows():
    """Zeros, a NaN, an infinity, values whose squares are beyond fp32: as the formula in fp32 has it, each in its own row."""
    D = 300
    x = normal((6, D), torch.float32, 1)
    x[0] = 0
    x[1, 5] = float("nan")
    x[2, 7] = INF
    x[3] = 2.0 ** -70                                              # squares below fp32: eps decides
    x[4] = 1e30
    y, h, rstd = pqt.pqt_rms_norm(x, eps=1e-6)
    assert not bool(y[0].any()) and bool(y[1].isnan().all()) and bool(rstd[1].isnan())
    assert float(rstd[2]) == 0 and bool(y[2, 7].isnan()) and not bool(y[2, :7].any())
    within(y[3:4], x[3:4].double() * 1e3, x[3:4].double() * 1e3 * 8 * U, "tiny")
    assert not bool(y[4].any())
    want, rel, _ = norm_reference(x[5:], None, 1e-6)
    within(y[5:], want, want.abs() * rel, "the row beside them")
    blocks, _, _ = pqt.pqt_rms_norm(x, eps=1e-6, blocks=True)
    codes = blocks.codes.view(torch.uint8)
    assert bool((codes[1, :D] == 0x7f).all()) and int(codes[2, 7]) == 0x7f and not bool((codes[2, :7] & 0x7f).any()) and not bool(codes[:, D:].any())
    zero, _, rstd0 = pqt.pqt_rms_norm(torch.zeros((2, 77), device=dev()), eps=0.0, blocks=True)   # 0 * inf past the row's end is no value of it
    assert bool(rstd0.isinf().all()) and not bool(zero.codes.view(torch.uint8)[:, 77:].any())


@gpu
def test_rms_norm_of_nothing():
    x = torch.zeros((0, 48), dtype=torch.bfloat16, device=dev())
    y, h, rstd = pqt.pqt_rms_norm(x, None, x)
    assert y.shape == h.shape == (0, 48) and rstd.shape == (0,)
    assert pqt.pqt_rms_norm(x, blocks=True)[0].codes.shape == (0, 128)
    dx, dw = pqt.pqt_rms_norm_gradient(x, x, None, rstd, x)
    assert dx.shape == (0, 48) and dw.shape == (48,) and not bool(dw.any())


def norm_gradient_reference(grad, h, w, rstd, through):
    """(dx, its tolerance, dweight, its tolerance)."""
    rows, D = h.shape
    G, H, R = grad.double(), h.double(), rstd.double()[:, None]
    z = H * R
    g = G * w.double() if w is not None else G
    s = (g * z).mean(1, keepdim=True)
    dx = R * (g - z * s)
    tol = R * (g.abs() * 4 + z.abs() * (g * z).abs().mean(1, keepdim=True) * (D + 8)) * U
    if through is not None:
        dx = dx + through.double()
        tol = tol + (dx.abs() + through.double().abs()) * 2 * U
    return dx, tol, (G * z).sum(0), (G * z).abs().sum(0) * (rows + 4) * U


@gpu
@pytest.mark.parametrize("rows,D,kind,out,weight,residual,pad", NORM + [(1, 16384, "f16", "f16", "f16", True, 0), (3, 8193, "f32", "f32", "f32", True, 3), (130, 16390, "bf16", "bf16", "f32", True, 0),
                                                                       (600, 1000, "bf16", "bf16", "bf16", True, 0)])
def test_rms_norm_gradient(rows, D, kind, out, weight, residual, pad):
    h, through, w = norm_inputs(rows, D, kind, weight, residual, pad)
    grad = normal((rows, D), TYPES[kind], 9, pad, 0.1)
    _, _, rstd = pqt.pqt_rms_norm(h, w)
    view, check = guarded(rows, D, TYPES[kind])
    dx, dw = pqt.pqt_rms_norm_gradient(grad, h, w, rstd, through, out=view)
    want, tol, want_w, tol_w = norm_gradient_reference(grad, h, w, rstd, through)
    within(dx, want, tol, "dx")
    within(dw, want_w, tol_w, "dweight")
    check()
    again = pqt.pqt_rms_norm_gradient(grad, h, w, rstd, through)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)


@gpu
def test_rms_norm_gradient_by_differences():
    """f = <y, c> + <h, t> of x and of the residual, along random directions, by central differences of the 64-bit formula at the kernel's point."""
    rows, D = 5, 96
    x, r, w = normal((rows, D), torch.float32, 1), normal((rows, D), torch.float32, 2), 1 + 0.2 * normal((1, D), torch.float32, 3)[0]
    c, t = normal((rows, D), torch.float32, 4), normal((rows, D), torch.float32, 5)
    _, h, rstd = pqt.pqt_rms_norm(x, w, r)
    dx, dw = pqt.pqt_rms_norm_gradient(c, h, w, rstd, t)

    def f(X, R, W):
        H = X + R
        return float((H / (H.square().mean(1, keepdim=True) + 1e-6).sqrt() * W * c.double()).sum() + (H * t.double()).sum())
    X, R, W, e = x.double(), r.double(), w.double(), 1e-4
    for seed in range(3):
        a, b = normal((rows, D), torch.float32, 20 + seed).double(), normal((1, D), torch.float32, 30 + seed)[0].double()
        # differences of a function of size ~1e2 with third derivatives of that size: 1e2 e^2, and 1e-13 / e of rounding; kernels 1e2 D U
        for got, want in (((dx.double() * a).sum(), (f(X + e * a, R, W) - f(X - e * a, R, W)) / (2 * e)), ((dx.double() * a).sum(), (f(X, R + e * a, W) - f(X, R - e * a, W)) / (2 * e)),
                          ((dw.double() * b).sum(), (f(X, R, W + e * b) - f(X, R, W - e * b)) / (2 * e))):
            assert abs(float(got) - want) <= 1e-3, (float(got), want)


# ---- attention -------------------------------------------------------------------------------------------------------
def attention_inputs(lengths, heads, kv, d, kind, buckets=32, reach=128, padded=0, pad=0, ids=64, behind=0, seed=0, before=0):
    """q, k, v as slices of one buffer, NaN where no token is; starts, lengths; bias and distances."""
    wide = (heads + 2 * kv) * d
    spans = [padded] * len(lengths) if padded else lengths
    n = before + sum(spans) + behind
    qkv = torch.full((n, wide + pad), float("nan"), dtype=TYPES[kind], device=dev())
    starts = [before]
    for s in spans:
        starts.append(starts[-1] + s)
    for i, (at, m) in enumerate(zip(starts, lengths)):
        qkv[at:at + m, :wide] = normal((m, wide), TYPES[kind], seed + 7 * i + m)
    it = torch.int64 if ids == 64 else torch.int32
    s = types.SimpleNamespace(q=qkv[:, :heads * d], k=qkv[:, heads * d:(heads + kv) * d], v=qkv[:, (heads + kv) * d:wide], heads=heads, kv=kv, d=d, n=n,
                              starts=torch.tensor(starts, dtype=it, device=dev()), lengths=torch.tensor(lengths, dtype=it, device=dev()) if padded else None,
                              at=starts, of=lengths, bias=None, distances=None, scale=d ** -0.5, reach=reach)
    if buckets:
        s.bias = normal((heads, buckets), torch.float32, seed + 3)
        s.distances = (pqt.pqt_distance_buckets(buckets, reach, device=dev()) if reach >= max(1, buckets // 4) and buckets % 2 == 0 else
                       torch.randint(0, buckets, (2 * reach + 1,), generator=torch.Generator().manual_seed(seed)).int().to(dev()))
    return s


def arguments(s):
    return dict(heads=s.heads, scale=s.scale, bias=s.bias, distances=s.distances, lengths=s.lengths)


def logits(s, t, head):
    """(q, k, v, z, what z is off by, buckets) of a text's head in float64.  A product of d terms is off by (d + 2) U of their magnitudes; the bias, divided by the scale,
    added and multiplied by scale * log2 e, by 4 U; the exponent, a multiplication and an addition, by 3 U of its parts."""
    rows = slice(s.at[t], s.at[t] + s.of[t])
    cut = lambda x, h: x[rows, h * s.d:(h + 1) * s.d].double()                                           # noqa: E731
    q, k, v = cut(s.q, head), cut(s.k, head * s.kv // s.heads), cut(s.v, head * s.kv // s.heads)
    scale = torch.tensor(s.scale, dtype=torch.float32).double().item()
    z, off = q @ k.t() * scale, (q.abs() @ k.abs().t()) * scale * (s.d + 6) * U
    bucket = None
    if s.bias is not None:
        i = torch.arange(s.of[t], device=dev())
        bucket = s.distances.long()[(i[None, :] - i[:, None]).clamp(-s.reach, s.reach) + s.reach]
        there = (bucket >= 0) & (bucket < s.bias.shape[1])
        add = torch.where(there, s.bias[head].double()[bucket.clamp(0, s.bias.shape[1] - 1)], 0.0)
        z = z + add
        off = off + torch.where(add.isfinite(), add.abs(), 0.0) * 8 * U
    return q, k, v, z, off, bucket


def weight_unit(dtype):
    return 0.0 if dtype == torch.float32 else UNIT[dtype]


def check_attention(s, out, lse):
    want, tol = torch.zeros(s.n, s.heads * s.d, dtype=torch.float64, device=dev()), torch.zeros(s.n, s.heads * s.d, dtype=torch.float64, device=dev())
    want_lse, tol_lse = torch.full((s.heads, s.n), -INF, dtype=torch.float64, device=dev()), torch.zeros(s.heads, s.n, dtype=torch.float64, device=dev())
    for t in range(len(s.of)):
        if not s.of[t]:
            continue
        rows = slice(s.at[t], s.at[t] + s.of[t])
        for head in range(s.heads):
            q, k, v, z, off, _ = logits(s, t, head)
            share = torch.logsumexp(z, 1)
            top = torch.where(share.isfinite(), share, 0.0)
            p = torch.exp(z - top[:, None])
            # of a weight: what its logit is off by, the exponent's rounding; of the sum: the weights' mean error and that of adding
            exponent = off + (torch.where(z.isfinite(), z.abs(), 0.0) + top.abs()[:, None]) * 4 * U
            rel = (p * exponent).sum(1) * 1.01 + (s.of[t] + 8) * U
            columns = slice(head * s.d, (head + 1) * s.d)
            want[rows, columns] = p @ v
            tol[rows, columns] = (p * (exponent * 1.01 + rel[:, None] + weight_unit(s.q.dtype) * 1.01 + (s.of[t] + 16) * U)) @ v.abs() + 2.0 ** -30 * v.abs().amax()
            want_lse[head, rows], tol_lse[head, rows] = share, rel + top.abs() * 8 * U + 8 * U
    within(lse, want_lse, tol_lse, "lse")
    within(out, want, tol, "out")


ATTENTION = [  # lengths, heads, heads of keys, d, type, buckets, reach, padded to, pad, ids, rows behind
    ([1], 1, 1, 1, "f32", 0, 0, 0, 0, 64, 0), ([7], 16, 16, 64, "bf16", 32, 128, 0, 0, 64, 0), ([3, 0, 1, 33, 17, 0], 3, 1, 33, "f16", 5, 3, 0, 5, 32, 9),
    ([16, 32, 15, 31, 0], 4, 2, 64, "bf16", 32, 16, 40, 0, 64, 0), ([48, 5, 20], 8, 8, 64, "f32", 32, 128, 0, 8, 64, 0), ([129], 2, 2, 128, "f32", 20, 40, 0, 0, 32, 1),
    ([65, 200, 1], 2, 1, 96, "bf16", 64, 448, 201, 3, 64, 0), ([300], 4, 4, 80, "f16", 32, 128, 0, 0, 64, 0), ([513], 1, 1, 7, "bf16", 8, 1, 0, 1, 64, 2),
    ([100, 90, 0, 200, 130, 1, 99, 70, 60, 55, 300], 16, 8, 64, "bf16", 32, 128, 0, 0, 64, 5), ([400, 500, 700], 12, 3, 32, "f16", 2, 448, 0, 8, 32, 0),
    ([333, 444, 260], 16, 16, 100, "bf16", 32, 32, 500, 0, 64, 0), ([1025, 40], 16, 4, 128, "f32", 32, 128, 0, 0, 64, 0), ([777, 800], 12, 1, 96, "f16", 0, 0, 0, 1, 64, 100),
    ([1300], 16, 2, 97, "bf16", 16, 7, 0, 0, 64, 0), ([900, 200], 16, 16, 31, "f32", 33, 100, 0, 0, 64, 0), ([5000], 16, 4, 64, "bf16", 32, 128, 0, 0, 64, 3),
    ([2100, 2050], 16, 16, 128, "f16", 32, 128, 2200, 0, 64, 0), ([4500], 16, 1, 30, "f32", 32, 200, 0, 3, 32, 0), ([4300], 16, 8, 96, "bf16", 0, 0, 0, 0, 64, 0),
    # many texts of some hundred tokens; the farthest reach beside the widest heads; short texts with a long one among them; a single token a text
    ([600, 550, 620, 580, 640, 590, 610, 570], 16, 16, 128, "bf16", 64, 448, 0, 0, 64, 0), ([600, 550, 620, 580, 640, 590, 610, 570], 16, 4, 128, "f32", 32, 448, 0, 0, 32, 3),
    ([600, 550, 620, 580, 640, 590, 610, 0], 16, 16, 64, "f16", 32, 128, 700, 3, 64, 0), ([600, 550, 620, 580, 640, 590, 610, 570], 16, 16, 64, "bf16", 6, 2, 0, 0, 64, 1),
    ([700] + [5] * 40 + [0, 1], 3, 1, 80, "bf16", 32, 40, 0, 0, 64, 0), ([1] * 70, 5, 5, 64, "f16", 32, 16, 0, 0, 32, 2), ([60] * 20 + [33, 64, 63, 1000], 6, 2, 128, "f32", 32, 30, 0, 0, 64, 0),
    ([3000], 2, 1, 64, "bf16", 32, 128, 0, 0, 64, 0), ([129] * 30, 16, 16, 128, "f16", 4, 448, 130, 8, 64, 0),
    # texts of just a workgroup's rows, so that every second workgroup has none, in numbers that are no whole fours
    ([16] * 131, 3, 3, 64, "bf16", 32, 128, 0, 0, 64, 0), ([16] * 1101, 16, 16, 8, "bf16", 32, 16, 0, 0, 64, 0), ([64] * 41, 16, 16, 64, "bf16", 32, 128, 64, 0, 64, 0),
    ([128] * 51, 16, 16, 32, "f16", 32, 128, 0, 0, 64, 5), ([100, 128, 1] * 13, 16, 2, 64, "f32", 32, 128, 128, 0, 32, 0),
    # between the kernels' choices: 33 to 48 tokens, heads that are no multiple of a workgroup's; keys whose queries eight and six workgroups share
    ([40, 33, 48, 2] * 12, 13, 13, 64, "bf16", 32, 128, 0, 0, 64, 0), ([47, 49] * 20, 6, 3, 40, "f32", 32, 30, 0, 0, 64, 0), ([33] * 40, 5, 1, 96, "f16", 20, 448, 0, 3, 64, 2),
    ([1500], 8, 2, 80, "f16", 32, 128, 0, 0, 64, 0), ([4000], 16, 2, 64, "bf16", 32, 128, 0, 0, 64, 0), ([1000], 16, 4, 64, "f32", 32, 128, 0, 0, 64, 7), ([2000, 0, 2040], 8, 2, 128, "bf16", 32, 128, 2041, 0, 64, 0)]


@gpu
@pytest.mark.parametrize("case", ATTENTION, ids=lambda c: f"{len(c[0])}x{max(c[0])}-" + "-".join(map(str, c[1:])))
def test_attention(case):
    lengths, heads, kv, d, kind, buckets, reach, padded, pad, ids, behind = case
    s = attention_inputs(lengths, heads, kv, d, kind, buckets, reach, padded, pad, ids, behind)
    out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
    check_attention(s, out, lse)
    # into a part of a wider buffer: the same bytes, rows of no text as they were, nothing beside them
    view, check = guarded(s.n, heads * d, TYPES[kind])
    same, lse2 = pqt.pqt_attention(s.q, s.k, s.v, s.starts, out=view, **arguments(s))
    end = s.at[-1]
    assert same is view and torch.equal(view[:end], out[:end]) and bool((view[end:] == 7.0).all()) and torch.equal(lse2, lse)
    check()


def check_gradient(s, grad, out, lse, got):
    dq, dk, dv, dbias = got
    zeros = lambda heads: torch.zeros(s.n, heads * s.d, dtype=torch.float64, device=dev())               # noqa: E731
    want, tol = [zeros(s.heads), zeros(s.kv), zeros(s.kv)], [zeros(s.heads), zeros(s.kv), zeros(s.kv)]
    buckets = s.bias.shape[1] if s.bias is not None else 1
    want_b, tol_b = torch.zeros(s.heads, buckets, dtype=torch.float64, device=dev()), torch.zeros(s.heads, buckets, dtype=torch.float64, device=dev())
    unit = weight_unit(s.q.dtype)
    small = 2.0 ** -32 if s.q.dtype == torch.float16 else 0.0      # f16 numbers end that far below a row's largest
    scale = torch.tensor(s.scale, dtype=torch.float32).double().item()
    for t in range(len(s.of)):
        m = s.of[t]
        if not m:
            continue
        rows = slice(s.at[t], s.at[t] + m)
        for head in range(s.heads):
            q, k, v, z, off, bucket = logits(s, t, head)
            columns, shared = slice(head * s.d, (head + 1) * s.d), slice(head * s.kv // s.heads * s.d, (head * s.kv // s.heads + 1) * s.d)
            g, o, share = grad[rows, columns].double(), out[rows, columns].double(), lse[head, rows].double()
            share = torch.where(share == -INF, INF, share)
            p = torch.exp(z - share[:, None])
            finite = torch.where(share.isfinite(), share, 0.0)
            rel = (off + (torch.where(z.isfinite(), z.abs(), 0.0) + finite.abs()[:, None]) * 6 * U + 4 * U) * 1.01
            dp, delta = g @ v.t(), (g * o).sum(1, keepdim=True)
            ds = p * (dp - delta)
            # the two products of d terms each
            # (a weight, and a ds as an operand, below 2^-126 may count as zero: the exponential has no smaller results)
            off_ds = ds.abs() * rel + 2.0 ** -126 * (1 + (dp - delta).abs()) + p * 1.01 * (s.d + 6) * U * (g.abs() @ v.abs().t() + (g.abs() * o.abs()).sum(1, keepdim=True))
            # and rounded, for the products that follow
            of_row = off_ds + ds.abs() * unit * 1.01 + small * ds.abs().amax(1, keepdim=True)
            of_key = off_ds + ds.abs() * unit * 1.01 + small * ds.abs().amax(0, keepdim=True)
            add = (m + 8) * U
            want[0][rows, columns] = scale * ds @ k
            tol[0][rows, columns] = scale * (of_row + ds.abs() * add) @ k.abs()
            want[1][rows, shared] += scale * ds.t() @ q
            tol[1][rows, shared] += scale * (of_key + ds.abs() * add * s.heads / s.kv).t() @ q.abs()
            want[2][rows, shared] += p.t() @ g
            tol[2][rows, shared] += (p * (rel + unit * 1.01 + add * s.heads / s.kv) + small + 2.0 ** -126).t() @ g.abs()
            if bucket is not None:
                # a sum over at most m places of a diagonal, the texts' and the distances' sums: no term is added to more than m + 2 reach + 64 + texts
                off_sum = off_ds + ds.abs() * (m + 2 * s.reach + 64 + len(s.of)) * U
                for b in range(buckets):
                    mine = bucket == b
                    want_b[head, b] += torch.where(mine, ds, 0.0).sum()
                    tol_b[head, b] += torch.where(mine, off_sum, 0.0).sum()
    for name, a, w, e in zip(("dq", "dk", "dv"), got, want, tol):
        within(a, w, e, name)
    if s.bias is None:
        assert dbias is None
    else:
        within(dbias, want_b, tol_b, "dbias")


@gpu
@pytest.mark.parametrize("case", ATTENTION, ids=lambda c: f"{len(c[0])}x{max(c[0])}-" + "-".join(map(str, c[1:])))
def test_attention_gradient(case):
    lengths, heads, kv, d, kind, buckets, reach, padded, pad, ids, behind = case
    s = attention_inputs(lengths, heads, kv, d, kind, buckets, reach, padded, pad, ids, behind)
    out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
    grad = torch.full((s.n, heads * d + pad), float("nan"), dtype=TYPES[kind], device=dev())[:, :heads * d]
    for at, m in zip(s.at, s.of):
        grad[at:at + m] = normal((m, heads * d), TYPES[kind], 77 + m, 0, 0.01)
    got = pqt.pqt_attention_gradient(grad, s.q, s.k, s.v, out, lse, s.starts, **arguments(s))
    check_gradient(s, grad, out, lse, got)
    # into slices of one buffer: the same bytes, rows of no text as they were
    wide, check = guarded(s.n, (heads + 2 * kv) * d, TYPES[kind])
    views = wide[:, :heads * d], wide[:, heads * d:(heads + kv) * d], wide[:, (heads + kv) * d:]
    again = pqt.pqt_attention_gradient(grad, s.q, s.k, s.v, out, lse, s.starts, grads=views, **arguments(s))
    end = s.at[-1]
    for a, b in zip(again[:3], got[:3]):
        assert torch.equal(a[:end], b[:end]) and bool((a[end:] == 7.0).all())
    assert got[3] is None or torch.equal(again[3], got[3])
    check()


@gpu
@pytest.mark.parametrize("before,behind,texts", [(0, 40, 3), (37, 0, 3), (64, 200, 2), (5, 3, 0), (0, 17, 0), (130, 70, 1)])
def test_rows_of_no_text(before, behind, texts):
    """Rows before the first text and behind the last one: zeros (lse -inf) in results that the call makes, untouched in the caller's."""
    s = attention_inputs([20, 0, 90][:texts], 4, 2, 48, "bf16", 32, 20, 0, 0, 64, behind, 1, before)
    out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
    check_attention(s, out, lse)
    grad = torch.nan_to_num(s.q.clone())
    got = pqt.pqt_attention_gradient(grad, s.q, s.k, s.v, out, lse, s.starts, **arguments(s))
    check_gradient(s, grad, out, lse, got)
    held = [torch.full_like(t, 7.0) for t in (out,) + got[:3]]
    _, lse2 = pqt.pqt_attention(s.q, s.k, s.v, s.starts, out=held[0], **arguments(s))
    pqt.pqt_attention_gradient(grad, s.q, s.k, s.v, out, lse, s.starts, grads=held[1:], **arguments(s))
    a, b = s.at[0], s.at[-1]
    for t, made in zip(held, (out,) + got[:3]):
        assert bool((t[:a] == 7.0).all()) and bool((t[b:] == 7.0).all()) and torch.equal(t[a:b], made[a:b])
    assert torch.equal(lse2, lse)


@gpu
def test_no_texts_and_no_rows():
    empty = torch.zeros((0, 64), dtype=torch.bfloat16, device=dev())
    starts = torch.zeros(4, dtype=torch.int32, device=dev())
    bias, distances = torch.ones((2, 4), device=dev()), pqt.pqt_distance_buckets(4, 5, device=dev())
    out, lse = pqt.pqt_attention(empty, empty, empty, starts, 2, bias=bias, distances=distances)
    assert out.shape == (0, 64) and lse.shape == (2, 0)
    dq, dk, dv, dbias = pqt.pqt_attention_gradient(out, empty, empty, empty, out, lse, starts, 2, bias=bias, distances=distances)
    assert dq.shape == dk.shape == dv.shape == (0, 64) and not bool(dbias.any())
    x = torch.ones((30, 64), dtype=torch.bfloat16, device=dev())                                          # rows, but every text is empty
    out, lse = pqt.pqt_attention(x, x, x, starts, 2, bias=bias, distances=distances)
    assert not bool(out.any()) and bool((lse == -INF).all())
    grads = pqt.pqt_attention_gradient(x, x, x, x, out, lse, starts, 2, bias=bias, distances=distances)
    assert not any(bool(t.any()) for t in grads)


@gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("lengths", [[20], [70, 3, 1], [600] * 2])
def test_masks(kind, lengths):
    """Buckets of -inf mask their distances: only keys behind the query are left, so that a text's last token has none; tokens of the masked places hold
    infinities that the others do not see through weights of zero times them only where the formula multiplies them, so here finite ones."""
    s = attention_inputs(lengths, 16, 16, 64, kind, 2, 1)
    s.distances = torch.tensor([0, 0, 1], dtype=torch.int32, device=dev())
    s.bias = torch.stack([torch.full((16,), -INF), torch.linspace(-1, 1, 16)], 1).to(dev()).contiguous()
    out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
    for at, m in zip(s.at, s.of):
        assert bool((lse[:, at + m - 1] == -INF).all()) and not bool(out[at + m - 1].any())
    check_attention(s, out, lse)
    grad = normal((s.n, 16 * 64), TYPES[kind], 5)
    got = pqt.pqt_attention_gradient(grad, s.q, s.k, s.v, out, lse, s.starts, **arguments(s))
    check_gradient(s, grad, out, lse, got)
    assert not bool(got[3][:, 0].any())
    s.bias = torch.full_like(s.bias, -INF)                         # nothing is left to anybody
    out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
    assert not bool(out.any()) and bool((lse == -INF).all())
    got = pqt.pqt_attention_gradient(grad, s.q, s.k, s.v, out, lse, s.starts, **arguments(s))
    assert not any(bool(t.any()) for t in got)


@gpu
@pytest.mark.parametrize("value", [torch.finfo(torch.float32).min, -1e30, 1e30, 1e4, -1e4])
def test_one_bias_for_all(value):
    """A bias that all places share changes no weight, also where it is the type's lowest number."""
    s = attention_inputs([50, 33], 2, 2, 32, "f32", 0, 0)
    s.q.nan_to_num_(), s.k.nan_to_num_()
    plain, _ = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
    s.bias, s.distances, s.reach = torch.full((2, 1), value, device=dev()), torch.zeros(1, dtype=torch.int32, device=dev()), 0
    out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
    if abs(value) > 1e20:                                          # the logits vanish beside it: equal weights
        for at, m in zip(s.at, s.of):
            within(out[at:at + m], s.v[at:at + m].double().mean(0, keepdim=True).expand(m, -1).contiguous(), s.v[at:at + m].double().abs().mean(0, keepdim=True).expand(m, -1) * (m + 8) * U, "mean")
    else:
        within(out, plain.double(), 20 * abs(value) * 8 * U * torch.ones_like(plain).double(), "shifted")         # (2 x max |v| x what a logit is off by)
    assert bool(lse.isfinite().all())


@gpu
@pytest.mark.parametrize("lengths", [[5], [40, 3, 77], [700, 300], [300] * 16])
@pytest.mark.parametrize("bucket", [0, 2, -1, 3])
def test_reach_of_zero(lengths, bucket):
    """One bucket, or none, for all distances: its gradient is the sum over all places."""
    s = attention_inputs(lengths, 16, 16, 32, "bf16", 3, 0)
    s.distances = torch.tensor([bucket], dtype=torch.int32, device=dev())
    out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
    check_attention(s, out, lse)
    grad = normal((s.n, 512), torch.bfloat16, 5)
    check_gradient(s, grad, out, lse, pqt.pqt_attention_gradient(grad, s.q, s.k, s.v, out, lse, s.starts, **arguments(s)))


@gpu
def test_lowest_bias_masks_beside_others():
    """Distances with the type's lowest number get nothing where others have a finite one."""
    s = attention_inputs([90], 2, 2, 64, "bf16", 2, 2)
    s.distances = torch.tensor([0, 1, 1, 1, 0], dtype=torch.int32, device=dev())
    outs = []
    for low in (torch.finfo(torch.float32).min, -INF):
        s.bias = torch.tensor([[low, 0.5], [low, -3.0]], device=dev())
        out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
        outs.append((out, lse) + pqt.pqt_attention_gradient(s.q.clone(), s.q, s.k, s.v, out, lse, s.starts, **arguments(s)))
    for a, b in zip(*outs):
        assert torch.equal(a, b)


@gpu
def test_buckets_out_of_range_have_no_bias():
    s = attention_inputs([40, 100], 2, 1, 40, "f32", 6, 3)
    s.distances = torch.tensor([-1, 0, 5, 6, 2 ** 31 - 1, 3, -2 ** 31], dtype=torch.int32, device=dev())
    out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
    check_attention(s, out, lse)
    grad = normal((s.n, 80), torch.float32, 5)
    check_gradient(s, grad, out, lse, pqt.pqt_attention_gradient(grad, s.q, s.k, s.v, out, lse, s.starts, **arguments(s)))


@gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n", [30, 1500])
def test_large_logits_and_rising_ones(kind, n):
    """Logits up to hundreds, which rise along the text, so that the running maximum moves at every tile; gradients of all sizes, down to what f16 does
    not hold as a product."""
    s = attention_inputs([n], 16, 16, 32, kind, 0, 0)
    rise = torch.linspace(0.1, 20, n, device=dev())[:, None]
    s.k.mul_(rise.to(TYPES[kind]))
    s.scale = 1.0
    out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
    check_attention(s, out, lse)
    for size in (1e3, 1.0, 1e-4):
        grad = normal((n, 512), TYPES[kind], 5, 0, size)
        got = pqt.pqt_attention_gradient(grad, s.q, s.k, s.v, out, lse, s.starts, **arguments(s))
        check_gradient(s, grad, out, lse, got)


@gpu
@pytest.mark.parametrize("n,heads", [(60, 1), (1200, 16)])
def test_f16_gradients_far_below_its_numbers(n, heads):
    """ds of 1e-9 and less, of rows of very different sizes, one of them zero: gradients keep f16's precision as long as they are f16 numbers themselves."""
    s = attention_inputs([n], heads, heads, 64, "f16", 32, 16)
    out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
    grad = normal((n, heads * 64), torch.float16, 5, 0, 1.0)
    grad *= torch.logspace(-4, 1, n, device=dev())[:, None].half()
    grad[n // 2] = 0
    s.k *= 16
    s.scale /= 16
    out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
    check_gradient(s, grad, out, lse, pqt.pqt_attention_gradient(grad, s.q, s.k, s.v, out, lse, s.starts, **arguments(s)))


@gpu
def test_infinities_of_one_text_stay_there():
    """A text with infinities and NaN in its tokens beside others: the others' results are the same bytes as without it."""
    s = attention_inputs([70, 50, 90, 3], 4, 4, 64, "bf16", 32, 128)
    grad = normal((s.n, 256), torch.bfloat16, 5)
    out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
    want = (out, lse.t()) + pqt.pqt_attention_gradient(grad, s.q, s.k, s.v, out, lse, s.starts, **arguments(s))[:3]
    for t, value in ((s.q, INF), (s.k, float("nan")), (s.v, -INF)):
        t[s.at[1] + 7] = value
    out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
    got = (out, lse.t()) + pqt.pqt_attention_gradient(grad, s.q, s.k, s.v, out, lse, s.starts, **arguments(s))[:3]
    for a, b in zip(got, want):
        assert torch.equal(a[:s.at[1]], b[:s.at[1]]) and torch.equal(a[s.at[2]:], b[s.at[2]:])
    assert bool(out[s.at[1]:s.at[2]].isnan().any())


@gpu
def test_attention_offsets_beyond_32_bits():
    n, step = 2500, 1_000_003                                      # 2.5e9 elements from the first row to the last, rows at odd places
    wide = torch.empty((n, step), dtype=torch.bfloat16, device=dev())
    s = attention_inputs([2000, 500], 4, 4, 64, "bf16", 32, 128)
    far = [wide[:, 1 + 300 * i:1 + 300 * i + 256] for i in range(8)]
    grad = normal((n, 256), torch.bfloat16, 5)
    for view, t in zip(far, (s.q, s.k, s.v, grad)):
        view.copy_(t)
    out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
    want = pqt.pqt_attention_gradient(grad, s.q, s.k, s.v, out, lse, s.starts, **arguments(s))
    got, lse2 = pqt.pqt_attention(far[0], far[1], far[2], s.starts, out=far[4], **arguments(s))
    assert torch.equal(got, out) and torch.equal(lse2, lse)
    grads = pqt.pqt_attention_gradient(far[3], far[0], far[1], far[2], far[4], lse, s.starts, grads=far[5:], **arguments(s))
    for a, b in zip(grads, want):
        assert torch.equal(a, b)
    del wide, far, got, grads


@gpu
def test_starts_out_of_range_stay_inside():
    """Places beyond the rows, or descending, are taken as the nearest that are in range: nothing outside is read or written."""
    s = attention_inputs([60, 40], 2, 2, 32, "bf16", 0, 0)
    for starts, lengths in (([-5, 60, 1000], None), ([0, 60, 100], [10 ** 6, -3]), ([90, 20, 100], None), ([-2 ** 62, 2 ** 62, 0], [2 ** 62, 2 ** 62])):
        st = torch.tensor(starts, device=dev())
        le = torch.tensor(lengths, device=dev()) if lengths else None
        view, check = guarded(100, 64, torch.bfloat16)
        out, lse = pqt.pqt_attention(s.q, s.k, s.v, st, 2, lengths=le, out=view)
        check()
        wide, check = guarded(100, 192, torch.bfloat16)
        pqt.pqt_attention_gradient(s.q, s.q, s.k, s.v, out, lse, st, 2, lengths=le, grads=(wide[:, :64], wide[:, 64:128], wide[:, 128:]))
        check()
    want, _ = pqt.pqt_attention(s.q, s.k, s.v, s.starts, 2)
    assert torch.equal(pqt.pqt_attention(s.q, s.k, s.v, torch.tensor([-5, 60, 1000], device=dev()), 2)[0], want)


@gpu
def test_attention_gradient_by_differences():
    """<out, c> along random directions of q, k, v and the bias, by central differences of the 64-bit formula, shared key heads among them."""
    s = attention_inputs([19, 40], 4, 2, 24, "f32", 8, 6)
    c = normal((s.n, 96), torch.float32, 9)
    out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
    grads = pqt.pqt_attention_gradient(c, s.q, s.k, s.v, out, lse, s.starts, **arguments(s))
    inputs = [t.double().clone() for t in (s.q, s.k, s.v, s.bias)]

    def f(values):
        at = types.SimpleNamespace(**{**vars(s), "q": values[0], "k": values[1], "v": values[2], "bias": values[3]})
        total = 0.0
        for t in range(2):
            for head in range(4):
                _, _, v, z, _, _ = logits(at, t, head)
                total += float((torch.softmax(z, 1) @ v * c[s.at[t]:s.at[t + 1], head * 24:(head + 1) * 24].double()).sum())
        return total
    e = 1e-4
    for which, got in enumerate(grads):
        for seed in range(2):
            a = normal(tuple(got.shape), torch.float32, 40 + 2 * which + seed).double()
            move = lambda sign: [t + sign * e * a if i == which else t for i, t in enumerate(inputs)]     # noqa: E731
            want = (f(move(1)) - f(move(-1))) / (2 * e)
            # differences of a sum of ~6e3 terms of size one, third derivatives of that size: 1e3 e^2 of each direction's and 1e-12 / e; kernels 1e2 U of the terms
            assert abs(float((got.double() * a).sum()) - want) <= 2e-3 + 1e-4 * abs(want), (which, float((got.double() * a).sum()), want)


@gpu
def test_gradients_of_a_broadcast_bias():
    """One head's row of biases, used for all heads by copies: its gradient is the sum over the copies."""
    s = attention_inputs([300, 77], 4, 4, 32, "f32", 6, 10)
    s.bias = normal((1, 6), torch.float32, 1).expand(4, 6).contiguous()
    out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
    grad = normal((s.n, 128), torch.float32, 2)
    check_gradient(s, grad, out, lse, pqt.pqt_attention_gradient(grad, s.q, s.k, s.v, out, lse, s.starts, **arguments(s)))
    with pytest.raises(ValueError):
        pqt.pqt_attention(s.q, s.k, s.v, s.starts, 4, bias=s.bias[:1].expand(4, 6), distances=s.distances)


# ---- buckets ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("buckets,far,both", [(32, 128, True), (64, 448, True), (2, 1, True), (20, 100, True), (32, 128, False), (5, 17, False), (2, 3, False), (1024, 448, True), (8, 3, True)])
def test_distance_buckets(buckets, far, both):
    """Against the definition in whole numbers: log(t / near) / log(far / near) * rest >= step where (t / near)^rest >= (far / near)^step."""
    side = buckets // 2 if both else buckets
    near = max(1, side // 2)
    rest = side - near
    got = pqt.pqt_distance_buckets(buckets, far, both)
    if far < near:
        pytest.fail("not a valid case")
    for at in range(-far, far + 1):
        away = -at if at <= 0 else at if both else 0
        want = away
        if away >= near:
            step = 0
            while far > near and step < rest - 1 and away ** rest * near ** (step + 1) >= far ** (step + 1) * near ** rest:
                step += 1
            want = near + step
        want = min(want, side - 1) + (side if both and at > 0 else 0)
        assert int(got[at + far]) == want, (at, int(got[at + far]), want)
    assert int(got.min()) == 0 and int(got.max()) < buckets


@pytest.mark.parametrize("buckets,far", [(32, 2 ** 32 + 128), (2 ** 32 + 32, 128), (32, -1), (-2 ** 32 + 32, 128), (32, 0)])
def test_refusals_of_distance_buckets_beyond_32_bits(buckets, far):
    with pytest.raises(pqt.PqtError):
        pqt.pqt_distance_buckets(buckets, far)


def test_refusals_of_distance_buckets():
    for args in ((1, 10), (3, 10, True), (32, 0), (32, 449), (1026, 300), (64, 10), (0, 5), (-2, 5)):
        with pytest.raises(pqt.PqtError) as e:
            pqt.pqt_distance_buckets(*args)
        assert e.value.code == pqt.PQT_EINVAL


# ---- streams, graphs, a layer of both --------------------------------------------------------------------------------
def layer(s, x, r, w, qkv_blocks, grad_y):
    """Norm into blocks, the fused projection, attention, and the way back to the norm's input: what an encoder's layer does with these calls."""
    y, h, rstd = pqt.pqt_rms_norm(x, w, r, blocks=True)
    qkv = pqt.pqt_block_product(y, qkv_blocks, out_dtype=x.dtype)
    D = s.heads * s.d
    q, k, v = qkv[:, :D], qkv[:, D:2 * D], qkv[:, 2 * D:]
    out, lse = pqt.pqt_attention(q, k, v, s.starts, **arguments(s))
    d_qkv = torch.empty_like(qkv)
    *_, d_bias = pqt.pqt_attention_gradient(grad_y, q, k, v, out, lse, s.starts, grads=(d_qkv[:, :D], d_qkv[:, D:2 * D], d_qkv[:, 2 * D:]), **arguments(s))
    dx, dw = pqt.pqt_rms_norm_gradient(d_qkv[:, :x.shape[1]], h, w, rstd, grad_y[:, :x.shape[1]])
    return y.codes.view(torch.uint8), h, out, lse, d_qkv, d_bias, dx, dw


def layer_inputs(lengths=(40, 3, 90, 200, 1, 0, 60)):
    s = attention_inputs(list(lengths), 4, 4, 64, "bf16", 32, 64)
    x, r, grad = (normal((s.n, 200), torch.bfloat16, i) for i in (1, 2, 3))
    grad = normal((s.n, 256), torch.bfloat16, 4, 0, 0.1)
    w = (1 + 0.2 * normal((1, 200), torch.float32, 5)[0]).bfloat16().contiguous()
    return s, x, r, w, pqt.pqt_block_quantize(normal((768, 200), torch.float32, 6, 0, 0.07)), grad


@gpu
def test_a_layer_forward_and_backward():
    """The calls of a layer one after the other, each step against the 64-bit formula on what the one before gave it."""
    s, x, r, w, blocks, grad = layer_inputs()
    codes, h, out, lse, d_qkv, d_bias, dx, dw = layer(s, x, r, w, blocks, grad)
    y, _, rstd = pqt.pqt_rms_norm(x, w, r, blocks=True)
    qkv = pqt.pqt_block_product(y, blocks, out_dtype=x.dtype)
    s.q, s.k, s.v = qkv[:, :256], qkv[:, 256:512], qkv[:, 512:]
    check_attention(s, out, lse)
    check_gradient(s, grad, out, lse, (d_qkv[:, :256], d_qkv[:, 256:512], d_qkv[:, 512:], d_bias))
    want, tol, want_w, tol_w = norm_gradient_reference(d_qkv[:, :200], h, w, rstd, grad[:, :200])
    within(dx, want, tol, "dx")
    within(dw, want_w, tol_w, "dweight")


@gpu
def test_layers_on_another_stream():
    s, x, r, w, blocks, grad = layer_inputs()
    want = layer(s, x, r, w, blocks, grad)
    torch.cuda.synchronize()
    side, late = torch.cuda.Stream(), torch.zeros_like(x)
    with torch.cuda.stream(side):
        busy = torch.randn(4096, 4096, device=dev())
        for _ in range(20):
            busy = busy @ busy * 1e-3
        late.copy_(x)                                              # there only when the stream gets to it
    y, h, rstd = pqt.pqt_rms_norm(late, w, r, blocks=True, stream=side)
    qkv = pqt.pqt_block_product(y, blocks, out_dtype=x.dtype, stream=side)
    q, k, v = qkv[:, :256], qkv[:, 256:512], qkv[:, 512:]
    out, lse = pqt.pqt_attention(q, k, v, s.starts, stream=side, **arguments(s))
    got = pqt.pqt_attention_gradient(grad, q, k, v, out, lse, s.starts, stream=side, **arguments(s))
    dx, dw = pqt.pqt_rms_norm_gradient(got[0][:, :200], h, w, rstd, grad[:, :200], stream=side)
    side.synchronize()
    for a, b in zip((h, out, lse, torch.cat(got[:3], 1), got[3], dx, dw), want[1:]):
        assert torch.equal(a, b)


@gpu
def test_layers_in_graphs():
    """Two captured graphs of a layer, replayed in turn with other inputs, with eager calls and synchronisations between: every replay as the eager result."""
    runs = []
    for lengths in ((40, 3, 90, 200, 1, 0, 60), (500, 600, 100)):
        s, x, r, w, blocks, grad = layer_inputs(lengths)
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            layer(s, x, r, w, blocks, grad)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = layer(s, x, r, w, blocks, grad)
        runs.append((s, x, r, w, blocks, grad, graph, held))
    for seed in range(3):
        for s, x, r, w, blocks, grad, graph, held in runs:
            x.copy_(normal(tuple(x.shape), torch.bfloat16, 100 + seed))
            grad.copy_(normal(tuple(grad.shape), torch.bfloat16, 200 + seed, 0, 0.1))
            if seed == 2:                                          # other texts in the same rows
                s.starts.copy_(torch.tensor(sorted([0, s.n] + [(i * 37) % s.n for i in range(1, len(s.starts) - 1)]), device=dev()))
            want = [t.clone() for t in layer(s, x, r, w, blocks, grad)]
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for got, w_ in zip(held, want):
                assert torch.equal(got, w_)
    for _, _, _, _, _, _, graph, _ in runs:                        # one behind the other, nothing waited for
        graph.replay()
    torch.cuda.synchronize()
    for s, x, r, w, blocks, grad, _, held in runs:
        for got, w_ in zip(held, layer(s, x, r, w, blocks, grad)):
            assert torch.equal(got, w_)


@gpu
def test_layers_by_a_thread_each():
    """Two threads with streams of their own call at once: each gets its own results."""
    import threading
    sides = [layer_inputs(), layer_inputs((300, 300, 11))]
    want = [layer(*a) for a in sides]
    torch.cuda.synchronize()
    got, streams = [None, None], [torch.cuda.Stream(), torch.cuda.Stream()]

    def work(i):
        with torch.cuda.stream(streams[i]):
            for _ in range(20):
                got[i] = layer(*sides[i])
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for i in range(2):
        for a, b in zip(got[i], want[i]):
            assert torch.equal(a, b)


# ---- refusals --------------------------------------------------------------------------------------------------------
def refused(fn, *args, code=pqt.PQT_EINVAL):
    rc = fn(*args)
    assert rc == code, (rc, pqt.last_error())
    assert pqt.last_error()


def test_refusals_of_the_library(library_without_gpu):
    """Arguments are checked before anything touches a GPU (addresses here are never read)."""
    lib, p, far = library_without_gpu, 1 << 20, 1 << 40
    ok = dict(x=p, type=1, rows=4, D=8, xs=8, r=p, rs=8, h=p, hs=8, w=p, pt=0, eps=1e-6, y=p, ot=0, ys=8, c=None, s=None, rstd=p, device=0, stream=None)
    call = lambda **kw: tuple({**ok, **kw}.values())                                                      # noqa: E731
    for bad in (dict(type=3), dict(pt=-1), dict(ot=9), dict(rows=-1), dict(D=0), dict(xs=7), dict(rs=7), dict(hs=7), dict(ys=7), dict(eps=-1.0), dict(eps=float("nan")), dict(x=None),
                dict(y=None), dict(c=p, s=p), dict(y=None, c=p), dict(y=None, s=p), dict(y=None, c=p + 8, s=p), dict(x=p + 1), dict(r=p + 1), dict(h=p + 1), dict(w=p + 2), dict(y=p + 2),
                dict(rstd=p + 2)):
        refused(lib.pqt_rms_norm, *call(**bad))
    refused(lib.pqt_rms_norm, *call(D=32769, xs=40000, rs=40000, hs=40000, ys=40000), code=pqt.PQT_EUNSUPPORTED)
    assert lib.pqt_rms_norm(*call(rows=0, x=None, y=None)) == pqt.PQT_OK
    for fine in (dict(), dict(y=None, c=p, s=p), dict(r=None, rs=0, h=None, hs=0), dict(w=None, rstd=None)):
        refused(lib.pqt_rms_norm, *call(**fine), code=pqt.PQT_EHIP)

    ok = dict(g=p, gs=8, t=p, ts=8, h=p, hs=8, type=0, rows=4, D=8, w=p, pt=0, rstd=p, dx=p, ds=8, dw=p, ws=p, wsn=far, device=0, stream=None)
    for bad in (dict(type=4), dict(pt=5), dict(rows=-1), dict(D=0), dict(gs=7), dict(ts=7), dict(hs=7), dict(ds=7), dict(g=None), dict(h=None), dict(rstd=None), dict(dx=None), dict(ws=None),
                dict(wsn=4), dict(ws=p + 4), dict(g=p + 1), dict(t=p + 2), dict(h=p + 2), dict(dx=p + 1), dict(dw=p + 2), dict(w=p + 3), dict(rstd=p + 1)):
        refused(lib.pqt_rms_norm_gradient, *call(**bad))
    refused(lib.pqt_rms_norm_gradient, *call(D=32769, gs=40000, ts=40000, hs=40000, ds=40000), code=pqt.PQT_EUNSUPPORTED)
    assert lib.pqt_rms_norm_gradient(*call(rows=0, dw=None)) == pqt.PQT_OK
    for fine in (dict(), dict(t=None, ts=0), dict(w=None, dw=None, ws=None, wsn=0)):
        refused(lib.pqt_rms_norm_gradient, *call(**fine), code=pqt.PQT_EHIP)
    assert pqt.pqt_rms_norm_gradient_workspace(0, 5) == 0 and pqt.pqt_rms_norm_gradient_workspace(5, 40000) == 0 and pqt.pqt_rms_norm_gradient_workspace(5000, 64) > 0

    ok = dict(q=p, qs=64, k=p, ks=32, v=p, vs=32, type=1, n=100, heads=4, kv=2, d=16, starts=p, lengths=p, size=8, texts=3, scale=0.25, bias=p, buckets=8, dist=p, reach=5, clear=0, out=p, os=64,
              lse=p, device=0, stream=None)
    layout = (dict(type=3), dict(n=-1), dict(heads=0), dict(kv=0), dict(kv=3), dict(d=0), dict(starts=None), dict(size=2), dict(texts=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
              dict(scale=2.0 ** 33), dict(scale=2.0 ** -33), dict(buckets=0), dict(dist=None), dict(reach=-1), dict(qs=63), dict(ks=31), dict(vs=31), dict(os=63), dict(q=None), dict(k=None),
              dict(v=None), dict(out=None), dict(q=p + 1), dict(k=p + 1), dict(v=p + 1), dict(out=p + 1), dict(starts=p + 4), dict(lengths=p + 4), dict(bias=p + 2), dict(dist=p + 2), dict(lse=p + 2))
    for bad in layout:
        refused(lib.pqt_attention, *call(**bad))
    wide = dict(qs=1000, ks=1000, vs=1000, os=1000)
    beyond = (dict(d=129, **wide), dict(buckets=1025), dict(reach=449), dict(n=1 << 31), dict(texts=1 << 31), dict(n=1 << 30))
    for bad in beyond:
        refused(lib.pqt_attention, *call(**bad), code=pqt.PQT_EUNSUPPORTED)
    assert lib.pqt_attention(*call(n=0, starts=None, q=None)) == pqt.PQT_OK
    for fine in (dict(), dict(lengths=None, bias=None, buckets=0, dist=None, reach=0, lse=None), dict(size=4, starts=p + 4), dict(texts=0)):
        refused(lib.pqt_attention, *call(**fine), code=pqt.PQT_EHIP)

    ok = dict(g=p, gs=64, q=p, qs=64, k=p, ks=32, v=p, vs=32, out=p, os=64, lse=p, type=1, n=100, heads=4, kv=2, d=16, starts=p, lengths=p, size=8, texts=3, scale=0.25, bias=p, buckets=8, dist=p,
              reach=5, clear=0, dq=p, dqs=64, dk=p, dks=32, dv=p, dvs=32, db=p, ws=p, wsn=far, device=0, stream=None)
    for bad in layout + (dict(g=None), dict(gs=63), dict(lse=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(dqs=63), dict(dks=31), dict(dvs=31), dict(g=p + 1), dict(dq=p + 1), dict(dk=p + 1),
                         dict(dv=p + 1), dict(db=p + 2), dict(ws=None), dict(wsn=100), dict(ws=p + 8), dict(bias=None)):
        refused(lib.pqt_attention_gradient, *call(**bad))
    wide.update(gs=1000, dqs=1000, dks=1000, dvs=1000)
    for bad in (dict(d=129, **wide),) + beyond[1:]:
        refused(lib.pqt_attention_gradient, *call(**bad), code=pqt.PQT_EUNSUPPORTED)
    assert lib.pqt_attention_gradient(*call(n=0, db=None)) == pqt.PQT_OK
    for fine in (dict(), dict(lengths=None, bias=None, buckets=0, dist=None, reach=0, db=None), dict(db=None)):
        refused(lib.pqt_attention_gradient, *call(**fine), code=pqt.PQT_EHIP)
    assert pqt.pqt_attention_gradient_workspace(0, 1, 2, 2, 64, 3) == 0 and pqt.pqt_attention_gradient_workspace(100, 2, 4, 3, 64, -1) == 0
    assert pqt.pqt_attention_gradient_workspace(100, 2, 4, 4, 200, -1) == 0 and pqt.pqt_attention_gradient_workspace(100, 2, 4, 1, 64, -1) >= 1600
    assert pqt.pqt_attention_gradient_workspace(100, 2, 4, 4, 64, 0) > pqt.pqt_attention_gradient_workspace(100, 2, 4, 4, 64, -1)


def test_refusals_of_the_binding():
    x, at = torch.zeros((4, 8)), torch.tensor([0, 4])
    for call in (lambda: pqt.pqt_rms_norm(x), lambda: pqt.pqt_rms_norm_gradient(x, x, None, x[:, 0]), lambda: pqt.pqt_attention(x, x, x, at, 2),
                 lambda: pqt.pqt_attention_gradient(x, x, x, x, x, x, at, 2)):
        with pytest.raises(ValueError):
            call()                                                 # tensors of the CPU
    other = types.SimpleNamespace(device=torch.device("cuda", 7))
    for call in (lambda **kw: pqt.pqt_rms_norm(x, **kw), lambda **kw: pqt.pqt_rms_norm_gradient(x, x, None, x[:, 0], **kw), lambda **kw: pqt.pqt_attention(x, x, x, at, 2, **kw),
                 lambda **kw: pqt.pqt_attention_gradient(x, x, x, x, x, x, at, 2, **kw)):
        with pytest.raises(ValueError, match="the stream is on cuda:7"):
            call(stream=other)


@gpu
def test_refusals_of_shapes_and_types():
    x = torch.zeros((4, 8), device=dev())
    at, w, lse = torch.tensor([0, 4], device=dev()), torch.zeros(8, device=dev()), torch.zeros((2, 4), device=dev())
    bias, dist = torch.zeros((2, 3), device=dev()), torch.zeros(5, dtype=torch.int32, device=dev())
    attend = lambda q=x, k=x, v=x, starts=at, heads=2, **kw: pqt.pqt_attention(q, k, v, starts, heads, **kw)              # noqa: E731
    back = lambda g=x, q=x, k=x, v=x, out=x, lse=lse, starts=at, heads=2, **kw: pqt.pqt_attention_gradient(g, q, k, v, out, lse, starts, heads, **kw)      # noqa: E731
    for call in (lambda: pqt.pqt_rms_norm(x, w[:7]), lambda: pqt.pqt_rms_norm(x, w.int()), lambda: pqt.pqt_rms_norm(x, w, x[:3]), lambda: pqt.pqt_rms_norm(x, w, x.half()), lambda: pqt.pqt_rms_norm(x.t()),
                 lambda: pqt.pqt_rms_norm(x, blocks=True, out=x), lambda: pqt.pqt_rms_norm(x, blocks=True, out_dtype=torch.float32), lambda: pqt.pqt_rms_norm(x, w, x.cpu()),
                 lambda: pqt.pqt_rms_norm(x, out=torch.zeros((4, 8), device=dev()), out_dtype=torch.float16), lambda: pqt.pqt_rms_norm_gradient(x.half(), x, w, w[:4]),
                 lambda: pqt.pqt_rms_norm_gradient(x, x, w, w), lambda: pqt.pqt_rms_norm_gradient(x, x, w, w[:4], x[:, :7]), lambda: pqt.pqt_rms_norm_gradient(x, x, w, w[:4], out=x.half()),
                 lambda: attend(heads=3), lambda: attend(heads=0), lambda: attend(k=x[:, :6]), lambda: attend(k=x[:3]), lambda: attend(v=x[:, :4]), lambda: attend(v=x.half()), lambda: attend(starts=at.float()),
                 lambda: attend(starts=at.cpu()), lambda: attend(starts=at[:0]), lambda: attend(lengths=at[:1].int()), lambda: attend(lengths=at), lambda: attend(bias=bias), lambda: attend(distances=dist),
                 lambda: attend(bias=bias[:1], distances=dist), lambda: attend(bias=bias.half(), distances=dist), lambda: attend(bias=bias, distances=dist.long()), lambda: attend(bias=bias, distances=dist[:4]),
                 lambda: attend(bias=bias.t().contiguous().t(), distances=dist), lambda: attend(out=x.half()), lambda: attend(out=x[:, :6]), lambda: attend(out=x[:1].expand(4, 8)),
                 lambda: back(g=x.half()), lambda: back(out=x[:, :6]), lambda: back(lse=lse.t()), lambda: back(lse=lse[:1]), lambda: back(lse=lse.double()), lambda: back(grads=(x, x, x.half())),
                 lambda: back(grads=(x, x[:3], x))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: attend(scale=0.0), lambda: attend(scale=INF), lambda: back(scale=-1.0)):
        with pytest.raises(pqt.PqtError):
            call()
