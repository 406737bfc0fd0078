"""The query encoder's operators at sizes where every kernel is past its first round: groups that walk their rows, results stored past the
caches, sorts with several rounds a tile, and every kernel of the block products, whole and shared out, by type of result.

The references are computed in 64 bits by torch, most of them on the GPU; the tolerances are those of test_query_encoder.py: a sum of c terms in any order is
off by at most c u times the sum of their magnitudes (u = 2^-24), and less where the additions that a term passes through are known to be fewer."""
import os
import subprocess

import pytest
import torch

import test_query_encoder as base
from test_query_encoder import DEPTH, LEAST, TYPES, U, UNIT, dev, gpu, guarded, normal, pqt, some_tokens

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STREAM_BYTES = 32 << 20                                           # larger results are stored past the caches


def within(got, want, tol, what):
    """As in test_query_encoder.py, on the GPU."""
    t = got.dtype
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = ~((got.double() - want).abs() <= tol + want.abs() * UNIT[t] * (1 + 2.0 ** -6) + LEAST[t])
    if bool(bad.any()):
        i = tuple(int(v) for v in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} values off, first at {i}: {float(got[i])} for {float(want[i])}")


# ---- which kernel multiplies -----------------------------------------------------------------------------------------
PRODUCT = [  # m, n, k, type, bias, pad; the kernel's tile, workgroups that share a tile's blocks of k
    (4200, 4100, 300, "bf16", True, 1, 128, 1), (4200, 4100, 300, "f16", False, 0, 128, 1), (4200, 4100, 300, "f32", True, 3, 128, 1),
    (2300, 2301, 2047, "bf16", False, 0, 128, 1), (2300, 2301, 2047, "f16", True, 1, 128, 1), (2300, 2301, 2047, "f32", False, 0, 128, 1),
    (1301, 1270, 8193, "bf16", True, 1, 128, 4), (1301, 1270, 8193, "f16", False, 0, 128, 4), (1100, 1290, 8321, "f32", True, 2, 128, 7),
    (8191, 960, 2000, "bf16", False, 0, 128, 1), (960, 2000, 8191, "f32", False, 0, 128, 4),
    (8191, 4099, 520, "bf16", True, 5, 256, 1), (700, 900, 8193, "bf16", False, 1, 64, 4), (700, 900, 8193, "f16", False, 0, 64, 7), (700, 900, 8193, "f32", True, 0, 64, 7),
    (1000, 1000, 1000, "bf16", True, 0, 64, 1), (1000, 1000, 1000, "f16", False, 0, 64, 1), (1000, 1000, 1000, "f32", False, 0, 64, 1),
    (16, 33_000, 300, "f16", True, 0, 16, 1), (64, 4096, 1000, "bf16", False, 0, 64, 1)]


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("host") / "product_plan")
    res = subprocess.run(["g++", "-std=c++17", "-O1", os.path.join(ROOT, "tests", "host", "product_plan.cpp"), "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr

    def run(sizes):
        """(tile, splits, blocks of k of a workgroup, 64 columns a workgroup) of every (m, n, k, type)."""
        lines = "".join(f"{m} {n} {k} {int(t != 'bf16')}\n" for m, n, k, t in sizes)
        out = subprocess.run([exe], input=lines, capture_output=True, text=True, check=True).stdout
        return [tuple(int(v) for v in line.split()) for line in out.splitlines()]
    return run


def test_the_products_below_take_these_kernels(plan):
    for case, got in zip(PRODUCT, plan([c[:4] for c in PRODUCT])):
        assert got[:2] == case[6:8], (case, got)


def test_every_product_kernel_has_a_test(plan):
    """Whole and shared out: what the sizes of the tests here and of test_block_product reach."""
    sizes = [c[:4] for c in PRODUCT] + [c[:4] for c in base.PRODUCT]
    reached = {(t, p[0], p[1] > 1, p[3]) for (_, _, _, t), p in zip(sizes, plan(sizes))}
    for t in TYPES:
        assert {(t, 16, False, 0), (t, 64, False, 0), (t, 64, True, 0), (t, 128, False, 0), (t, 128, True, 0)} <= reached, (t, reached)
    assert ("bf16", 256, False, 0) in reached and ("f16", 16, False, 1) in reached


def test_plans_stay_in_their_limits(plan):
    """A plan's workgroups cover the blocks of k, an even number each where they share them, none of them empty, at most sixteen."""
    g = torch.Generator().manual_seed(0)
    sizes = [(int(torch.exp(torch.rand(1, generator=g) * 11)) + 1, int(torch.exp(torch.rand(1, generator=g) * 11)) + 1,
              int(torch.exp(torch.rand(1, generator=g) * 15)) + 1, ("bf16", "f32")[i % 2]) for i in range(2000)]
    for (m, n, k, t), (tile, splits, per, _) in zip(sizes, plan(sizes)):
        kb = -(-k // 128)
        assert tile in ((16,) if m <= 16 else (64, 128, 256) if t == "bf16" else (64, 128)), (m, n, k, t, tile)
        assert 1 <= splits <= 16 and (splits - 1) * per < kb <= splits * per and (splits == 1 or (per % 2 == 0 and tile in (64, 128))), (m, n, k, t, splits, per)


def values(blocks):
    v = blocks.codes.float().double() * torch.exp2(blocks.scales.double() - 127).repeat_interleave(128, 1)
    return v[:, :blocks.cols]


@gpu
@pytest.mark.parametrize("m,n,k,kind,bias,pad,tile,splits", PRODUCT)
def test_block_product(m, n, k, kind, bias, pad, tile, splits):
    x, w = normal((m, k), torch.float32, m + k), normal((n, k), torch.float32, n + k + 1, 0, 0.1 / k ** 0.5)
    x *= torch.exp(torch.linspace(-3, 3, k, device=dev()))
    a, b = pqt.pqt_block_quantize(x), pqt.pqt_block_quantize(w)
    v = normal((1, n), torch.float32, 5)[0].contiguous() if bias else None
    view, check = guarded(m, n, TYPES[kind], pad + 1)
    got = pqt.pqt_block_product(a, b, bias=v, out=view)
    A, B = values(a), values(b)
    want = A @ B.t().contiguous()
    # an instruction adds up 32 products (bf16: 128), a wavefront's instructions follow each other, at most 16 such sums are joined: additions that
    # are each off by at most 2^-23 of a partial sum; bf16 results may lose 2^-13 of the largest of eight products for each of the others
    tol = (A.abs() @ B.abs().t().contiguous()) * ((k / 32 + 48) * 2.0 ** -23 + (8 * 2.0 ** -13 if kind == "bf16" else 0.0))
    if bias:
        want = want + v.double()
        tol = tol + U * (want.abs() + v.double().abs())
    within(got, want, tol, "product")
    check()
    assert torch.equal(pqt.pqt_block_product(a, b, bias=v, out_dtype=TYPES[kind]), got)


@gpu
@pytest.mark.parametrize("m,n,k,kind,bias,pad,tile,splits", PRODUCT)
def test_block_product_of_integers(m, n, k, kind, bias, pad, tile, splits):
    """Forty small whole numbers a row, which every type holds the sums of: exact, so that no block and no row of a fragment can be missing."""
    g = torch.Generator().manual_seed(k)
    x, w = torch.zeros((m, k)), torch.zeros((n, k))
    for t, rows in ((x, m), (w, n)):
        t.scatter_(1, torch.randint(0, k, (rows, 40), generator=g), torch.randint(-3, 4, (rows, 40), generator=g).float())
    s = torch.exp2(3 * torch.arange(-(-k // 128)) % 7 - 3.0).repeat_interleave(128)[:k]       # scales that differ from block to block, both sides cancel
    x, w = (x * s).to(dev()), (w / s).to(dev())
    got = pqt.pqt_block_product(pqt.pqt_block_quantize(x), pqt.pqt_block_quantize(w), out_dtype=TYPES[kind])
    assert torch.equal(got.double(), x.double() @ w.double().t().contiguous())


@gpu
def test_products_that_overlap_in_time():
    """Two streams, each with calls that need a workspace: what they write is what they write alone."""
    a, b = (pqt.pqt_block_quantize(normal((r, 8193), torch.float32, r)) for r in (700, 900))
    grad, tok = normal((40_001, 96), torch.float32, 3), some_tokens(40_001, 3000, 4)
    x = normal((3000, 900), torch.float32, 5)
    _, mean, rstd = pqt.pqt_layer_norm(x)

    def calls():
        return [pqt.pqt_block_product(a, b, out_dtype=torch.float32), pqt.pqt_embed_gradient(grad, tok, 3000), *pqt.pqt_layer_norm_gradient(x, x, None, mean, rstd),
                pqt.pqt_block_product(b, a, out_dtype=torch.bfloat16)]
    want = calls()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    results = []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                results.append(calls())
    torch.cuda.synchronize()
    for got in results:
        assert all(torch.equal(g, w) for g, w in zip(got, want))


# ---- embedding -------------------------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("n,V,D,kind,out,ids,pad", [
    (600_001, 1000, 3, "f32", "f32", 64, 1), (150_001, 3000, 40, "bf16", "bf16", 32, 0), (60_001, 2000, 250, "f16", "f32", 64, 5), (50_003, 5000, 600, "bf16", "f32", 64, 8),
    (20_011, 900, 1030, "bf16", "bf16", 32, 3), (9001, 300, 4099, "f32", "f16", 64, 0)])
def test_embed_that_walks_the_tokens(n, V, D, kind, out, ids, pad):
    """More tokens than 2,048 workgroups have lanes for at once; the last four results are stored past the caches."""
    table = normal((V, D), TYPES[kind], n + D, pad)
    tok = some_tokens(n, V, n, torch.int32 if ids == 32 else torch.int64)
    assert D < 250 or n * D * (4 if out == "f32" else 2) > STREAM_BYTES
    view, check = guarded(n, D, TYPES[out])
    got = pqt.pqt_embed(table, tok, 11.3137085, out=view)
    t = tok.long()
    keep = (t >= 0) & (t < V)
    want = torch.where(keep[:, None], table.double()[t.clamp(0, V - 1)] * float(torch.tensor(11.3137085)), 0.0)
    within(got, want, want.abs() * U, "embed")
    check()


@gpu
@pytest.mark.parametrize("n,V,D,kind,tokens", [
    (600_001, 70_000, 9, "f32", "words"), (600_001, 3_000_000, 8, "bf16", "words"), (1_100_003, 500, 5, "f16", "words"), (600_001, 70_000, 8, "f32", "one"),
    (600_001, 70_000, 8, "f32", "high"), (600_001, 70_000, 8, "f32", "descending"), (300_007, 70_000, 160, "bf16", "words")])
def test_embed_gradient_of_many_places(n, V, D, kind, tokens):
    """Tiles of the sort with more places than its threads look at in one round; every place in one bucket of a digit, and other orders."""
    i = torch.arange(n, device=dev())
    tok = {"words": lambda: some_tokens(n, V, n), "one": lambda: torch.full_like(i, 41_234), "high": lambda: (i * 7919) % 300 + 40_960, "descending": lambda: (n - 1 - i) // 9}[tokens]()
    grad = normal((n, D), TYPES[kind], 3)
    want, size, count = base.gradient_reference(grad, tok, V, 0.37)       # on the CPU: atomics of 64 bits queue up at a frequent token
    view, check = guarded(V, D, torch.float32)
    got = pqt.pqt_embed_gradient(grad, tok, V, 0.37, out=view)
    base.within(got, want, (count + 2) * U * size, "gradient")
    assert not bool(got[(count[:, 0] == 0).to(dev())].any())
    check()
    assert torch.equal(pqt.pqt_embed_gradient(grad, tok, V, 0.37), got)
    old = normal((V, D), torch.float32, 9)
    held = pqt.pqt_embed_gradient(grad, tok, V, 0.37, out=old.clone(), accumulate=True)
    old = old.double().cpu()
    base.within(held, want + old, (count + 2) * U * size + U * (want.abs() + old.abs()), "accumulated")


# ---- layer norm ------------------------------------------------------------------------------------------------------
def large_inputs(rows, D, kind, pad):
    x = normal((rows, D), TYPES[kind], rows + D, pad, 1.5)
    x += normal((1, D), TYPES[kind], 5) * 2                       # columns with an offset
    return x, normal((1, D), torch.float32, 6)[0].contiguous(), normal((1, D), torch.float32, 7)[0].contiguous()


# a row by 8, 16, 32 and 64 lanes (1, 2 and 4 pieces), by 256 threads (2 and 4) and by 1,024 (2 and 4): more rows than the workgroups have at once
@gpu
@pytest.mark.parametrize("rows,D,kind,out,pad", [
    (70_001, 60, "f32", "f32", 0), (40_003, 128, "bf16", "f32", 1), (20_001, 250, "f16", "f16", 6), (9001, 500, "f32", "bf16", 0), (20_003, 960, "bf16", "bf16", 64),
    (9001, 2000, "bf16", "f32", 0), (5001, 4000, "bf16", "bf16", 3), (2501, 8100, "f32", "f32", 0), (1301, 16_000, "bf16", "bf16", 0), (700, 30_001, "f16", "f16", 1)])
def test_layer_norm_that_walks_the_rows(rows, D, kind, out, pad):
    x, w, b = large_inputs(rows, D, kind, pad)
    view, check = guarded(rows, D, TYPES[out])
    y, mean, rstd = pqt.pqt_layer_norm(x, w, b, 1e-5, out=view)
    x, w, b = x.double(), w.double(), b.double()
    m = x.mean(1, keepdim=True)
    var = ((x - m) ** 2).mean(1, keepdim=True)
    r = 1 / torch.sqrt(var + float(torch.tensor(1e-5)))
    h = (x - m) * r
    off = DEPTH * U * x.abs().mean(1, keepdim=True)               # of the mean
    spread = 2 * DEPTH * U + off ** 2 / var                       # of rstd, relative
    within(y, h * w + b, w.abs() * (r * off + spread * h.abs()) + 6 * U * ((w * h).abs() + b.abs()), "y")
    within(mean, m[:, 0], off[:, 0], "mean")
    within(rstd, r[:, 0], (spread * r)[:, 0], "rstd")
    check()


def test_layer_norm_results_past_the_caches():
    """Some of the results above are."""
    sizes = [mark.args[1] for mark in test_layer_norm_that_walks_the_rows.pytestmark if mark.name == "parametrize"][0]
    assert sum(rows * D * (4 if out == "f32" else 2) > STREAM_BYTES for rows, D, _, out, _ in sizes) >= 3


# a row by 8 to 64 lanes, by two, four and eight wavefronts; then rows that two kernels take: three rounds or more of every workgroup
@gpu
@pytest.mark.parametrize("rows,D,kind,pad", [
    (50_001, 60, "f32", 0), (30_001, 128, "bf16", 1), (15_001, 250, "f16", 0), (7001, 500, "f32", 3), (7001, 1000, "bf16", 0), (3503, 2000, "bf16", 8), (3503, 2047, "f32", 0),
    (1801, 4000, "bf16", 0), (1801, 4095, "f32", 1), (901, 8000, "f16", 0), (901, 8191, "f32", 0), (901, 12_000, "bf16", 2), (1100, 8200, "f32", 0), (1100, 16_387, "bf16", 5)])
def test_layer_norm_gradient_of_many_rows(rows, D, kind, pad):
    x, w, _ = large_inputs(rows, D, kind, pad)
    grad = normal((rows, D), TYPES[kind], 77, pad)
    _, mean, rstd = pqt.pqt_layer_norm(x, w)
    view, check = guarded(rows, D, TYPES[kind])
    dx, dw, db = pqt.pqt_layer_norm_gradient(grad, x, w, mean, rstd, out=view)
    x, G, w64, m, r = x.double(), grad.double(), w.double(), mean.double()[:, None], rstd.double()[:, None]
    h = (x - m) * r
    g = G * w64
    s1, s2 = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    # h: a difference and a product, 2 u of |h|; sums over the row as in DEPTH
    tol = r * (6 * U * (g.abs() + s1.abs() + (h * s2).abs()) + (DEPTH + 2) * U * g.abs().mean(1, keepdim=True) + (DEPTH + 5) * U * h.abs() * (g * h).abs().mean(1, keepdim=True))
    within(dx, r * (g - s1 - h * s2), tol, "dx")
    within(dw, (G * h).sum(0), (rows + 4) * U * (G * h).abs().sum(0), "dweight")
    within(db, G.sum(0), (rows + 1) * U * G.abs().sum(0), "dbias")
    check()


@gpu
@pytest.mark.parametrize("rows,D,kind", [(2, 1000, "bf16"), (16, 1000, "f32"), (17, 1000, "f16"), (129, 60, "f32"), (2, 8200, "f32"), (3, 16_385, "bf16")])
def test_layer_norm_gradient_of_few_rows_closely(rows, D, kind):
    test_layer_norm_gradient_of_many_rows(rows, D, kind, 0)


@gpu
@pytest.mark.parametrize("rows,D", [(70, 960), (2100, 4100), (30_001, 100)])
def test_layer_norm_bad_rows(rows, D):
    """A row with a NaN or an infinity is all NaN; its neighbours, and the rows that its group has before and after it, keep their bits."""
    x, w, b = large_inputs(rows, D, "bf16", 0)
    good = pqt.pqt_layer_norm(x, w, b)[0]
    at = [3, rows // 2, rows - 1]
    x[at[0], D // 2], x[at[1], 0], x[at[2], D - 1] = float("nan"), float("inf"), -float("inf")
    y = pqt.pqt_layer_norm(x, w, b)[0]
    bad = torch.zeros(rows, dtype=torch.bool, device=dev())
    bad[at] = True
    assert bool(y[bad].isnan().all()) and torch.equal(y[~bad], good[~bad])
