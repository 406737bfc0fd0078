"""The query encoder's layers where calls are unusual: places that do not ascend, and what the tests beside these leave out.

References and tolerances are those of test_query_encoder_layers.py."""
import math

import pytest
import torch

import test_query_encoder_layers as base
from test_query_encoder_layers import INF, LEAST, TYPES, U, UNIT, arguments, attention_inputs, dev, gpu, guarded, normal, pqt, within


def ptr(t):
    return None if t is None else t.data_ptr()


def places(kind, texts, n, seed):
    g = torch.Generator().manual_seed(seed)
    at = torch.randint(0, n + 1, (texts + 1,), generator=g)
    if kind == "descending":
        at = at.sort(descending=True)[0]
    elif kind == "one out of place":
        at = at.sort()[0]
        at[texts // 3] = n
    elif kind == "out of range":
        at = at * 3 - n
    return at


@gpu
@pytest.mark.parametrize("kind", ["descending", "permuted", "one out of place", "out of range"])
@pytest.mark.parametrize("texts,n", [(210, 2277), (70, 900), (100, 9000), (5000, 6000)])
def test_places_in_any_order_stay_inside(kind, texts, n):
    """More texts than a look sees, in any order, rows of none cleared: nothing outside the results is written (which rows are, is not defined)."""
    heads, kv, d = 4, 2, 32
    x = normal((n, (heads + 2 * kv) * d), torch.bfloat16, 1)
    q, k, v = x[:, :heads * d], x[:, heads * d:(heads + kv) * d], x[:, (heads + kv) * d:]
    at = places(kind, texts, n, 7).to(dev())
    bias, distances = normal((heads, 32), torch.float32, 3), pqt.pqt_distance_buckets(32, 128, device=dev())
    out, check = guarded(n, heads * d, torch.bfloat16)
    sums = torch.full((heads * n + 64,), 7.0, device=dev())
    stream = torch.cuda.current_stream().cuda_stream
    layout = (at.data_ptr(), None, 8, texts, d ** -0.5, ptr(bias), 32, ptr(distances), 128, 1)
    pqt._check(pqt._lib.pqt_attention(ptr(q), x.stride(0), ptr(k), x.stride(0), ptr(v), x.stride(0), pqt.PQT_BF16, n, heads, kv, d, *layout, ptr(out), out.stride(0),
                                      sums.data_ptr() + 128, 0, stream))
    check()
    assert bool((sums[:32] == 7.0).all()) and bool((sums[32 + heads * n:] == 7.0).all())
    lse = torch.zeros((heads, n), device=dev())                    # (rows of no text the forward pass found hold anything)
    grads, check = guarded(n, (heads + 2 * kv) * d, torch.bfloat16)
    parts = grads[:, :heads * d], grads[:, heads * d:(heads + kv) * d], grads[:, (heads + kv) * d:]
    step = grads.stride(0)
    dbias, need = torch.empty_like(bias), pqt.pqt_attention_gradient_workspace(n, texts, heads, kv, d, 128)
    ws = torch.full((need + 512,), 7, dtype=torch.uint8, device=dev())
    pqt._check(pqt._lib.pqt_attention_gradient(ptr(q), x.stride(0), ptr(q), x.stride(0), ptr(k), x.stride(0), ptr(v), x.stride(0), ptr(q), x.stride(0), ptr(lse), pqt.PQT_BF16, n, heads, kv, d,
                                               *layout, ptr(parts[0]), step, ptr(parts[1]), step, ptr(parts[2]), step, ptr(dbias), ws.data_ptr() + 256, need, 0, stream))
    check()
    assert bool((ws[:256] == 7).all()) and bool((ws[256 + need:] == 7).all())


# ---- large finite biases ---------------------------------------------------------------------------------------------
FAR = [-1e6, -1e8, -1e9, -1e10, -1e12, 1e12, 1e30, torch.finfo(torch.float32).min]
TEXTS = [[20, 1, 0, 33], [70, 3, 1, 60], [300] * 16, [2100, 2050]]     # short texts, workgroups of 64 and of 128 rows, far steps in runs


def counted(s, value):
    """What a bias counts as: finite bias / scale within 2^90."""
    return max(-2.0 ** 90, min(value / s.scale, 2.0 ** 90)) * s.scale


def between(s, out, lse, value, uniform):
    """Whatever the rounding of logits beside such a bias leaves of their differences, results are means of v: weights that are not negative and add up to one."""
    unit = base.weight_unit(s.q.dtype) * 1.01
    for at, m in zip(s.at, s.of):
        if not m:
            continue
        v = s.v[at:at + m].double()
        off = (m + 16) * U * v.abs().amax(0) + unit * v.abs().amax(0)
        off = off + v.abs().amax(0) * UNIT[s.q.dtype] * 1.01 + LEAST[s.q.dtype]
        got = out[at:at + m].double()
        assert bool((got <= v.amax(0) + off).all() and (got >= v.amin(0) - off).all())
        if uniform:
            want = v.mean(0, keepdim=True).expand(m, -1)
            within(out[at:at + m], want, ((m + 16) * U + unit) * v.abs().mean(0, keepdim=True).expand(m, -1), "mean")
        z = torch.stack([s.q[at:at + m, h * s.d:(h + 1) * s.d].double() @ s.k[at:at + m, h * s.d:(h + 1) * s.d].double().t() for h in range(s.heads)]).abs().amax() * s.scale
        want = counted(s, value)
        assert bool(((lse[:, at:at + m].double() - want).abs() <= float(z) + math.log(m) + abs(want) * 16 * U).all())


@gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d", [32, 64, 80])
@pytest.mark.parametrize("lengths", TEXTS, ids=lambda t: f"{len(t)}x{max(t)}")
def test_one_far_bias_for_all(kind, d, lengths):
    """A bias beside which logits are rounded, the same for all places.  From 1e9 on (bias / scale above 2^32, whose numbers are 512 apart) products below 2^8 vanish: equal weights."""
    s = attention_inputs(lengths, 8, 8, d, kind, 0, 0)
    s.bias, s.distances, s.reach = torch.zeros((8, 1), device=dev()), torch.zeros(1, dtype=torch.int32, device=dev()), 0
    size = lambda t: float(t.double().unflatten(1, (8, d)).square().sum(2).amax().sqrt())               # noqa: E731
    assert size(s.q) * size(s.k) < 2 ** 8
    for value in FAR:
        s.bias.fill_(value)
        out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
        between(s, out, lse, value, abs(value) >= 1e9)


@gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d", [32, 64, 80])
@pytest.mark.parametrize("lengths", TEXTS, ids=lambda t: f"{len(t)}x{max(t)}")
def test_one_key_left_with_a_far_bias(kind, d, lengths):
    """All places masked but the query's own, whose bias is far: its value is the result.  And all but those behind: the last token has none, the one before it the last."""
    s = attention_inputs(lengths, 8, 8, d, kind, 2, 1)
    for value in FAR + [-1e4, 5.0]:
        s.bias = torch.tensor([[value, -INF]] * 8, device=dev())
        s.distances = torch.tensor([1, 0, 1], dtype=torch.int32, device=dev())
        out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
        want = s.v.double()
        within(out, want, want.abs() * 8 * U, "own value")
        assert bool(lse.isfinite().all())
        s.distances = torch.tensor([1, 1, 0], dtype=torch.int32, device=dev())
        out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
        for at, m in zip(s.at, s.of):
            if m:
                assert bool((lse[:, at + m - 1] == -INF).all()) and not bool(out[at + m - 1].any())
            if m > 1:
                last = s.v[at + m - 1:at + m].double()
                within(out[at + m - 2:at + m - 1], last, last.abs() * 8 * U, "last value")
                assert bool(out[at:at + m].isfinite().all()) and bool(lse[:, at:at + m - 1].isfinite().all())


@gpu
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_products_far_below_zero(kind):
    """A single token whose logit is -1e30 or so has all of the weight, as one of any size has."""
    x = torch.full((3, 64), 1e14, dtype=TYPES[kind], device=dev())
    v = normal((3, 64), TYPES[kind], 1)
    starts = torch.arange(4, device=dev())
    out, lse = pqt.pqt_attention(x, -x, v, starts, 1)
    assert torch.equal(out, v) and bool((lse < -1e28).all())


def mean_gradient(s, grad, out, got, share):
    """Against the formula with the weights share(text's tokens) given, as large biases leave them: one weight of its row's is exact to 8 U."""
    dq, dk, dv, dbias = got
    unit, small = base.weight_unit(s.q.dtype) * 1.01, 2.0 ** -32 if s.q.dtype == torch.float16 else 0.0
    scale = torch.tensor(s.scale, dtype=torch.float32).double().item()
    names = ("dq", "dk", "dv")
    want, tol = [[torch.zeros(s.n, s.heads * s.d, dtype=torch.float64, device=dev()) for _ in names] for _ in range(2)]
    want_b, tol_b = [torch.zeros(s.heads, s.bias.shape[1], dtype=torch.float64, device=dev()) for _ in range(2)]
    for at, m in zip(s.at, s.of):
        if not m:
            continue
        p, bucket = share(m)
        for h in range(s.heads):
            rows, columns = slice(at, at + m), slice(h * s.d, (h + 1) * s.d)
            q, k, v, g, o = (t[rows, columns].double() for t in (s.q, s.k, s.v, grad, out))
            ds = p * (g @ v.t() - (g * o).sum(1, keepdim=True))
            off = ds.abs() * (m + 12) * U + p * 1.01 * (s.d + 6) * U * (g.abs() @ v.abs().t() + (g.abs() * o.abs()).sum(1, keepdim=True)) + 2.0 ** -120
            row = off + ds.abs() * unit + small * ds.abs().amax(1, keepdim=True)
            key = off + ds.abs() * unit + small * ds.abs().amax(0, keepdim=True)
            add = (m + 8) * U
            for i, (w, e) in enumerate(((scale * ds @ k, scale * (row + ds.abs() * add) @ k.abs()), (scale * ds.t() @ q, scale * (key + ds.abs() * add).t() @ q.abs()),
                                        (p.t() @ g, (p * ((m + 12) * U + unit + add) + small + 2.0 ** -120).t() @ g.abs()))):
                want[i][rows, columns], tol[i][rows, columns] = w, e
            for b in range(s.bias.shape[1]):
                want_b[h, b] += ds[bucket == b].sum()
                tol_b[h, b] += (off + ds.abs() * (m + 2 * s.reach + 64 + len(s.of)) * U)[bucket == b].sum()
    for name, a, w, e in zip(names, got, want, tol):
        within(a, w, e, name)
    within(dbias, want_b, tol_b, "dbias")


def rows_add_up(s, grad, got):
    """Every row's weights add up to one, whatever they are: dv's sum over the keys is grad's over the queries, and dbias' over all buckets nothing."""
    unit = base.weight_unit(s.q.dtype) * 1.01
    for at, m in zip(s.at, s.of):
        if not m:
            continue
        g, dv = grad[at:at + m].double(), got[2][at:at + m].double()
        off = g.abs().sum(0) * ((2 * m + 24) * U + unit) + dv.abs().sum(0) * UNIT[s.q.dtype] * 1.01 + m * (LEAST[s.q.dtype] + 2.0 ** -24 * g.abs().amax(0))
        assert bool(((dv.sum(0) - g.sum(0)).abs() <= off).all()), float(((dv.sum(0) - g.sum(0)).abs() - off).amax())
    assert all(bool(t.isfinite().all()) for t in got)


@gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d", [32, 64, 80, 128])
@pytest.mark.parametrize("lengths", TEXTS, ids=lambda t: f"{len(t)}x{max(t)}")
def test_gradient_of_one_far_bias_for_all(kind, d, lengths):
    """A bias beside which logits are rounded, the same for all places: their weights add up to one, and are equal from 1e9 on."""
    s = attention_inputs(lengths, 8, 8, d, kind, 0, 0)
    s.bias, s.distances, s.reach = torch.zeros((8, 1), device=dev()), torch.zeros(1, dtype=torch.int32, device=dev()), 0
    grad = normal((s.n, 8 * d), TYPES[kind], 5)
    for value in [-4e3, -1e4, -1e5] + FAR:                         # (lse is so large that both kernels take rows' sums anew)
        s.bias.fill_(value)
        out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
        got = pqt.pqt_attention_gradient(grad, s.q, s.k, s.v, out, lse, s.starts, **arguments(s))
        rows_add_up(s, grad, got)
        if abs(value) >= 1e9:
            mean_gradient(s, grad, out, got, lambda m: (torch.full((m, m), 1.0 / m, dtype=torch.float64, device=dev()), torch.zeros((m, m), device=dev())))


@gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d", [32, 64, 80, 128])
@pytest.mark.parametrize("lengths", TEXTS, ids=lambda t: f"{len(t)}x{max(t)}")
def test_gradient_of_one_key_left_with_a_far_bias(kind, d, lengths):
    """All places masked but the query's own, whose bias is far: dv is grad, and nothing else has a gradient."""
    s = attention_inputs(lengths, 8, 8, d, kind, 2, 1)
    s.distances = torch.tensor([1, 0, 1], dtype=torch.int32, device=dev())
    grad = normal((s.n, 8 * d), TYPES[kind], 5)
    for value in FAR + [-1e4]:
        s.bias = torch.tensor([[value, -INF]] * 8, device=dev())
        out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
        got = pqt.pqt_attention_gradient(grad, s.q, s.k, s.v, out, lse, s.starts, **arguments(s))
        mean_gradient(s, grad, out, got, lambda m: (torch.eye(m, dtype=torch.float64, device=dev()), 1 - torch.eye(m, device=dev())))


@gpu
@pytest.mark.parametrize("kind", TYPES)
def test_gradient_of_far_rows_beside_others(kind):
    """Heads whose biases are all 1e5 lower beside ordinary ones, shared key heads, a padded batch, workgroups that share a key's queries: the ordinary heads' gradients are the
    same bytes as without them, and the lower ones' weights add up to one a row."""
    s = attention_inputs([900, 1, 0, 40], 8, 2, 64, kind, 32, 40, 901)
    grad = torch.nan_to_num(normal((s.n, 512), TYPES[kind], 5))
    out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
    plain = pqt.pqt_attention_gradient(grad, s.q, s.k, s.v, out, lse, s.starts, **arguments(s))
    s.bias[:4] -= 1e5                                              # the heads of the first keys' head
    far, far_lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
    got = pqt.pqt_attention_gradient(grad, s.q, s.k, s.v, far, far_lse, s.starts, **arguments(s))
    base.check_attention(s, far, far_lse)
    for a, b, w in zip(got, plain, (256, 64, 64)):
        assert torch.equal(a[:, w:], b[:, w:])
    assert torch.equal(got[3][4:], plain[3][4:])
    assert bool((far_lse[:4][lse[:4].isfinite()] < -9e4).all())
    for at, m in zip(s.at, s.of):                                  # four heads' weights add up to four
        if m:
            g, dv = grad[at:at + m, :256].double().unflatten(1, (4, 64)), got[2][at:at + m, :64].double()
            off = g.abs().sum((0, 1)) * ((2 * m + 40) * U + base.weight_unit(s.q.dtype) * 1.01) + dv.abs().sum(0) * UNIT[s.q.dtype] * 1.01 + m * 2.0 ** -20
            assert bool(((dv.sum(0) - g.sum((0, 1))).abs() <= off).all())


# ---- results that the call makes beside the caller's -----------------------------------------------------------------
@gpu
@pytest.mark.parametrize("given", [(0,), (1,), (2,), (0, 2), (1, 2), (), (0, 1, 2)])
def test_gradients_some_of_which_the_call_makes(given):
    """Of three results some are the caller's, whose rows of no text stay as they were, the others the call's own, whose are zeros."""
    s = attention_inputs([20, 0, 90], 4, 2, 48, "bf16", 32, 20, 0, 0, 64, 70, 1, 30)
    grad = torch.nan_to_num(normal((s.n, 192), torch.bfloat16, 5))
    out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
    want = pqt.pqt_attention_gradient(grad, s.q, s.k, s.v, out, lse, s.starts, **arguments(s))
    held = [torch.full((s.n, w), 7.0, dtype=torch.bfloat16, device=dev()) if i in given else None for i, w in enumerate((192, 96, 96))]
    left = [torch.full((s.n, w), float("nan"), dtype=torch.bfloat16, device=dev()) for w in (192, 96, 96) for _ in range(8)]
    del left                                                       # what the allocator hands out next
    got = pqt.pqt_attention_gradient(grad, s.q, s.k, s.v, out, lse, s.starts, grads=held, **arguments(s))
    a, b = s.at[0], s.at[-1]
    for i in range(3):
        assert torch.equal(got[i][a:b], want[i][a:b])
        rest = torch.cat([got[i][:a], got[i][b:]])
        assert bool((rest == (7.0 if i in given else 0.0)).all()) and (held[i] is None or got[i] is held[i])
    assert torch.equal(got[3], want[3])


@gpu
def test_gradients_are_three_or_none():
    x = torch.zeros((4, 8), device=dev())
    at, lse = torch.tensor([0, 4], device=dev()), torch.zeros((2, 4), device=dev())
    for grads in ((x,), (x, x), (x, x, x, x)):
        with pytest.raises(ValueError):
            pqt.pqt_attention_gradient(x, x, x, x, x, lse, at, 2, grads=grads)


# ---- sizes past 32 bits ----------------------------------------------------------------------------------------------
def test_bias_of_more_buckets_or_distances_than_32_bits():
    """2^32 + 4 buckets are not four, nor as many distances five."""
    meta = torch.device("meta")
    of = lambda buckets, distances: (torch.empty((2, buckets), device=meta), torch.empty(distances, dtype=torch.int32, device=meta))       # noqa: E731
    for bias, distances in (of(2 ** 32 + 4, 5), of(4, 2 ** 32 + 5)):
        with pytest.raises(pqt.PqtError) as e:
            pqt._bias(bias, distances, 2, meta)
        assert e.value.code == pqt.PQT_EUNSUPPORTED
    assert pqt._bias(*of(4, 5), 2, meta)[1::2] == (4, 2)


def test_workspace_of_more_heads_than_32_bits():
    for args in ((100, 2, 2 ** 32 + 4, 4, 64, -1), (100, 2, 4, 2 ** 32 + 4, 64, -1), (100, 2, 4, 4, 2 ** 32 + 64, -1), (100, 2, 4, 4, 64, 2 ** 32), (100, 2, 4 - 2 ** 32, 4, 64, 0)):
        assert pqt.pqt_attention_gradient_workspace(*args) == 0
    assert pqt.pqt_attention_gradient_workspace(100, 2, 4, 4, 64, -1) > 0


@gpu
def test_rows_of_more_values_than_32_bits():
    """A row of 2^32 + 64 values is one head of too many, not of 64."""
    x, at = torch.empty((1, 2 ** 32 + 64), dtype=torch.bfloat16, device=dev()), torch.tensor([0, 1], device=dev())
    for heads in (1, 2 ** 31 + 32):
        with pytest.raises(pqt.PqtError) as e:
            pqt.pqt_attention(x, x, x, at, heads)
        assert e.value.code == pqt.PQT_EUNSUPPORTED


MIXED = [c for c in base.ATTENTION if c[5] and 1 < sum(c[0]) <= 5000]


@gpu
@pytest.mark.parametrize("case", MIXED, ids=lambda c: f"{len(c[0])}x{max(c[0])}-" + "-".join(map(str, c[1:])))
def test_rows_that_a_far_bias_leaves_among_others(case):
    """A mask of -2e4 on the query itself and all behind it, as training code has it in place of -inf: a text's first token has nothing else, the others do.  Logits there are off by
    some 2e4 * 8 U, a weight by a hundredth: the formula tells what is right."""
    lengths, heads, kv, d, kind, buckets, reach, padded, pad, ids, behind = case
    s = attention_inputs(lengths, heads, kv, d, kind, buckets, reach, padded, pad, ids, behind)
    s.bias[:, s.distances[s.distances.shape[0] // 2:].unique().long()] -= 2e4
    out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
    base.check_attention(s, out, lse)
    grad = torch.full((s.n, heads * d + pad), float("nan"), dtype=TYPES[kind], device=dev())[:, :heads * d]
    for at, m in zip(s.at, s.of):
        grad[at:at + m] = normal((m, heads * d), TYPES[kind], 77 + m, 0, 0.01)
        assert m == 0 or bool((lse[:, at] < -1.9e4).all())
    got = pqt.pqt_attention_gradient(grad, s.q, s.k, s.v, out, lse, s.starts, **arguments(s))
    base.check_gradient(s, grad, out, lse, got)
    again = pqt.pqt_attention_gradient(grad, s.q, s.k, s.v, out, lse, s.starts, **arguments(s))
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@gpu
def test_far_rows_in_a_graph():
    """A captured gradient of such rows, replayed with other inputs and with none of them."""
    s = attention_inputs([300, 1, 0, 77], 4, 2, 64, "bf16", 32, 40)
    grad = torch.nan_to_num(normal((s.n, 256), torch.bfloat16, 5))
    biases = [s.bias.clone(), s.bias - 1e9, s.bias.clone()]
    biases[2][:, :16] = torch.finfo(torch.float32).min

    def both():
        out, lse = pqt.pqt_attention(s.q, s.k, s.v, s.starts, **arguments(s))
        return (out, lse) + pqt.pqt_attention_gradient(grad, s.q, s.k, s.v, out, lse, s.starts, **arguments(s))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for bias in biases + biases[::-1]:
        s.bias.copy_(bias)
        want = [t.clone() for t in both()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)) and all(bool(t.isfinite().all()) for t in want)
