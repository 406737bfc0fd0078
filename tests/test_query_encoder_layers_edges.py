"""The query encoder's layers where calls are unusual: places that do not ascend, and what the tests beside these leave out.

References and tolerances are those of test_query_encoder_layers.py."""
import pytest
import torch

import test_query_encoder_layers as base
from test_query_encoder_layers import INF, TYPES, dev, gpu, guarded, normal, pqt


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
