"""The query encoder's layers at sizes where every kernel is past its first round: groups of lanes that walk their rows, texts of more rows than two tiles in fp32, more texts than
two looks see, and more workgroups than a run of the joining kernel has rows.

References and tolerances are those of test_query_encoder_layers.py."""
import pytest
import torch

import test_query_encoder_layers as base
from test_query_encoder_layers import gpu

# rows, D, type, y's type, weight's type, residual, pad: more rows than all groups of a launch take at once (2,048 workgroups of 256 threads, 512 of 1,024)
WALK = [(70_001, 60, "bf16", "bf16", "bf16", True, 0), (33_001, 100, "f16", "f32", "f32", True, 4), (17_003, 200, "f32", "f32", "f32", False, 0), (17_003, 250, "bf16", "bf16", None, True, 1),
        (9_001, 500, "f16", "f16", "f16", True, 0), (9_001, 1000, "bf16", "bf16", "bf16", True, 0), (8_300, 2000, "f32", "bf16", "f32", True, 3), (2_501, 4000, "f16", "f16", "bf16", False, 0),
        (2_501, 8100, "bf16", "bf16", "bf16", True, 0), (1_100, 16_001, "f32", "f32", "f32", True, 0), (1_037, 30_001, "bf16", "bf16", "f32", True, 0)]
# of the gradient: 256 workgroups of 512 threads
WALK_BACK = [(50_001, 60, "bf16", None, "bf16", True, 0), (20_001, 100, "f32", None, "f32", True, 4), (9_001, 250, "f16", None, None, False, 1), (5_000, 500, "bf16", None, "f32", True, 0),
             (7_001, 1000, "bf16", None, "bf16", True, 0), (5_003, 1024, "f32", None, "f32", False, 0), (3_503, 2047, "f16", None, "f16", True, 3), (1_801, 4095, "bf16", None, "bf16", True, 0),
             (901, 8191, "f32", None, "f32", True, 0), (901, 12_000, "bf16", None, "bf16", True, 0), (1_100, 16_387, "bf16", None, "bf16", True, 0), (700, 9_001, "f32", None, "f32", True, 0),
             # one workgroup, whose groups have two rows each
             (100, 60, "bf16", None, "f32", True, 0), (13, 1000, "f32", None, "f32", True, 0), (7, 2000, "f16", None, "f16", True, 0), (3, 4000, "bf16", None, "bf16", True, 0),
             (2, 8000, "f32", None, "f32", True, 0)]


def size_of(case):
    return f"{case[0]}x{case[1]}-{case[2]}"


@gpu
@pytest.mark.parametrize("case", WALK, ids=size_of)
def test_rms_norm_that_walks_the_rows(case):
    base.test_rms_norm(*case)


@gpu
@pytest.mark.parametrize("case", WALK_BACK, ids=size_of)
def test_rms_norm_gradient_of_many_rows(case):
    base.test_rms_norm_gradient(*case)


LONG = [  # lengths, heads, heads of keys, d, type, buckets, reach, padded to, pad, ids, rows behind: fp32, whose bounds tell every tile and step apart
    ([4100], 12, 12, 32, "f32", 32, 128, 0, 0, 64, 0), ([4100], 12, 4, 64, "f32", 32, 128, 0, 0, 64, 0), ([4100], 12, 12, 96, "f32", 20, 40, 0, 0, 64, 2), ([4100], 12, 2, 128, "f32", 32, 448, 0, 0, 64, 0),
    ([2100, 1900], 16, 16, 64, "f32", 0, 0, 0, 0, 64, 0), ([2100, 1900], 16, 8, 96, "f32", 0, 0, 2100, 0, 32, 0), ([1, 4300], 16, 4, 32, "f32", 32, 128, 0, 0, 64, 0),
    ([4200], 12, 12, 60, "f32", 32, 128, 0, 1, 64, 0), ([4200], 12, 3, 90, "f32", 6, 2, 0, 0, 64, 0), ([2100, 2110], 12, 12, 127, "f32", 32, 128, 0, 0, 64, 1)]


def name_of(case):
    return f"{len(case[0])}x{max(case[0])}-" + "-".join(map(str, case[1:]))


@gpu
@pytest.mark.parametrize("case", LONG, ids=name_of)
def test_attention_of_long_texts_in_fp32(case):
    base.test_attention(case)


@gpu
@pytest.mark.parametrize("case", LONG, ids=name_of)
def test_attention_gradient_of_long_texts_in_fp32(case):
    base.test_attention_gradient(case)


def many(texts, most):
    return torch.randint(0, most + 1, (texts,), generator=torch.Generator().manual_seed(texts)).tolist()


MANY = [(many(6000, 16), 1, 1, 32, "f32", 4, 3, 0, 0, 64, 40), (many(4500, 7), 2, 1, 16, "bf16", 2, 5, 7, 0, 32, 0)]


@gpu
@pytest.mark.parametrize("case", MANY, ids=name_of)
def test_attention_of_thousands_of_texts(case):
    """Three looks at the starts, empty texts among them; more than 8,192 workgroups, so that each run of the joining kernel has more rows than a round of it."""
    base.test_attention(case)


@gpu
@pytest.mark.parametrize("case", MANY, ids=name_of)
def test_attention_gradient_of_thousands_of_texts(case):
    base.test_attention_gradient(case)
