"""Which rows a workgroup of attention has: the search among the texts' starts, on the CPU."""
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def workgroups(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("host") / "text_rows")
    res = subprocess.run(["g++", "-std=c++17", "-O1", os.path.join(ROOT, "tests", "host", "text_rows.cpp"), "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr

    def run(cases):
        """Of every (M, n, clear, starts, lengths or None), its workgroups' (begin, span, len, row0, mine, text, before)."""
        lines = "".join(f"{M} {n} {int(clear)} {int(lengths is not None)} {len(starts) - 1} " + " ".join(map(str, starts + (lengths or []))) + "\n" for M, n, clear, starts, lengths in cases)
        out = iter(subprocess.run([exe], input=lines, capture_output=True, text=True, check=True).stdout.splitlines())
        return [[tuple(int(v) for v in next(out).split()) for _ in range(n // M + len(starts))] for M, n, _, starts, _ in cases]
    return run


def ranges(M, row):
    """What a workgroup clears as rows of no text, and what it has of a text's rows, as (from, to)."""
    begin, span, _, row0, mine, text, before = row
    if not mine:
        return (0, 0), (0, 0)
    cleared = (0, 0)
    if before or not text:                                         # as the kernels have it
        cleared = (begin - before if before else begin + row0, begin if before and text else min(begin + row0 + M, begin + span))
    return cleared, (begin + row0, min(begin + row0 + M, begin + span)) if text else (0, 0)


def lists(ascending, count, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda lo, hi: int(torch.randint(lo, hi + 1, (1,), generator=g))                                 # noqa: E731
    for i in range(count):
        texts, n = (r(0, 5), r(1, 100)) if i % 3 == 0 else (r(60, 70), r(1, 900)) if i % 3 == 1 else (r(100, 300), r(1, 4000))
        starts = [r(0, n) for _ in range(texts + 1)]
        kind = i % 4
        if ascending or kind == 0:
            starts.sort()
            if not ascending:                                      # one of them out of its place
                starts[r(0, texts)] = r(0, n)
        elif kind == 1:
            starts.sort(reverse=True)
        elif kind == 2:
            starts = [v * 3 - n for v in starts]                   # out of range, too
        yield (16, 64, 128)[r(0, 2)], n, r(0, 1), starts, [r(-3, 2 * n) for _ in range(texts)] if r(0, 1) else None


def test_rows_of_ascending_texts(workgroups):
    """Every row of every text belongs to one workgroup of that text, every row of none is cleared by one where that is asked for."""
    cases = list(lists(True, 300, 1))
    for (M, n, clear, starts, lengths), rows in zip(cases, workgroups(cases)):
        seen, cleared = [None] * n, [0] * n
        for row in rows:
            (a, b), (c, d) = ranges(M, row)
            for i in range(a, b):
                cleared[i] += 1
            for i in range(c, d):
                assert seen[i] is None
                seen[i] = (row[0], row[1], row[2])
        of = [None] * n
        for s, (a, b) in enumerate(zip(starts, starts[1:])):
            for i in range(a, b):
                of[i] = (a, b - a, min(b - a, max(0, lengths[s])) if lengths is not None else b - a)
        assert seen == of
        assert cleared == [int(clear and v is None) for v in of]


def test_rows_of_any_places_stay_inside(workgroups):
    """Places that descend, in no order or out of range: whatever a workgroup takes for its rows lies within the n there are."""
    cases = list(lists(False, 900, 2)) + [(16, 2277, 1, [2277 - 10 * i for i in range(211)], None)]
    for (M, n, _, starts, _), rows in zip(cases, workgroups(cases)):
        for t, row in enumerate(rows):
            begin, span, length, row0, mine, _, _ = row
            if mine:
                assert 0 <= begin and 0 <= span and begin + span <= n and 0 <= length <= span and 0 <= row0 <= span, (M, n, t, row)
            for a, b in ranges(M, row):
                assert 0 <= a and b <= n, (M, n, t, row)
