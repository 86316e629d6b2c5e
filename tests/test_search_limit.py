"""The search for a row's cut ends well within its limit of passes: the arithmetic of its ranges, pass by pass, for the
widest keys and the worst first range."""
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BINS = 512


def _passes(first, last, cut, lowest):
    """Passes until a range [first, last] of keys that holds `cut` is one value; ranges as the kernel moves them."""
    n = 0
    while True:
        n += 1
        wider = 8 * (last - first) + 8 if last - first < 0x0fffffff else 0xffffffff
        if cut < first:
            first, last = (first - wider if first > wider else 0), first - 1
        elif cut > last:
            first, last = last + 1, (last + wider if lowest - last > wider else lowest)
        else:
            shift = 0
            while (last - first) >> shift >= BINS:
                shift += 1
            if shift == 0:
                return n
            start = first + ((cut - first) >> shift << shift)
            first, last = start, min(last, start + (1 << shift) - 1)


@pytest.mark.parametrize("bits", [16, 32])
def test_a_search_ends_within_its_limit(bits):
    lowest = (1 << bits) - 1
    edges = sorted({0, 1, 7, 8, 9, 511, 512, 513, lowest // 3, lowest // 2, lowest - 513, lowest - 1, lowest})
    most = 0
    for a in edges:
        for b in edges:
            if b < a:
                continue
            for cut in edges:
                most = max(most, _passes(a, b, cut, lowest))
    # a search by count, one pass more where S ends before k, and a search by mass from the largest logit on
    total = most + 1 + max(_passes(0, c, c, lowest) for c in edges)
    limit = int(re.search(r"kMostRounds = (\d+)", open(os.path.join(ROOT, "paper_2607_20791_gb300", "csrc", "sample_top.cu")).read()).group(1))
    said = int(re.search(r"\((\d+) passes are enough", open(os.path.join(ROOT, "include", "rgd.h")).read()).group(1))
    assert total <= said <= limit // 2, (most, total)
