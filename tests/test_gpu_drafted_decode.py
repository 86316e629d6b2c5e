"""The drafting operators together (examples/drafted_decode.py): greedy rows produce what they do without
drafts, the cache's counts stay those of its tables, forked and ended rows leave the others as they were."""
import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "drafted_decode.py")
    spec = importlib.util.spec_from_file_location("drafted_decode", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _counts_match(d):
    held = np.concatenate([d.table.cpu().numpy().ravel(), d.prompt_table.cpu().numpy().ravel()])
    want = np.bincount(held[held >= 0], minlength=d.pages)
    assert np.array_equal(want, d.refs.cpu().numpy())


@pytest.mark.parametrize("seed", [0, 1])
def test_greedy_rows_do_not_depend_on_the_drafts(gpu_lib, seed):
    ex = _example()
    d, drafted, accepted = ex.run(draft=3, steps=10, seed=seed)
    plain, alone, none = ex.run(draft=0, steps=10, seed=seed)
    assert none == 0 and 0 < accepted < 3
    _counts_match(d)
    for r in range(0, d.R, d.rpg):
        n = min(len(drafted[r]), len(alone[r]))
        assert n >= 10 and drafted[r][:n] == alone[r][:n]
    assert [len(x) for x in alone] == [10] * plain.R


def test_rows_fork_and_end(gpu_lib):
    ex = _example()
    d, _, _ = ex.run(draft=3, steps=5, seed=2)
    twin, _, _ = ex.run(draft=3, steps=5, seed=2)
    d.fork(0, 1)
    _counts_match(d)
    assert int(d.refs.max()) == 2
    a, b = d.step()[0], twin.step()[0]
    assert a[0].tolist() == b[0].tolist() and a[3:].tolist() == b[3:].tolist()  # (a fork takes nothing from the others)
    _counts_match(d)
    live = d.end([2, 4])
    assert live == int((d.refs > 0).sum()) and int((d.refs[live:] != 0).sum()) == 0
    _counts_match(d)
    a, b = d.step()[0], twin.step()[0]
    assert a[0].tolist() == b[0].tolist() and a[3].tolist() == b[3].tolist() and a[2].tolist() == [-1] * 4
    d.check()
