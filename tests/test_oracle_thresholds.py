"""Pins of what the oracle of sampling admits: exact where nothing is next to a threshold, both sides where a
threshold is an edge, and nothing else."""
import numpy as np
import pytest

from oracle import dense


def test_agrees_with_the_sampler_away_from_thresholds():
    rng = np.random.default_rng(1)
    checked = 0
    for i in range(400):
        v = int(rng.integers(1, 300))
        row = (3 * rng.standard_normal(v)).astype(np.float32)
        if i % 3 == 0:
            row = np.round(row)
        t, k = rng.choice([0.3, 1.0, 2.0]), int(rng.choice([0, 1, 5, 50]))
        p, m, u = rng.choice([1.0, 0.95, 0.5, 0.0]), rng.choice([0.0, 0.05]), rng.random()
        want = dense.sample(row, t, k, p, m, u, 1e-5)
        a = dense.admitted(row, t, k, p, m)
        if want.near:
            continue
        checked += 1
        assert a.fewest == a.most == want.kept
        assert a.fault(want.kept, want.token, want.prob, u) == ""
        assert a.fault(want.kept + 1, want.token, want.prob, u) and a.fault(want.kept - 1, want.token, want.prob, u)
        for other in range(v):
            # (a token of no weight has an empty stretch, which may lie at the mark: its own weight tells it apart)
            assert other == want.token or a.fault(want.kept, other, want.prob, u)
        assert "probability" in a.fault(want.kept, want.token, want.prob * (1 + 1e-5), u)
    assert checked > 250


def test_an_edge_admits_both_sides():
    a = dense.admitted(np.zeros(8, np.float32), 1.0, 0, 0.5, 0.0)
    assert (a.fewest, a.most) == (4, 5)  # 0.5 of eight equal weights is four of them, or a little more
    assert a.fault(4, 1, 0.25, 0.25) == "" and a.fault(4, 0, 0.25, 0.25) == "" and a.fault(4, 2, 0.25, 0.25)
    assert a.fault(5, 1, 0.2, 0.25) == "" and a.fault(5, 1, 0.25, 0.25) and a.fault(5, 2, 0.2, 0.25)
    assert a.fault(3, 0, 1 / 3, 0.25) and a.fault(6, 1, 1 / 6, 0.25)
    assert "not kept" in a.fault(4, 4, 0.25, 0.9999)


@pytest.mark.parametrize("top_p, kept", [(0.49, 4), (0.51, 5), (0.0, 1), (1.0, 8)])
def test_a_threshold_between_edges_admits_one_count(top_p, kept):
    a = dense.admitted(np.zeros(8, np.float32), 1.0, 0, top_p, 0.0)
    assert a.fewest == a.most == kept


def test_equal_logits_are_kept_by_index():
    row = np.array([1, 2, -0.0, 2, 0, 2, 0], np.float32)
    assert dense.admitted(row, 1.0, 2, 1.0, 0.0).order.tolist() == [1, 3]
    assert dense.admitted(row, 1.0, 5, 1.0, 0.0).order.tolist() == [1, 3, 5, 0, 2]
    a = dense.admitted(np.array([1.0, np.nan, -np.inf, 1.0], np.float32), 1.0, 0, 1.0, 0.0)
    assert a.order.tolist() == [0, 3] and a.fault(2, 1, 0.5, 0.5) and a.fault(2, 3, 0.5, 0.5) == ""


def test_mistakes_of_a_search_are_seen_in_long_rows():
    """One token more or fewer than the cut, a tie of the wrong index, a draw one token on: in rows as long as real ones
    the check that leaves rounding its room still tells them."""
    rng = np.random.default_rng(2)
    rows = {"zipf": -1.1 * np.log(np.arange(1, 60001.0))[rng.permutation(60000)], "flat": 0.01 * rng.standard_normal(60000),
            "steps": np.round(4 * rng.standard_normal(60000)) / 4}
    for name, row in rows.items():
        row = row.astype(np.float32)
        a = dense.admitted(row, 1.5, 0, 0.9, 0.0)
        want = dense.sample(row, 1.5, 0, 0.9, 0.0, 0.4321)
        assert a.most - a.fewest <= (1 if name != "zipf" else 8) and a.fewest <= want.kept <= a.most
        assert a.fault(want.kept, want.token, want.prob, 0.4321) == ""
        assert a.fault(a.fewest - 1, want.token, want.prob, 0.4321) and a.fault(a.most + 1, want.token, want.prob, 0.4321)
        kept = np.sort(a.order[:want.kept])
        i = int(np.searchsorted(kept, want.token))
        assert a.fault(want.kept, int(kept[i - 40]), want.prob, 0.4321) and a.fault(want.kept, int(kept[i + 40]), want.prob, 0.4321)
        dropped = np.setdiff1d(np.arange(60000), kept)
        assert "not kept" in a.fault(want.kept, int(dropped[0]), want.prob, 0.4321)
