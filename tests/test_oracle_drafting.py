"""Pins of the drafting oracle: verification, 4-bit products, cache pages."""
import numpy as np
import pytest
from scipy.special import softmax

from oracle import drafting


def _rows(seed, n, vocab):
    rng = np.random.default_rng(seed)
    return rng.normal(0, 2, (n, vocab)).astype(np.float32)


def test_probabilities_are_the_truncated_softmax():
    row = _rows(0, 1, 50)[0]
    assert np.allclose(drafting.probabilities(row, 1.5, 0.0), softmax(row.astype(np.float64) / np.float32(1.5)), rtol=1e-13)
    p = drafting.probabilities(row, 1.0, 0.1)
    full = softmax(row.astype(np.float64))
    assert np.array_equal(p > 0, full >= np.float32(0.1) * full.max())
    assert abs(p.sum() - 1) < 1e-12
    row[3] = np.nan
    assert drafting.probabilities(row, 1.0, 0.0)[3] == 0


@pytest.mark.parametrize("certain", [False, True])
@pytest.mark.parametrize("min_p", [0.0, 0.2])
def test_first_token_is_distributed_as_the_target(certain, min_p):
    """P(emit x) = q(x) min(1, p(x) / q(x)) + P(reject) rest(x) = p(x): the uniforms' measure is summed
    exactly over a grid of acceptance and draw uniforms that resolves every step."""
    vocab, T = 5, 1.3
    t, d = _rows(1, 2, vocab), _rows(2, 1, vocab)
    p = drafting.probabilities(t[0], T, min_p)
    q = drafting.probabilities(d[0], T, min_p)
    got, N = np.zeros(vocab), 400
    grid = (np.arange(N) + 0.5) / N
    for x in range(vocab):
        weight = float(x == 2) if certain else q[x]
        if weight == 0:
            continue
        for u in grid:
            v = drafting.verify_row(t, None if certain else d, [x], False, T, min_p, [u], 0.5)
            if v.accepted == 1:
                got[x] += weight / N
                continue
            rest = p.copy() if not certain else np.where(np.arange(vocab) == x, 0, p)
            rest = np.maximum(p - q, 0) if not certain else rest
            got += weight / N * rest / rest.sum()
            break_token = drafting.verify_row(t, None if certain else d, [x], False, T, min_p, [u], 0.0).token
            assert break_token == np.flatnonzero(rest)[0]  # (draw_u = 0: the first token of the rest)
    assert np.abs(got - p).max() < 2.0 / N


def test_accepted_tokens_and_the_last_draw_by_hand():
    # p = (1/2, 1/4, 1/4), q = (1/4, 1/2, 1/4): token 1 is accepted with probability 1/2
    t = np.log(np.array([[0.5, 0.25, 0.25]] * 3, np.float32))
    q = np.log(np.array([[0.25, 0.5, 0.25]] * 2, np.float32))
    v = drafting.verify_row(t, q, [1, 0], False, 1.0, 0.0, [0.49, 0.99], 0.74)
    assert (v.accepted, v.token) == (2, 1) and np.allclose(v.accept_prob, [0.5, 1.0], rtol=1e-6)
    v = drafting.verify_row(t, q, [1, 0], False, 1.0, 0.0, [0.51, 0.0], 0.99)
    assert (v.accepted, v.token) == (0, 0)  # max(0, p - q) = (1/4, 0, 0)
    v = drafting.verify_row(t, q, [0, 7], False, 1.0, 0.0, [0.5, 0.0], 0.6)
    assert (v.accepted, v.token) == (1, 1)  # a token outside the vocabulary is rejected; the draw is from p
    v = drafting.verify_row(t, None, [2], False, 1.0, 0.0, [0.3], 0.9)
    assert (v.accepted, v.token) == (0, 1)  # a certain draft leaves p without its token
    g = drafting.verify_row(t, None, [0, 0], True, 1.0, 0.0, [0.9, 0.9], 0.9)
    assert (g.accepted, g.token) == (2, 0)
    g = drafting.verify_row(t, None, [0, 1], True, 1.0, 0.0, [0.9, 0.9], 0.9)
    assert (g.accepted, g.token) == (1, 0)


def test_w4_by_hand_and_against_a_loop():
    w = np.array([[0x21, 0x0f]], np.uint8)  # q = 1, 2, 15, (0)
    assert drafting.w4_unpack(w, 3).tolist() == [[1, 2, 15]]
    x = np.array([[1.0, 10.0, 100.0]])
    assert drafting.w4_product(x, w, [[0.5]], None, 32)[0, 0] == 0.5 * (-7 - 60 + 700)
    assert drafting.w4_product(x, w, [[0.5]], [[1]], 32)[0, 0] == 0.5 * (0 + 10 + 1400)
    rng = np.random.default_rng(3)
    n, k, g = 3, 77, 32
    w = rng.integers(0, 256, (n, 39), dtype=np.uint8)
    s, z = rng.random((n, 3)), rng.integers(0, 16, (n, 3))
    x = rng.normal(size=(2, k))
    ref = np.zeros((2, n))
    for j in range(n):
        for i in range(k):
            q = (w[j, i // 2] >> (4 * (i % 2))) & 15
            ref[:, j] += x[:, i] * (int(q) - int(z[j, i // g])) * s[j, i // g]
    assert np.allclose(drafting.w4_product(x, w, s, z, g), ref, rtol=1e-12)


def _consistent(p):
    counts = np.bincount(p.table[p.table >= 0], minlength=len(p.refs))
    assert np.array_equal(counts, p.refs)


def test_pages_keep_their_counts_and_their_tokens():
    """Rows grow, fork, roll back and end at random; what each row holds is what was written for it."""
    rng = np.random.default_rng(4)
    rows, cols, pages = 6, 6, 30
    p = drafting.Pages(np.full((rows, cols), -1), np.zeros(rows, int), np.zeros(pages, int), np.zeros((pages, 16), int))
    held = [[] for _ in range(rows)]
    for step in range(200):
        op = rng.integers(4)
        if op == 0:
            n = np.minimum(rng.integers(0, 20, rows), cols * 16 - p.length)
            values = rng.integers(1, 1 << 30, (rows, 20))
            ok = p.reserve(n)
            p.write(values, n, ok)
            for r in range(rows):
                if ok[r]:
                    held[r] += values[r, :n[r]].tolist()
                    p.length[r] += n[r]
        elif op == 1:
            p.length = np.array([rng.integers(0, l + 1) for l in p.length])
            p.trim(p.length)
            held = [h[:l] for h, l in zip(held, p.length)]
        elif op == 2:
            a, b = rng.choice(rows, 2, replace=False)
            p.trim(np.zeros(rows, int), np.arange(rows) == b)
            p.fork([a], [b])
            held[b] = list(held[a])
        else:
            live = p.compact()
            assert (p.refs[live:] == 0).all() and (p.refs[:live] > 0).all()
        _consistent(p)
        for r in range(rows):
            got = [int(p.data[p.table[r, t // 16], t % 16]) for t in range(p.length[r])]
            assert got == held[r], (step, r)
