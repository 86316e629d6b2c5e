"""Pins of the dense operators' oracle: closed forms, hand cases and invariants."""
import math

import numpy as np
import pytest

from oracle import dense


def test_frequencies():
    f, m = dense.frequencies(8, 10000.0)
    assert np.allclose(f, [1, 0.1, 0.01, 0.001], rtol=1e-14) and m == 1
    assert np.allclose(dense.frequencies(8, 10000.0, "linear", 4.0)[0] * 4, f, rtol=1e-14)
    # the last pair is slowed down by the whole factor, the first not at all
    g = dense.frequencies(8, 10000.0, "base", 16.0)[0]
    assert g[0] == 1 and g[-1] == pytest.approx(f[-1] / 16, rel=1e-12)
    # 100 trained positions: pair 0 turns 15.9 times (kept), pair 2 and 3 less than once (slowed), pair 1 1.59 times
    g = dense.frequencies(8, 10000.0, "bands", 8.0, 100.0)[0]
    s = (100 * 0.1 / (2 * math.pi) - 1) / 3
    assert np.allclose(g, [1, 0.1 * (s + (1 - s) / 8), 0.01 / 8, 0.001 / 8], rtol=1e-14)
    g, m = dense.frequencies(64, 10000.0, "ramp", 40.0, 4096.0)
    f = dense.frequencies(64, 10000.0)[0]
    assert np.allclose(g[:10], f[:10]) and np.allclose(g[-5:] * 40, f[-5:]) and np.all(np.diff(g / f) <= 1e-12)
    assert m == pytest.approx(0.1 * math.log(40) + 1)


def test_rotation_turns_pairs_and_keeps_what_lies_behind():
    x = np.arange(10, dtype=float).reshape(1, 1, 10)
    f = np.array([math.pi / 2, math.pi])
    assert np.allclose(dense.rotate(x, [1], f, "half")[0, 0], [-2, -1, 0, -3, 4, 5, 6, 7, 8, 9])
    assert np.allclose(dense.rotate(x, [1], f, "pairs")[0, 0], [-1, 0, -2, -3, 4, 5, 6, 7, 8, 9])
    y = dense.rotate(x, [7], np.array([0.3, 0.2]), "half", magnitude=2.0)
    assert np.allclose((y[..., :4] ** 2).sum(), 4 * (x[..., :4] ** 2).sum()) and np.allclose(y[..., 4:], x[..., 4:])
    # products of a query and a key go by the difference of their positions
    q, k = np.random.default_rng(0).standard_normal((2, 1, 1, 8))
    f = np.array([1.0, 0.5, 0.1, 0.01])
    for layout in ("half", "pairs"):
        a = (dense.rotate(q, [11], f, layout) * dense.rotate(k, [4], f, layout)).sum()
        b = (dense.rotate(q, [1007], f, layout) * dense.rotate(k, [1000], f, layout)).sum()
        assert a == pytest.approx(b, abs=1e-9)


def test_norm():
    x = np.array([[[3.0, 4.0, 0.0, 0.0]]])
    y = dense.rotate(x, [0], np.zeros(1), "half", weight=[2, 1, 1, 1], eps=0.0)
    assert np.allclose(y, [[[6 / 2.5, 4 / 2.5, 0, 0]]])
    assert np.allclose(dense.rotate(0 * x, [5], np.ones(1), "half", eps=1e-6), 0)


def test_e4m3_values_and_rounding():
    v = dense.decode_e4m3(np.arange(256))
    assert v[0x00] == 0 and v[0x01] == 2.0 ** -9 and v[0x08] == 2.0 ** -6 and v[0x38] == 1 and v[0x7e] == 448
    assert np.isnan(v[[0x7f, 0xff]]).all() and v[0xfe] == -448 and v[0xb8] == -1
    fine = [c for c in range(256) if c & 0x7f != 0x7f]
    assert np.array_equal(dense.encode_e4m3(v[fine]), fine)
    # 17 lies between 16 and 18: to the even code; so do 1.0625 and 1.1875
    assert np.array_equal(dense.decode_e4m3(dense.encode_e4m3([17.0, 19.0, 1.0625, 1.1875, 460.0, -2.0 ** -10])), [16, 20, 1, 1.25, 448, -0.0])


def test_e4m3_matches_torch():
    torch = pytest.importorskip("torch")
    x = torch.randn(20000, generator=torch.Generator().manual_seed(1)) * torch.exp(4 * torch.randn(20000, generator=torch.Generator().manual_seed(2)))
    x = x.clamp(-448, 448)
    assert np.array_equal(dense.encode_e4m3(x.numpy()), x.to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_quantize_blocks():
    x = np.zeros((130, 200), np.float32)
    x[0, 0], x[0, 5], x[129, 199] = 7.0, -3.5, 14.0
    codes, scales = dense.quantize(x, 1)
    assert scales.shape == (130, 2) and scales[0, 0] == np.float32(7) / np.float32(448) and scales[0, 1] == 0
    assert np.allclose(dense.decode_e4m3(codes[0, [0, 5]]) * scales[0, 0], [7, -3.5])
    codes, scales = dense.quantize(x, 128)
    assert scales.shape == (2, 2) and np.count_nonzero(scales) == 2 and dense.decode_e4m3(codes[129, 199]) == 448


def test_product_against_blocks():
    rng = np.random.default_rng(3)
    x, w = rng.integers(0, 127, (3, 300)).astype(np.uint8), rng.integers(0, 127, (140, 300)).astype(np.uint8)
    sx, sw = rng.random((3, 3)), rng.random((2, 3))
    y, mag = dense.product(x, sx, w, sw)
    want = sum(sx[1, b] * sw[1, b] * (dense.decode_e4m3(x[1, b * 128:(b + 1) * 128]) @ dense.decode_e4m3(w[135, b * 128:(b + 1) * 128]))
               for b in range(3))
    assert y[1, 135] == pytest.approx(want, rel=1e-12) and (mag >= np.abs(y) - 1e-9).all()


def test_sampling_filters():
    row = np.log(np.array([0.1, 0.4, 0.2, 0.2, 0.1], np.float32))
    full = [dense.sample(row, 1.0, 0, 1.0, 0.0, u).token for u in (0.05, 0.3, 0.6, 0.8, 0.95)]
    assert full == [0, 1, 2, 3, 4]
    assert dense.sample(row, 1.0, 2, 1.0, 0.0, 0.99).token == 2  # the lower index of two equal ones
    assert dense.sample(row, 1.0, 0, 0.61, 0.0, 0.99) == dense.Drawn(3, 3, pytest.approx(0.25, rel=1e-6), False)
    assert dense.sample(row, 1.0, 0, 1.0, 0.3, 0.0).kept == 3
    assert dense.sample(row, 1.0, 3, 0.51, 0.0, 0.0).kept == 2  # (of what top-k leaves: 0.4 of 0.8 is not 0.51)
    assert dense.sample(row, 0.0, 3, 0.5, 0.0, 0.9) == dense.Drawn(1, 1, 1.0, False)
    assert dense.sample(np.array([-np.inf, np.nan, 1.0, -np.inf]), 1.0, 0, 1.0, 0.0, 0.999).kept == 1
    assert dense.sample(row, 1.0, 0, 0.0, 0.0, 0.9).kept == 1
    # the draws' frequencies are the probabilities
    us = (np.arange(4000) + 0.5) / 4000
    hits = np.bincount([dense.sample(row, 2.0, 0, 1.0, 0.0, u).token for u in us], minlength=5) / 4000
    p = np.sqrt([0.1, 0.4, 0.2, 0.2, 0.1])
    assert np.abs(hits - p / p.sum()).max() < 1e-3
