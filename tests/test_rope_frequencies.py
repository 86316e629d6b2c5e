"""Rotary frequencies (a host function) vs the oracle.

turns = f / (2 pi) 2^64 in doubles: f goes through a power and up to six operations, each off by 2^-53 of
itself and the power by a few units; ln(base) i of the exponent adds at most 20 of them."""
import math

import numpy as np
import pytest

from oracle import dense
from paper_2607_20791_gb300 import binding
from paper_2607_20791_gb300.build import build


@pytest.mark.parametrize("scaling", ["none", "linear", "base", "bands", "ramp"])
@pytest.mark.parametrize("rot, base, factor, trained", [(2, 1e4, 4.0, 512.0), (20, 1e4, 1.0, 4096.0), (64, 1e4, 40.0, 4096.0),
                                                        (128, 5e5, 8.0, 8192.0), (128, 1.5, 2.0, 300.0)])
def test_frequencies(scaling, rot, base, factor, trained):
    binding.load_library(build())
    turns, magnitude = binding.rgd_rope_frequencies(rot, base, scaling, factor, trained)
    f, m = dense.frequencies(rot, base, scaling, factor, trained)
    got = np.array([int(t) % 2 ** 64 for t in turns], dtype=object)
    want = np.array([x / (2 * math.pi) for x in f])
    assert magnitude == pytest.approx(m, rel=1e-15)
    assert all(abs(int(g) / 2 ** 64 - w) <= 64 * 2.0 ** -53 * w + 2.0 ** -64 for g, w in zip(got, want))


def test_bounds_and_codes():
    binding.load_library(build())
    a = binding.rgd_rope_frequencies(64, 1e4, binding.RGD_ROPE_BANDS, 8.0, 4096.0, 1.0, 32.0)[0]
    b = dense.frequencies(64, 1e4, "bands", 8.0, 4096.0, 1.0, 32.0)[0]
    assert np.allclose(a.numpy() / 2.0 ** 64 * 2 * math.pi, b, rtol=1e-12)
    assert binding.rgd_rope_frequencies(0, 1e4)[0].numel() == 0
