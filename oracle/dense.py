"""Rotation, 8-bit products and filtered sampling, oracle side (test infrastructure only).

* :func:`frequencies` -- radians per position of each rotated pair, with the scalings for
  positions past the trained length; :func:`rotate` -- head norms and rotation, each pair as
  a complex number.
* :func:`decode_e4m3`, :func:`quantize`, :func:`product` -- the 8-bit type by its definition
  (sign, 4 bits of exponent with bias 7, 3 of mantissa, no infinities), block scales in
  fp32 as stated, products in fp64.
* :func:`sample` -- temperature, min-p, top-k, top-p and a draw from a given uniform, token by
  token over a sorted list; :func:`admitted` -- which results the roundings of fp32 weights leave
  open for a row, also where a cut or the draw lies next to its threshold.

Pinned by ``tests/test_oracle_dense.py`` and ``tests/test_oracle_thresholds.py`` against closed forms and hand
cases.
"""
from __future__ import annotations

import dataclasses
import math

import numpy as np

from . import sampling


def frequencies(rot: int, base: float, scaling: str = "none", factor: float = 1.0, trained: float = 0.0,
                low: float = 1.0, high: float | None = None):
    """Radians per position of pair i, and the factor on the rotated part."""
    out, magnitude = [], 1.0
    if scaling == "base" and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    for i in range(rot // 2):
        f = base ** (-2 * i / rot)
        if scaling == "linear":
            f /= factor
        elif scaling == "bands":
            top = 4.0 if high is None else high
            wave = 2 * math.pi / f
            if wave > trained / low:
                f /= factor
            elif wave >= trained / top:
                s = (trained / wave - low) / (top - low)
                f = (1 - s) * f / factor + s * f
        elif scaling == "ramp":
            top = 32.0 if high is None else high
            a, b = (rot * math.log(trained / (n * 2 * math.pi)) / (2 * math.log(base)) for n in (top, low))
            a, b = max(math.floor(a), 0), min(math.ceil(b), rot - 1)
            slow = min(max((i - a) / max(b - a, 0.001), 0.0), 1.0)
            f = slow * f / factor + (1 - slow) * f
            magnitude = 0.1 * math.log(factor) + 1
        out.append(f)
    return np.array(out), magnitude


def rotate(x, positions, freq, layout: str, magnitude: float = 1.0, weight=None, eps=None):
    """``x`` [tokens, heads, D]; ``weight`` [D] or None, ``eps`` None: no norm.  Returns fp64."""
    x = np.asarray(x, np.float64)
    if eps is not None:
        x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps)
        if weight is not None:
            x = x * np.asarray(weight, np.float64)
    half = len(freq)
    turn = magnitude * np.exp(1j * np.outer(np.asarray(positions, np.float64), freq))[:, None, :]
    out = x.copy()
    first, second = (slice(0, half), slice(half, 2 * half)) if layout == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    z = (x[..., first] + 1j * x[..., second]) * turn
    out[..., first], out[..., second] = z.real, z.imag
    return out


def decode_e4m3(codes) -> np.ndarray:
    """The values of 8-bit codes, in fp64; 0x7f and 0xff are NaN."""
    c = np.asarray(codes).astype(np.int64)
    sign, e, m = np.where(c & 0x80, -1.0, 1.0), (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    return np.where((c & 0x7f) == 0x7f, np.nan, sign * v)


_VALUES = decode_e4m3(np.arange(0x7f))


def encode_e4m3(v) -> np.ndarray:
    """The nearest code of each value of magnitude up to 448 or more (held to 448), ties to the even code."""
    v = np.asarray(v, np.float64)
    a = np.minimum(np.abs(v), 448.0)
    hi = np.clip(np.searchsorted(_VALUES, a), 1, len(_VALUES) - 1)
    lo = hi - 1
    up, down = _VALUES[hi] - a, a - _VALUES[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return (code | np.where(np.signbit(v), 0x80, 0)).astype(np.uint8)


def quantize(x, block_rows: int):
    """Codes and fp32 scales of blocks of block_rows x 128, each step rounded in fp32 as stated."""
    x = np.asarray(x, np.float32)
    rows, cols = x.shape
    codes = np.zeros(x.shape, np.uint8)
    scales = np.zeros((-(-rows // block_rows), -(-cols // 128)), np.float32)
    for a in range(scales.shape[0]):
        for b in range(scales.shape[1]):
            at = (slice(a * block_rows, (a + 1) * block_rows), slice(b * 128, (b + 1) * 128))
            most = np.abs(x[at]).max()
            if most == 0:
                codes[at] = encode_e4m3(np.where(np.signbit(x[at]), -0.0, 0.0))
                continue
            m = max(most, np.float32(2.0 ** -100))
            scales[a, b] = m / np.float32(448)
            codes[at] = encode_e4m3(x[at] * (np.float32(448) / m))
    return codes, scales


def product(x_codes, x_scales, w_codes, w_scales):
    """y and, for error bounds, the sum of the magnitudes of its terms."""
    k, n = x_codes.shape[1], w_codes.shape[0]
    by = np.arange(k) // 128
    x = decode_e4m3(x_codes) * np.asarray(x_scales, np.float64)[:, by]
    w = decode_e4m3(w_codes) * np.asarray(w_scales, np.float64)[np.arange(n)[:, None] // 128, by]
    return x @ w.T, np.abs(x) @ np.abs(w).T


@dataclasses.dataclass
class Drawn:
    token: int
    kept: int
    prob: float
    near: bool  # a cut or the draw was closer than `band` of the whole to its threshold


def sample(row, temperature: float, top_k: int, top_p: float, min_p: float, u: float, band: float = 0.0) -> Drawn:
    row = np.asarray(row, np.float32)
    fine = np.where(np.isnan(row), -np.inf, row)
    if temperature == 0:
        return Drawn(int(np.argmax(fine)), 1, 1.0, False)
    top = fine.max()
    low = sampling.cutoff32(top, temperature, min_p)
    order = sorted((i for i in range(len(row)) if fine[i] >= low and fine[i] > -np.inf), key=lambda i: (-fine[i], i))
    if top_k > 0:
        order = order[:top_k]
    w = np.exp((fine[order].astype(np.float64) - float(top)) / float(np.float32(temperature)))
    upto, near = np.cumsum(w), False
    if top_p < 1:
        want = float(np.float32(top_p)) * upto[-1]
        n = int(np.searchsorted(upto, want)) + 1
        near = bool(np.abs(upto - want).min() <= band * upto[-1])
        order, w = order[:min(n, len(order))], w[:min(n, len(order))]
    back = np.argsort(order)
    index, w = np.asarray(order)[back], w[back]
    upto = np.cumsum(w)
    mark = float(np.float32(u)) * upto[-1]
    i = min(int(np.searchsorted(upto, mark, side="right")), len(w) - 1)
    edges = upto[w > 0]
    near = near or bool(np.abs(edges - mark).min() <= band * upto[-1] or mark <= band * upto[-1])
    return Drawn(int(index[i]), len(order), float(w[i] / upto[-1]), near)


class Admitted:
    """What a row's kept count, token and probability may be, for weights that are rounded.

    Exact weights w_i = 2^x_i, x_i = (l_i - top) log2(e) / T <= 0, the largest 1.  Rounded ones differ by at most
      e_i = w_i (4 * 2^-24 ln 2 |x_i| + 2^-22) + 2^-32:
    x's difference, quotient and product and its constant are rounded (four times 2^-24 of x), the power is good
    to 2^-22, and the weight becomes a whole multiple of 2^-31.  A threshold is a share of one such sum, rounded to
    a whole multiple, and is compared with another: both are off by the sum of S's e_i at most, and by 2^-31.
    """

    def __init__(self, row, temperature: float, top_k: int, top_p: float, min_p: float):
        row = np.asarray(row, np.float32)
        fine = np.where(np.isnan(row), np.float32(-np.inf), row)
        top = fine.max()
        low = sampling.cutoff32(top, temperature, min_p)
        at = np.nonzero((fine >= low) & (fine > -np.inf))[0]
        order = at[np.argsort(-fine[at], kind="stable")]  # (equal logits, 0 and -0 too, by index)
        if top_k > 0:
            order = order[:top_k]
        self.order = order
        x = (fine[order].astype(np.float64) - float(top)) / (float(np.float32(temperature)) * math.log(2))
        self.w = np.exp2(x)
        self.e = self.w * (4 * 2.0 ** -24 * math.log(2) * -x + 2.0 ** -22) + 2.0 ** -32
        upto, slack = np.cumsum(self.w), 2 * self.e.sum() + 2.0 ** -30
        self.fewest = self.most = len(order)
        if top_p < 1:
            want = float(np.float32(top_p)) * upto[-1]
            # n tokens are kept if they reach the threshold and n - 1 do not
            self.fewest = min(int(np.searchsorted(upto, want - slack)) + 1, len(order))
            self.most = min(int(np.searchsorted(upto, want + slack)) + 1, len(order))

    def fault(self, kept: int, token: int, prob: float, u: float) -> str:
        """Why a result cannot be; empty if it can."""
        if not self.fewest <= kept <= self.most:
            return f"kept {kept}, not {self.fewest} to {self.most}"
        back = np.argsort(self.order[:kept])
        index, w, e = self.order[:kept][back], self.w[:kept][back], self.e[:kept][back]
        i = int(np.searchsorted(index, token))
        if i == kept or index[i] != token:
            return f"token {token} is not kept"
        if w[i] + e[i] < 2.0 ** -31:
            return f"token {token} has no weight"
        upto, slack = np.cumsum(w), 2 * e.sum() + 2.0 ** -30
        mark = float(np.float32(u)) * upto[-1]
        if not upto[i] - w[i] - slack <= mark <= upto[i] + slack:
            return f"token {token} from {upto[i] - w[i]} to {upto[i]}, not at {mark}"
        want = w[i] / upto[-1]
        # (the weight and the sum as above, and three roundings of 2^-24: both to fp32, and the quotient)
        off = e[i] / upto[-1] + want * (e.sum() / upto[-1] + 3 * 2.0 ** -24)
        return "" if abs(prob - want) <= 1.01 * off else f"probability {prob}, not {want}"


def admitted(row, temperature: float, top_k: int, top_p: float, min_p: float) -> Admitted:
    """Of a row that is not greedy."""
    return Admitted(row, temperature, top_k, top_p, min_p)
