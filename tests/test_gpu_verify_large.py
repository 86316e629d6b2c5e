"""Draft verification over large vocabularies, sampled rows alone: every acceptance, probability and draw against
the definitions in fp64.  A draw is not compared as a token but as a place: the token's stretch of the cumulative
mass has to hold the mark u * total, up to what rounding may move either.

How far the kernel's numbers may be off, from its steps.  A weight: the exponent x = (l - top) log2(e) / T has four
roundings of 2^-24, so |x| ln 2 2^-22 relative, and 2^x 2 ulp (2^-22); a whole multiple of 2^-31 is 2^-32 absolute
(weights are at most 1 and their sum at least 1); the reciprocal of the sum and the product with it 2^-23.  Weights
of |x| > 40 are below 2^-40 and count for nothing, so over a row's mass, of sum 1,
    E = 40 ln 2 2^-22 + 2^-21 + 2 V 2^-32
bounds the error of any partial sum of p (its own roundings and the normaliser's).  max(0, p - q) has both sides'
errors and a rounding of 2^-32 for each token: 2 E + V 2^-32.  The mark is u times such a sum: twice that in all."""
import math

import numpy as np
import pytest

from conftest import report
from oracle import sampling
from paper_2607_20791_gb300 import binding

pytestmark = pytest.mark.gpu


def _probabilities(row, temp, min_p):
    import torch
    top = row.max()
    cut = float(sampling.cutoff32(np.float32(top.item()), temp, min_p))
    z = (row.double() - top.double()) / float(np.float32(temp))
    w = torch.where(row >= cut, z.exp(), 0.0)
    return w / w.sum()


def _off(row, d, temp, vocab):
    """Relative error of p(d)."""
    x = (float(row.max()) - float(row[d])) / temp
    return x * 2.0 ** -22 + 2.0 ** -21 + vocab * 2.0 ** -32 + 2.0 ** -32 * math.exp(min(60.0, x))


@pytest.mark.parametrize("pad, certain", [(0, False), (3, False), (0, True)])
@pytest.mark.parametrize("rows, draft, vocab, dtype", [
    (4, 3, 128256, "f32"), (4, 3, 128256, "bf16"), (3, 2, 262144, "f32"), (3, 2, 262144, "bf16"),  # (few positions: 16 blocks to each)
    (12, 3, 128256, "bf16"), (16, 2, 262144, "f32"),                                              # (8)
    (80, 4, 128256, "bf16"), (40, 3, 50257, "f32"), (100, 4, 32001, "bf16"),                      # (4, 2)
])
def test_places_of_the_draws(gpu_lib, rows, draft, vocab, dtype, pad, certain):
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows * 1000003 + vocab + pad)
    kind = torch.float32 if dtype == "f32" else torch.bfloat16
    t = torch.full((rows, draft + 1, vocab + pad), 1e4, device="cuda").to(kind)
    q = torch.full((rows, draft, vocab + pad), 1e4, device="cuda").to(kind)
    tokens = torch.empty(rows, draft, dtype=torch.int32, device="cuda")
    temp = np.array([1.0, 0.7, 2.5], np.float32)[np.arange(rows) % 3]
    min_p = np.array([0.0, 0.05], np.float32)[np.arange(rows) // 3 % 2]
    for r in range(rows):
        x = 2.0 * torch.randn(draft + 1, vocab, generator=g, device="cuda")
        t[r, :, :vocab] = x
        q[r, :, :vocab] = x[:draft] + 0.6 * torch.randn(draft, vocab, generator=g, device="cuda")
        for k in range(draft):
            of = _probabilities((t if certain else q)[r, k, :vocab].float(), temp[r], min_p[r])
            tokens[r, k] = of.argmax() if certain and k == 0 else torch.multinomial(of, 1, generator=g)
    au, du = torch.rand(rows, draft, generator=g, device="cuda"), torch.rand(rows, generator=g, device="cuda")
    if certain:
        au[:, 0] *= 1e-6  # (a certain draft's p is small here: the first is taken, the next is not)
    out = torch.empty(rows, draft + 1, dtype=torch.int32, device="cuda")
    acc, prob = torch.empty(rows, dtype=torch.int32, device="cuda"), torch.empty(rows, draft, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.zeros(binding.rgd_verify_draft_workspace_size(rows, draft), dtype=torch.uint8, device="cuda")
    dev = lambda a: torch.from_numpy(a).cuda()
    binding.rgd_verify_draft(t, None if certain else q, tokens, None, None, dev(temp), dev(min_p), au, du, None, out, acc, prob, ws,
                             vocab=vocab, dev_status=status)
    assert int(status.item()) == 0 and not bool(ws.any())
    out, acc, prob, tokens, au, du = (a.cpu().numpy() for a in (out, acc, prob, tokens, au, du))
    whole = 40 * math.log(2) * 2.0 ** -22 + 2.0 ** -21 + 2 * vocab * 2.0 ** -32
    widest = 0.0
    for r in range(rows):
        n, last = int(acc[r]), None
        assert 0 <= n <= draft
        assert (out[r, :n] == tokens[r, :n]).all() and 0 <= out[r, n] < vocab and (out[r, n + 1:] == -1).all()
        for k in range(draft):
            d = int(tokens[r, k])
            row = t[r, k, :vocab].float()
            p = _probabilities(row, temp[r], min_p[r])
            pd, off = float(p[d]), _off(row, d, temp[r], vocab)
            if certain:
                qd = 1.0
            else:
                side = q[r, k, :vocab].float()
                of = _probabilities(side, temp[r], min_p[r])
                qd, off = float(of[d]), off + _off(side, d, temp[r], vocab)
            want = min(1.0, pd / qd)
            assert abs(float(prob[r, k]) - want) <= off * want, (r, k, prob[r, k], want)
            u = float(au[r, k])
            if k < n:
                assert u * qd <= pd * (1 + 2 * off), (r, k)
            elif k == n:
                assert u * qd >= pd * (1 - 2 * off), (r, k)
                if certain:
                    last = p.clone()
                    last[d] = 0.0
                else:
                    last = (p - of).clamp(min=0.0)
        if last is None:
            last, slack = _probabilities(t[r, draft, :vocab].float(), temp[r], min_p[r]), 2 * whole
        else:
            slack = 2 * (2 * whole + vocab * 2.0 ** -32)
        c, token = last.cumsum(0), int(out[r, n])
        mark, upto = float(np.float32(du[r])) * float(c[-1]), float(c[token])
        assert upto - float(last[token]) - slack <= mark <= upto + slack, (r, token, mark, upto, float(last[token]))
        widest = max(widest, (upto - float(last[token]) - mark) / slack, (mark - upto) / slack)
    some, none = int((acc > 0).sum()), int((acc < draft).sum())
    report(f"draft verification {rows} x {draft} x {vocab} {dtype}: {some} rows with accepted drafts, {none} with a rejected one; "
           f"draws off by {max(widest, 0):.2g} of the bound")
    assert some >= 1 and none >= 1
