"""Sampling on the GPU vs what the oracle admits: every row is checked, also those whose cut or draw lies next to a
threshold.  Long and flat rows, whose cut is searched for, in every number of blocks a row.

The room that rounding leaves is derived at ``oracle.dense.Admitted``; it depends on the inputs alone."""
import numpy as np
import pytest

from conftest import report
from oracle import dense
from test_gpu_sample_top import _call, _logits

pytestmark = pytest.mark.gpu


def _searched(rows, rng):
    """Filters of rows whose cut is mostly searched for."""
    t = rng.choice([0.7, 1.0, 2.0, 5.0], rows)
    k = rng.choice([0, 0, 0, 50, 3000, 20000], rows)
    p = rng.choice([0.999, 0.95, 0.8, 0.5, 0.3], rows)
    m = rng.choice([0.0, 0.0, 0.01], rows)
    return t.astype(np.float32), k, p.astype(np.float32), m.astype(np.float32), rng.random(rows).astype(np.float32)


def _check(name, x, t, k, p, m, u, vocab):
    logits = x[:, :vocab].float().numpy()
    token, kept, prob, status = _call(x.cuda(), t, k, p, m, u, vocab=vocab)
    assert status == 0
    open_rows = widest = 0
    for r in range(len(logits)):
        a = dense.admitted(logits[r], t[r], int(k[r]), p[r], m[r])
        open_rows += a.most > a.fewest
        widest = max(widest, a.most - a.fewest)
        fault = a.fault(int(kept[r]), int(token[r]), float(prob[r]), float(u[r]))
        assert not fault, (r, t[r], k[r], p[r], m[r], u[r], fault)
    report(f"sampling {name}: every one of {len(logits)} rows checked, {open_rows} with a cut that rounding decides (of {widest + 1} at most)")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["zipf", "flat", "steps", "normal", "junk"])
@pytest.mark.parametrize("rows, vocab, pad", [(40, 3001, 0), (24, 32001, 2), (24, 128256, 0)])
def test_distributions(gpu_lib, rows, vocab, pad, kind, dtype):
    rng = np.random.default_rng(vocab + len(kind))
    _check(f"{rows} x {vocab} {dtype} {kind}", _logits(rows, vocab, kind, dtype, 20, pad), *_searched(rows, rng), vocab)


@pytest.mark.parametrize("kind", ["zipf", "flat"])
@pytest.mark.parametrize("rows, vocab, dtype", [(700, 1000, "f32"), (330, 5931, "bf16"), (170, 20000, "f32"), (310, 70001, "bf16"),
                                                (12, 500000, "f32"), (12, 1 << 20, "bf16"), (12, 1 << 20, "f32")])
def test_batches(gpu_lib, rows, vocab, dtype, kind):
    rng = np.random.default_rng(rows + 1)
    _check(f"{rows} x {vocab} {dtype} {kind}", _logits(rows, vocab, kind, dtype, 2), *_searched(rows, rng), vocab)
