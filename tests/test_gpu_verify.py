"""Draft verification on the GPU vs the fp64 oracle.

How far a probability may be off (relative to itself), from the kernel's steps: an
exponent x = (l - top) log2(e) / T has four roundings of 2^-24 each, so e^x is off by
|x| ln 2 2^-22; 2^x has 2 ulp (2^-22); a weight is rounded to 2^-31 (2^-32 absolute, which
against a weight w is 2^-32 / w, and against the sum at most V 2^-32); the reciprocal of the
sum and the product with it 2^-23.  Acceptances and draws closer to their thresholds than
that may differ; such rows are counted and must be rare."""
import numpy as np
import pytest

from conftest import report
from oracle import drafting, sampling
from paper_2607_20791_gb300 import binding

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


class Case:
    def __init__(self, rows, draft, vocab, dtype="f32", seed=0, pad=0, certain=False, temps=(1.0, 0.0, 0.7, 2.5),
                 min_ps=(0.0, 0.1, 0.05), spread=2.0, probe_every=5):
        rng = np.random.default_rng([seed, rows, draft, vocab])
        torch = _torch()
        kind = torch.float32 if dtype == "f32" else torch.bfloat16
        t = rng.normal(0, spread, (rows, draft + 1, vocab)).astype(np.float32)
        q = (t[:, :draft] + 0.6 * rng.normal(size=(rows, draft, vocab))).astype(np.float32)
        self.t = torch.full((rows, draft + 1, vocab + pad), 1e4).to(kind)  # (padding is never looked at)
        self.t[..., :vocab] = torch.from_numpy(t).to(kind)
        self.q = None if certain else torch.full((rows, draft, vocab + pad), 1e4).to(kind)
        if self.q is not None:
            self.q[..., :vocab] = torch.from_numpy(q).to(kind)
        i = np.arange(rows)
        self.temp, self.min_p = np.array(temps, np.float32)[i % len(temps)], np.array(min_ps, np.float32)[i // 2 % len(min_ps)]
        self.probe = (i % probe_every == 0).astype(np.uint8)
        self.n = np.where(i % 3 == 2, rng.integers(0, draft + 1, rows), draft).astype(np.int32)
        self.tokens = rng.integers(0, vocab, (rows, draft)).astype(np.int32)
        for r in range(rows):
            for k in range(draft):  # mostly the draft's own draw (or its best, where rows are greedy)
                if rng.random() < 0.8:
                    p = np.exp((q[r, k] - q[r, k].max()).astype(np.float64) / max(float(self.temp[r]), 0.2))
                    self.tokens[r, k] = rng.choice(vocab, p=p / p.sum())
        self.au, self.du = rng.random((rows, draft)).astype(np.float32), rng.random(rows).astype(np.float32)
        self.au, self.du = np.minimum(self.au, np.float32(1 - 2.0 ** -24)), np.minimum(self.du, np.float32(1 - 2.0 ** -24))
        self.active = (i % 7 != 6).astype(np.uint8)
        self.vocab, self.rows, self.draft = vocab, rows, draft

    def run(self, stream=None, workspace=None):
        torch = _torch()
        d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
        R, K = self.rows, self.draft
        self.out = torch.full((R, K + 1), -9, dtype=torch.int32, device="cuda")
        self.acc = torch.full((R,), -9, dtype=torch.int32, device="cuda")
        self.prob = torch.full((R, max(K, 1)), -9.0, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        ws = torch.zeros(binding.rgd_verify_draft_workspace_size(R, K), dtype=torch.uint8, device="cuda") if workspace is None else workspace
        args = (self.t.cuda(), None if self.q is None else self.q.cuda(), d(self.tokens) if K else None, d(self.n), d(self.probe),
                d(self.temp), d(self.min_p), d(self.au) if K else None, d(self.du), d(self.active))
        torch.cuda.synchronize()
        binding.rgd_verify_draft(*args, self.out, self.acc, self.prob if K else None, ws, vocab=self.vocab,
                                 dev_status=self.status, stream=stream)
        torch.cuda.synchronize()
        self.ws = ws
        return self

    def check(self, status=0):
        assert int(self.status.item()) == status
        out, acc, prob = self.out.cpu().numpy(), self.acc.cpu().numpy(), self.prob.cpu().numpy()
        t = self.t[..., :self.vocab].float().numpy()
        q = None if self.q is None else self.q[..., :self.vocab].float().numpy()
        near = 0
        for r in range(self.rows):
            if not self.active[r]:
                assert (out[r] == -1).all() and acc[r] == 0 and (prob[r, :self.draft] == 0).all()
                continue
            n = int(self.n[r])
            greedy = bool(self.probe[r]) or self.temp[r] == 0
            band = np.zeros(max(n, 1))
            if not greedy:
                rel = lambda row, top, d: (abs(top - row[d]) * 1.4427 / self.temp[r] * 0.7 * 2.0 ** -22 + 2.0 ** -21
                                           + self.vocab * 2.0 ** -32
                                           + 2.0 ** -32 * np.exp(min(60.0, (top - row[d]) / self.temp[r])))
                for k in range(n):
                    d = self.tokens[r, k]
                    if 0 <= d < self.vocab:
                        for row in [t[r, k]] + ([] if q is None else [q[r, k]]):
                            top = np.nanmax(row)
                            if row[d] >= sampling.cutoff32(top, self.temp[r], self.min_p[r]):
                                band[k] += rel(row, top, d)
            # a draw's sums: of weights down to where they no longer count
            drawn = 40 * 0.7 * 2.0 ** -22 + 2.0 ** -21 + self.vocab * 2.0 ** -32
            ref = drafting.verify_row(t[r, :n + 1], None if q is None else q[r, :n], self.tokens[r, :n], greedy,
                                      float(self.temp[r]), float(self.min_p[r]), self.au[r, :n], float(self.du[r]),
                                      band=max(drawn, band.max()))
            with np.errstate(invalid="ignore"):  # (a tiny temperature: an infinite band times a probability of 0)
                within = np.abs(prob[r, :n] - ref.accept_prob) <= band[:n] * ref.accept_prob + 1e-30
            assert np.all(within | (prob[r, :n] == ref.accept_prob)), (r, prob[r, :n], ref)
            assert (prob[r, n:self.draft] == 0).all()
            near += ref.near
            if acc[r] != ref.accepted or out[r, acc[r]] != ref.token:
                assert ref.near, (r, acc[r], out[r], ref)
                continue
            assert np.array_equal(out[r, :acc[r]], self.tokens[r, :acc[r]])
            assert (out[r, acc[r] + 1:] == -1).all()
        return near


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("certain", [False, True])
@pytest.mark.parametrize("vocab, pad", [(1, 0), (2, 0), (7, 0), (8, 0), (33, 3), (255, 1), (256, 8), (1000, 0), (4096, 0), (4099, 0),
                                        (8200, 56)])
def test_against_the_oracle(gpu_lib, vocab, pad, certain, dtype):
    c = Case(22, 3, vocab, dtype, seed=vocab, pad=pad, certain=certain)
    near = c.run().check()
    report(f"draft verification, vocab {vocab} {dtype}: {near} of 22 rows near a threshold")
    assert near <= 6
    assert (c.ws == 0).all()  # ready for the next call, whatever its shape


@pytest.mark.parametrize("rows, draft, vocab, dtype", [(3, 1, 32001, "f32"), (2, 5, 50257, "bf16"), (1, 2, 128256, "bf16"),
                                                       (2, 1, 262144, "f32"), (130, 2, 3000, "bf16"), (9, 12, 2048, "f32"),
                                                       (2, 40, 600, "f32"), (7, 0, 5000, "bf16")])
def test_sizes(gpu_lib, rows, draft, vocab, dtype):
    c = Case(rows, draft, vocab, dtype, seed=rows, spread=3.0)
    report(f"draft verification {rows} x {draft} x {vocab} {dtype}: {c.run().check()} rows near a threshold")


def test_a_row_does_not_depend_on_how_the_call_is_cut(gpu_lib):
    """One row alone is cut over more blocks than the same row among 300: every bit is the same."""
    torch = _torch()
    c = Case(300, 2, 9000, "bf16", seed=5).run()
    for r in (1, 2, 3, 8):
        one = Case(1, 2, 9000, "bf16")
        one.t, one.q = c.t[r:r + 1], c.q[r:r + 1]
        for name in ("temp", "min_p", "probe", "n", "tokens", "au", "du", "active"):
            setattr(one, name, getattr(c, name)[r:r + 1])
        one.run()
        assert torch.equal(one.out[0], c.out[r]) and torch.equal(one.acc[0], c.acc[r]) and torch.equal(one.prob[0], c.prob[r])


def test_masked_logits_ties_and_extremes(gpu_lib):
    """-inf and NaN logits have no weight, ties go to the lowest index, min-p 1 keeps the maxima alone, a tiny
    temperature the maximum."""
    c = Case(24, 2, 700, "f32", seed=6, temps=(1.0, 1e-30, 0.5, 0.0), min_ps=(0.0, 1.0, 0.2), probe_every=6)
    t, q = c.t.numpy(), c.q.numpy()
    t[:, :, 100:650] = -np.inf
    q[:, :, 50:690] = -np.inf
    t[3::4, :, 20] = np.nan
    q[::3, :, 21] = np.nan
    t[::5, :, 30] = t[::5, :, 40] = t[::5, :, 660] = 50.0  # exact ties of the maximum
    c.tokens[:, 0] = np.where(np.arange(24) % 2, 30, 660)
    c.tokens[4, 0] = 20  # (a NaN logit: p = 0)
    c.n[:] = 2
    c.run().check()


def test_rest_of_equal_distributions_and_exact_acceptance(gpu_lib):
    """p = q accepts everything at u < 1; u = 0 accepts whatever p gives weight."""
    c = Case(12, 3, 500, "f32", seed=7, temps=(1.0,), min_ps=(0.0,), probe_every=100)
    c.q = c.t[:, :3].clone()
    c.n[:], c.active[:], c.probe[:] = 3, 1, 0
    c.run()
    assert (c.acc.cpu().numpy() == 3).all() and (c.prob.cpu().numpy() == 1).all()
    d = Case(12, 3, 500, "f32", seed=8, temps=(1.0,), min_ps=(0.0,), probe_every=100)
    d.au[:], d.n[:], d.active[:], d.probe[:] = 0, 3, 1, 0
    d.run()
    assert (d.acc.cpu().numpy() == 3).all()


def test_emitted_first_token_is_distributed_as_the_target(gpu_lib):
    """Chi-square over 6000 rows of the same logits: drafts drawn from q, first emitted token against p."""
    torch = _torch()
    rows, vocab, T = 6000, 24, 1.2
    c = Case(rows, 1, vocab, "f32", seed=9, temps=(T,), min_ps=(0.02,), probe_every=10 ** 9)
    c.t[:], c.q[:] = c.t[:1].clone(), c.q[:1].clone()
    p = drafting.probabilities(c.t[0, 0].numpy(), T, 0.02)
    q = drafting.probabilities(c.q[0, 0].numpy(), T, 0.02)
    rng = np.random.default_rng(10)
    c.tokens = rng.choice(vocab, (rows, 1), p=q).astype(np.int32)
    c.n[:], c.active[:] = 1, 1
    c.run()
    first = c.out.cpu().numpy()[:, 0]
    got = np.bincount(first, minlength=vocab)
    assert got[p == 0].sum() == 0
    keep = p > 0
    chi2 = ((got[keep] - rows * p[keep]) ** 2 / (rows * p[keep])).sum()
    from scipy.stats import chi2 as dist
    assert chi2 < dist.ppf(1 - 1e-6, keep.sum() - 1)


def test_rejected_rows_and_status(gpu_lib):
    """Parameters out of range reject their row alone; a bad drafted token is rejected with the draw from p."""
    c = Case(16, 2, 300, "f32", seed=11, temps=(1.0,), min_ps=(0.0,), probe_every=100)
    c.active[:], c.n[:], c.probe[:] = 1, 2, 0
    c.temp[0], c.temp[1], c.min_p[2], c.min_p[3] = -1.0, np.nan, 1.5, -0.1
    c.n[4], c.n[5], c.du[6], c.au[7, 0] = 3, -1, 1.0, 1.0
    c.t[8, 0, :] = -np.inf
    c.t[9, 0, 5] = np.inf
    c.t[10, 2, :] = np.nan
    c.au[10] = 0.0  # (so that row 10 gets there)
    c.run()
    out, acc = c.out.cpu().numpy(), c.acc.cpu().numpy()
    for r in range(11):
        assert (out[r] == -1).all() and acc[r] == 0, r
    assert int(c.status.item()) == binding.RGD_DEV_BAD_PARAM
    c.active[:11] = 0
    c.tokens[12, 0], c.tokens[13, 0] = 300, -5
    c.run().check(status=binding.RGD_DEV_BAD_TOKEN)
    assert c.acc[12].item() == 0 and c.acc[13].item() == 0


def test_position_past_the_first_rejection_does_not_matter(gpu_lib):
    c = Case(4, 3, 200, "f32", seed=12, temps=(1.0,), min_ps=(0.0,), probe_every=100)
    c.active[:], c.n[:], c.probe[:] = 1, 3, 0
    c.tokens[:, 0] = 300  # always rejected
    c.t[:, 1:] = np.nan
    c.run()
    assert (c.acc.cpu().numpy() == 0).all() and (c.out.cpu().numpy()[:, 0] >= 0).all()


def test_workspace_reuse_stream_and_graph(gpu_lib):
    torch = _torch()
    big, small = Case(40, 4, 3001, "bf16", seed=13), Case(6, 2, 900, "f32", seed=14)
    ws = torch.zeros(binding.rgd_verify_draft_workspace_size(40, 4), dtype=torch.uint8, device="cuda")
    big.run(workspace=ws).check()
    small.run(workspace=ws).check()
    side = torch.cuda.Stream()
    big.run(stream=side, workspace=ws).check()
    d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    args = (big.t.cuda(), big.q.cuda(), d(big.tokens), d(big.n), d(big.probe), d(big.temp), d(big.min_p), d(big.au), d(big.du),
            d(big.active))
    want = big.out.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for _ in range(3):
            binding.rgd_verify_draft(*args, big.out, big.acc, None, ws, dev_status=big.status, stream=side)
    big.out.fill_(-9)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(big.out, want)


@pytest.mark.parametrize("rows, draft, vocab, dtype, certain", [(3, 3, 1000, "f32", False), (150, 4, 4096, "bf16", False),
                                                                (40, 3, 32001, "f32", False), (4, 4, 128256, "bf16", True),
                                                                (20, 5, 50000, "bf16", False)])
def test_same_result_every_time(gpu_lib, rows, draft, vocab, dtype, certain):
    """Calls back to back on one workspace: no result, sum or count of one is taken for another's."""
    torch = _torch()
    case = Case(rows, draft, vocab, dtype, seed=16, certain=certain).run()
    d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    args = (case.t.cuda(), None if case.q is None else case.q.cuda(), d(case.tokens), d(case.n), d(case.probe), d(case.temp),
            d(case.min_p), d(case.au), d(case.du), d(case.active))
    out, acc, prob = (torch.empty_like(x) for x in (case.out, case.acc, case.prob))
    wrong = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(300):
        binding.rgd_verify_draft(*args, out, acc, prob, case.ws, vocab=vocab, dev_status=case.status)
        wrong += (out != case.out).sum() + (acc != case.acc).sum() + (prob != case.prob).sum()
        out.fill_(-5)
    assert int(wrong.item()) == 0 and int(case.status.item()) == 0
    assert not bool(case.ws.any())
