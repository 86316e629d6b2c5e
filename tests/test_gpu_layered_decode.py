"""The dense operators together (examples/layered_decode.py): a step's logits against a plain form of the whole
model in fp32 on the same 8-bit values, and the same tokens eagerly and from one CUDA graph."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "layered_decode.py")
    spec = importlib.util.spec_from_file_location("layered_decode", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_runs_and_repeats(gpu_lib):
    import torch
    ex = _example()
    d, a = ex.run(steps=12, seed=1)
    _, b = ex.run(steps=12, seed=1)
    assert torch.equal(a, b)
    assert bool((a >= -1).all()) and bool((a < d.V).all()) and bool((a[0] >= 0).all())
    assert int((d.refs > 0).sum()) == int((d.table >= 0).sum()) + d.prompt_table.numel()


def test_graph_gives_the_eager_tokens(gpu_lib):
    import torch
    ex = _example()
    steps = 8
    d, want = ex.run(steps=steps, seed=3)
    e = ex.Decoder(seed=3)
    u = torch.rand(steps, e.R, generator=torch.Generator().manual_seed(4)).cuda()
    e.step(u[0])
    got, side, slot = [e.token.clone()], torch.cuda.Stream(), u[0].clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        e.step(slot)
    for i in range(1, steps):
        slot.copy_(u[i])
        graph.replay()
        got.append(e.token.clone())
    e.check()
    assert torch.equal(torch.stack(got), want)


def test_a_step_is_the_models(gpu_lib):
    """Every operator's result is rounded as the kernels round it (bf16 between them, 8 bits into products), so that
    what differs is fp32 arithmetic: a value next to a rounding's edge goes the other way now and then, which moves a logit by at
    most some 2^-4 of one term of its sum of 256; logits are about 2, 1 in 16 of them a term's size."""
    import torch
    ex = _example()
    d = ex.Decoder(seed=5, layers=2)
    u = torch.rand(6, d.R, generator=torch.Generator().manual_seed(6)).cuda()
    for i in range(5):
        d.step(u[i])
    token, length = d.token.clone(), d.length.clone()
    active = d.active.clone()
    d.step(u[5])
    d.check()

    def linear(lin, x, dtype):
        m, k = x.shape
        blocks = x.float().view(m, -1, 128)
        most = blocks.abs().amax(-1, keepdim=True)
        q = (blocks * torch.where(most > 0, torch.full_like(most, 448.0) / most, 0.0)).to(torch.float8_e4m3fn).float() * (most / torch.full_like(most, 448.0))
        w = lin.q[:, :k].float() * lin.scales.repeat_interleave(128, 1)[:, :k].repeat_interleave(128, 0)[:lin.n]
        return (q.view(m, k).double() @ w.double().T).to(dtype)

    x = d.embed[token.long().clamp(min=0)]
    freq = d.turns.double() / 2.0 ** 64 * 2 * math.pi
    for layer in range(d.L):
        qkv = linear(d.qkv[layer], x, torch.bfloat16).view(d.R, d.heads, d.D)
        q = qkv[:, :d.Hq].double()
        q = q / (q.square().mean(-1, keepdim=True) + 1e-6).sqrt() * d.norms[layer][0].double()
        angle = (d.first + length).double()[:, None, None] * freq
        a, b = q[..., :32], q[..., 32:]
        q = torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1).bfloat16().double()
        out = torch.zeros(d.R, d.Hq, d.D, dtype=torch.bfloat16, device="cuda")
        for r in range(d.R):
            def tokens(pool):  # [tokens, Hkv, D], the prompt's and the row's own with the new one
                own = pool[layer][d.table[r].clamp(min=0).long()].transpose(1, 2).reshape(-1, d.Hkv, d.D)[:int(length[r]) + 1]
                shared = pool[layer][d.prompt_table[r // d.rpg].long()].transpose(1, 2).reshape(-1, d.Hkv, d.D)
                return torch.cat([shared[:int(d.prompt_len[0])], own]).double()
            k, v = tokens(d.k).repeat_interleave(2, 1), tokens(d.v).repeat_interleave(2, 1)
            p = torch.softmax(torch.einsum("hd,thd->ht", q[r], k) / math.sqrt(d.D), -1)
            if active[r]:
                out[r] = torch.einsum("ht,thd->hd", p, v).bfloat16()
        x = x + linear(d.back[layer], out.view(d.R, d.width), torch.bfloat16)
    want = linear(d.head, x, torch.float32)
    on = active != 0
    off = (d.logits - want)[on].abs()
    assert float(off.max()) < 0.125 * float(want.abs().max()) and float(off.square().mean().sqrt()) < 0.02 * float(want[on].square().mean().sqrt())
