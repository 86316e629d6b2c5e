"""Gated decoding through several layers: the dense operators around the attention, end to end on the GPU.

A toy model of L layers with 8-bit weights decodes one token a row and step; each prompt group has a greedy probe and
some sample rows.  In every layer

  activations to 8 bits, 8-bit projection to queries, keys, values  (rgd_fp8_quantize, rgd_fp8_matmul)
  head norms, rotation, keys and values into the layer's pages      (rgd_qk_rope_cache)
  attention over [prompt of the group | the row's own suffix]       (rgd_prefix_decode_attn)
  8-bit projection back into the residual stream                    (rgd_fp8_quantize, rgd_fp8_matmul)

and at the end

  8-bit output matrix -> logits                                     (rgd_fp8_quantize, rgd_fp8_matmul)
  temperature, top-k, top-p, min-p from given uniforms              (rgd_sample_top)
  the probes' tokens through the refusal gate                       (rgd_probe_gate)

Pages are reserved once a step for all layers.  The prompts go through the same calls, a group's prompt as one row of
many tokens (its own attention is left out: prefill attention is not this library's).  Weights, embeddings and prompts
are random.  Run: python examples/layered_decode.py
"""
from __future__ import annotations

import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2607_20791_gb300 import binding  # noqa: E402

PAGE = 16


class Linear:
    """An [n, k] matrix in 8 bits, quantised once, in blocks of 128 x 128."""

    def __init__(self, weight):
        import torch
        n, k = weight.shape
        self.n, self.blocks = n, -(-k // 128)
        self.q = torch.zeros(n, (k + 15) // 16 * 16, dtype=torch.float8_e4m3fn, device="cuda")
        self.scales = torch.zeros(-(-n // 128), self.blocks, device="cuda")
        binding.rgd_fp8_quantize(weight.cuda(), self.q, self.scales, block_rows=128)

    def __call__(self, x, status, dtype=None):
        import torch
        m, k = x.shape
        q = torch.empty(m, self.q.shape[1], dtype=torch.float8_e4m3fn, device="cuda")
        s = torch.empty(m, self.blocks, device="cuda")
        y = torch.empty(m, self.n, dtype=dtype or x.dtype, device="cuda")
        binding.rgd_fp8_quantize(x, q, s, dev_status=status)
        binding.rgd_fp8_matmul(q, s, self.q, self.scales, y, k=k, dev_status=status)
        return y


class Decoder:
    def __init__(self, groups=2, rows_per_group=3, layers=2, vocab=1000, prompt=40, room=160, seed=0, scaling="bands"):
        import torch
        self.torch = torch
        g = torch.Generator().manual_seed(seed)
        self.G, self.rpg, self.L, self.V = groups, rows_per_group, layers, vocab
        self.R, self.Hq, self.Hkv, self.D = groups * rows_per_group, 4, 2, 64
        self.width, self.heads = self.Hq * self.D, self.Hq + 2 * self.Hkv
        self.embed = torch.randn(vocab, self.width, generator=g).bfloat16().cuda()
        spread = 1 / math.sqrt(self.width)
        self.qkv = [Linear(spread * torch.randn(self.heads * self.D, self.width, generator=g)) for _ in range(layers)]
        self.back = [Linear(spread * torch.randn(self.width, self.width, generator=g)) for _ in range(layers)]
        self.head = Linear(2 * spread * torch.randn(vocab, self.width, generator=g))
        self.norms = [[(1 + 0.1 * torch.randn(self.D, generator=g)).bfloat16().cuda() for _ in range(2)] for _ in range(layers)]
        turns, magnitude = binding.rgd_rope_frequencies(self.D, 10000.0, scaling, factor=8.0, trained_length=64.0)
        self.turns = turns.cuda()
        self.rope = binding.RopeShape(num_q_heads=self.Hq, num_k_heads=self.Hkv, head_dim=self.D, rotary_dim=self.D,
                                      layout=binding.RGD_ROPE_HALF, norm=1, eps=1e-6, magnitude=magnitude)

        pp, cols = -(-prompt // PAGE), -(-room // PAGE)
        pages = groups * pp + self.R * cols
        self.cache = binding.CacheShape(num_layers=layers, num_pages=pages, num_kv_heads=self.Hkv, page_size=PAGE, head_dim=self.D)
        self.k, self.v = (torch.zeros(layers, pages, self.Hkv, PAGE, self.D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        i32 = dict(dtype=torch.int32, device="cuda")
        self.prompt_table = torch.arange(groups * pp, **i32).view(groups, pp)
        self.prompt_len = torch.full((groups,), prompt, **i32)
        self.refs = torch.zeros(pages, **i32)
        self.refs[:groups * pp] = 1
        self.table, self.length = torch.full((self.R, cols), -1, **i32), torch.zeros(self.R, **i32)
        self.first = self.prompt_len.repeat_interleave(rows_per_group).contiguous()
        self.one = torch.ones(self.R, **i32)
        self.ws = torch.empty(binding.rgd_cache_workspace_size(self.cache, self.R), dtype=torch.uint8, device="cuda")
        self.ok = torch.zeros(self.R, dtype=torch.uint8, device="cuda")
        self.attn = binding.AttnShape(num_groups=groups, rows_per_group=rows_per_group, num_q_heads=self.Hq, num_kv_heads=self.Hkv,
                                      head_dim=self.D, page_size=PAGE, num_pages=pages, max_prompt_pages=pp, max_suffix_pages=cols,
                                      num_ctas=0, reserved=0)
        self.attn_ws = torch.zeros(binding.rgd_prefix_decode_attn_workspace_size(self.attn), dtype=torch.uint8, device="cuda")

        row = torch.arange(self.R)
        self.probe = (row % rows_per_group == 0).to(torch.uint8).cuda()
        self.temp = torch.where(row % rows_per_group == 0, 0.0, 1.2).cuda()
        self.top_k = torch.full((self.R,), 40, **i32)
        self.top_p, self.min_p = torch.full((self.R,), 0.95, device="cuda"), torch.full((self.R,), 0.01, device="cuda")
        self.active = torch.ones(self.R, dtype=torch.uint8, device="cuda")
        self.status = torch.zeros(1, **i32)
        self.trie = binding.Trie([[1, 2], [3]], 1)
        self.gate = binding.new_gate_state(groups)
        binding.rgd_gate_state_init(self.gate, groups)
        self.token = torch.zeros(self.R, **i32)
        self.logits = None
        self._fill(torch.randint(0, vocab, (groups, prompt), generator=g).cuda())

    def _pages(self, layer, x, rows, table, length, first, new, ok):
        """x [rows * tokens, width] projected; keys and values into the layer's pages; the rotated queries."""
        t = self.torch
        qkv = self.qkv[layer](x, self.status).view(rows, -1, self.heads, self.D)
        q, k, v = qkv[:, :, :self.Hq], qkv[:, :, self.Hq:self.Hq + self.Hkv], qkv[:, :, self.Hq + self.Hkv:]
        out = t.zeros(rows, qkv.shape[1], self.Hq, self.D, dtype=t.bfloat16, device="cuda")
        binding.rgd_qk_rope_cache(self.rope, self.cache, layer, q, k, v, first, self.turns, *self.norms[layer], new, table, length, ok,
                                  out, self.k, self.v, dev_status=self.status)
        return out

    def _fill(self, prompts):
        """The prompts' keys and values in every layer, and each row's first token."""
        t = self.torch
        x = self.embed[prompts].view(-1, self.width)
        zero = t.zeros(self.G, dtype=t.int32, device="cuda")
        for layer in range(self.L):
            q = self._pages(layer, x, self.G, self.prompt_table, zero, None, self.prompt_len, None)
            x = x + self.back[layer](q.view(-1, self.width), self.status)
        self.token.copy_(prompts[:, -1].repeat_interleave(self.rpg))

    def step(self, u):
        """One token a row from the uniforms u [R]; all on the current stream, without a look at the host."""
        t = self.torch
        x = self.embed[self.token.long().clamp(min=0)]
        binding.rgd_cache_reserve(self.cache, self.table, self.length, self.one, self.active, self.refs, self.k, self.v, self.ok,
                                  self.ws, dev_status=self.status)
        ends = self.length + 1
        for layer in range(self.L):
            q = self._pages(layer, x, self.R, self.table, self.length, self.first, self.one, self.ok)
            out = t.empty(self.R, self.Hq, self.D, dtype=t.bfloat16, device="cuda")
            binding.rgd_prefix_decode_attn(self.attn, q, self.k[layer], self.v[layer], self.prompt_table, self.prompt_len, self.table, ends,
                                           self.active, 1 / math.sqrt(self.D), out, None, self.attn_ws, self.status)
            x = x + self.back[layer](out.view(self.R, self.width), self.status)
        self.logits = self.head(x, self.status, t.float32)
        self.length += self.active.int()
        binding.rgd_sample_top(self.logits, self.probe, self.temp, self.top_k, self.top_p, self.min_p, u, self.active, self.token,
                               dev_status=self.status)
        # (an ended probe's row draws no token, which the gate does not look at)
        binding.rgd_probe_gate(self.trie, self.G, self.rpg, self.token, 1, self.rpg, -1, 1 << 20, self.gate, self.active, self.status)
        return self.token

    def check(self):
        self.torch.cuda.synchronize()
        if int(self.status.item()):
            raise RuntimeError(f"device status {int(self.status.item())}")


def run(steps=10, seed=0, **sizes):
    """The decoder after its steps, and the tokens of every one of them [steps, R]."""
    import torch
    d = Decoder(seed=seed, **sizes)
    u = torch.rand(steps, d.R, generator=torch.Generator().manual_seed(seed + 1)).cuda()
    got = [d.step(u[i]).clone() for i in range(steps)]
    d.check()
    return d, torch.stack(got)


def main():
    d, got = run()
    for r in range(d.R):
        print(f"row {r} ({'probe' if r % d.rpg == 0 else 'sample'}): {got[:, r].tolist()}")
    print("gate decisions", binding.decode_gate_state(d.gate)["decision"].tolist())


if __name__ == "__main__":
    main()
