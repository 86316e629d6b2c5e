"""Gated decoding with drafted tokens: a toy one-layer model, end to end on the GPU.

Every step, each row of a prompt group (one greedy probe, some sample rows) has a draft
propose K tokens (the model without its attention layer: embedding and output matrix alone);
the target model then looks at all K + 1 positions at once:

  embeddings -> 4-bit projections to queries, keys and values  (rgd_w4_matvec)
  room for K + 1 tokens and their keys and values in the cache (rgd_cache_reserve, _write)
  attention over [prompt of the group | the row's own suffix]  (rgd_prefix_decode_attn)
  4-bit output matrix -> the target's logits                   (rgd_w4_matvec)
  drafts accepted or rejected, one more token drawn            (rgd_verify_draft)
  the rejected tokens' pages given back                        (rgd_cache_trim)
  the probes' tokens through the refusal gate                  (rgd_probe_gate)

The attention takes a (row, position) as a row of its own: its block table is the row's, and
its suffix ends with the position's token, which makes the K + 1 positions causal.

Weights, embeddings and prompts are random; greedy rows produce what they would without
drafts, but for ties within rounding: the products' last bits go by how many rows they have.
Run: python examples/drafted_decode.py
"""
from __future__ import annotations

import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2607_20791_gb300 import binding  # noqa: E402

PAGE = 16


class Decoder:
    def __init__(self, groups=2, rows_per_group=3, draft=3, vocab=512, prompt=40, room=160, seed=0, trie=None):
        import torch
        self.torch = torch
        g = torch.Generator().manual_seed(seed)
        self.G, self.rpg, self.K, self.V = groups, rows_per_group, draft, vocab
        self.R, self.Hq, self.Hkv, self.D = groups * rows_per_group, 4, 2, 64
        width = self.Hq * self.D

        def weights(n, k, scale):  # 4-bit, groups of 64
            return (torch.randint(0, 256, (n, k // 2), generator=g, dtype=torch.uint8).cuda(),
                    (torch.rand(n, k // 64, generator=g) * scale + 0.5 * scale).bfloat16().cuda())
        self.embed = torch.randn(vocab, width, generator=g).bfloat16().cuda()
        self.w_qkv = weights((self.Hq + 2 * self.Hkv) * self.D, width, 0.02)
        self.w_head = weights(vocab, width, 0.1)

        # prompts and room for every row to grow; the prompts' pages count as their groups' own
        pp, cols = -(-prompt // PAGE), -(-room // PAGE)
        self.pages = groups * pp + self.R * cols
        self.cache = binding.CacheShape(num_layers=1, num_pages=self.pages, num_kv_heads=self.Hkv, page_size=PAGE,
                                        head_dim=self.D)
        pool = (1, self.pages, self.Hkv, PAGE, self.D)
        self.k, self.v = (torch.randn(pool, generator=g).bfloat16().cuda() for _ in range(2))
        i32 = dict(dtype=torch.int32, device="cuda")
        self.prompt_table = torch.arange(groups * pp, **i32).view(groups, pp)
        self.prompt_len = torch.full((groups,), prompt, **i32)
        self.refs = torch.zeros(self.pages, **i32)
        self.refs[:groups * pp] = 1
        self.table = torch.full((self.R, cols), -1, **i32)
        self.length = torch.zeros(self.R, **i32)
        self.ws = torch.empty(binding.rgd_cache_workspace_size(self.cache, self.R), dtype=torch.uint8, device="cuda")
        self.ok = torch.zeros(self.R, dtype=torch.uint8, device="cuda")
        self.live = torch.zeros(1, **i32)

        # one attention row for every row and position
        P = draft + 1
        self.attn = binding.AttnShape(num_groups=groups, rows_per_group=rows_per_group * P, num_q_heads=self.Hq,
                                      num_kv_heads=self.Hkv, head_dim=self.D, page_size=PAGE, num_pages=self.pages,
                                      max_prompt_pages=pp, max_suffix_pages=cols, num_ctas=0, reserved=0)
        self.attn_ws = torch.zeros(binding.rgd_prefix_decode_attn_workspace_size(self.attn), dtype=torch.uint8, device="cuda")

        row = torch.arange(self.R)
        self.probe = (row % rows_per_group == 0).to(torch.uint8).cuda()
        self.temp = torch.where(row % rows_per_group == 0, 0.0, 1.3).cuda()
        self.min_p = torch.full((self.R,), 0.05, device="cuda")
        self.seed = torch.arange(self.R, dtype=torch.int64, device="cuda") + 1000 * seed
        self.active = torch.ones(self.R, dtype=torch.uint8, device="cuda")
        self.verify_ws = torch.zeros(binding.rgd_verify_draft_workspace_size(self.R, draft), dtype=torch.uint8, device="cuda")
        self.last = torch.randint(0, vocab, (groups, 1), generator=g).expand(groups, rows_per_group).reshape(-1).int().cuda()
        self.status = torch.zeros(1, **i32)
        self.gate_status = torch.zeros(1, **i32)  # (its RGD_DEV_BAD_TOKEN: the -1 behind a row's tokens, skipped)
        self.trie = binding.Trie(trie or [[1, 2]], 2)
        self.gate = binding.new_gate_state(groups)
        binding.rgd_gate_state_init(self.gate, groups)
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.steps = 0

    def propose(self):
        """K tokens a row from the draft, and the logits they were drawn from."""
        t = self.torch
        tokens = t.zeros(self.R, self.K, dtype=t.int32, device="cuda")
        logits = t.zeros(self.R, self.K, self.V, device="cuda")
        prev, picked, flat = self.last, t.zeros(self.R, dtype=t.int32, device="cuda"), t.zeros(self.R, self.V, device="cuda")
        for k in range(self.K):
            binding.rgd_w4_matvec(self.embed[prev.long()], *self.w_head, None, 64, flat, dev_status=self.status)
            binding.rgd_sample_head(flat, self.probe, self.temp, self.min_p, self.seed, self.steps * 64 + k, None, picked,
                                    dev_status=self.status)
            logits[:, k], tokens[:, k] = flat, picked
            prev = picked.clone()
        return tokens, logits

    def step(self):
        """One step of every active row; returns its tokens [R, K + 1] (-1 behind the last) and how many were accepted."""
        t, R, P = self.torch, self.R, self.K + 1
        drafts, q_logits = self.propose()
        x = self.embed[t.cat([self.last[:, None], drafts], 1).long().view(-1)]
        qkv = t.empty(R * P, (self.Hq + 2 * self.Hkv) * self.D, dtype=t.bfloat16, device="cuda")
        binding.rgd_w4_matvec(x, *self.w_qkv, None, 64, qkv, dev_status=self.status)
        qkv = qkv.view(R, P, self.Hq + 2 * self.Hkv, self.D)
        k_new, v_new = qkv[:, :, self.Hq:self.Hq + self.Hkv], qkv[:, :, self.Hq + self.Hkv:]
        n = t.full((R,), P, dtype=t.int32, device="cuda")
        binding.rgd_cache_reserve(self.cache, self.table, self.length, n, self.active, self.refs, self.k, self.v, self.ok,
                                  self.ws, dev_status=self.status)
        binding.rgd_cache_write(self.cache, 0, k_new, v_new, n, self.table, self.length, self.ok, self.k, self.v,
                                dev_status=self.status)
        out = t.zeros(R * P, self.Hq, self.D, dtype=t.bfloat16, device="cuda")
        ends = (self.length[:, None] + 1 + t.arange(P, dtype=t.int32, device="cuda")).reshape(-1).contiguous()
        binding.rgd_prefix_decode_attn(self.attn, qkv[:, :, :self.Hq].contiguous(), self.k, self.v, self.prompt_table,
                                       self.prompt_len, self.table.repeat_interleave(P, 0), ends,
                                       self.active.repeat_interleave(P), 1 / math.sqrt(self.D), out, None, self.attn_ws,
                                       self.status)
        logits = t.empty(R * P, self.V, device="cuda")
        mixed = out.view(R * P, -1) + x  # (the residual stream)
        binding.rgd_w4_matvec(mixed, *self.w_head, None, 64, logits, dev_status=self.status)
        tokens = t.empty(R, P, dtype=t.int32, device="cuda")
        accepted = t.empty(R, dtype=t.int32, device="cuda")
        binding.rgd_verify_draft(logits.view(R, P, self.V), q_logits if self.K else None, drafts, None, self.probe, self.temp,
                                 self.min_p, t.rand(R, max(self.K, 1), device="cuda", generator=self.gen)[:, :self.K].contiguous(),
                                 t.rand(R, device="cuda", generator=self.gen), self.active, tokens, accepted, None,
                                 self.verify_ws, dev_status=self.status)
        # the token before the drafts and the accepted drafts stay in the cache, the others' pages go back
        on = self.active.int()
        self.length += (accepted + 1) * on
        binding.rgd_cache_trim(self.table, self.length, None, self.refs, dev_status=self.status)
        self.last = t.where(on > 0, tokens.gather(1, accepted[:, None].long())[:, 0], self.last)
        binding.rgd_probe_gate(self.trie, self.G, self.rpg, tokens, P, self.rpg * P, -1, 1 << 20, self.gate, None,
                               self.gate_status)
        self.steps += 1
        return tokens, accepted

    def fork(self, parent: int, child: int):
        """Row `child` starts over as a copy of row `parent`; what they share is copied when either writes."""
        t = self.torch
        only = t.zeros(self.R, dtype=t.uint8, device="cuda")
        only[child] = 1
        binding.rgd_cache_trim(self.table, t.zeros_like(self.length), only, self.refs, dev_status=self.status)
        pair = [t.tensor([i], dtype=t.int32, device="cuda") for i in (parent, child)]
        binding.rgd_cache_fork(*pair, self.table, self.length, self.refs, dev_status=self.status)
        self.last[child] = self.last[parent]

    def end(self, rows):
        """The rows give up their pages; the pages in use move to the front of the pool."""
        t = self.torch
        gone = t.zeros(self.R, dtype=t.uint8, device="cuda")
        gone[rows] = 1
        self.active[rows], self.length[rows] = 0, 0
        binding.rgd_cache_trim(self.table, self.length, gone, self.refs, dev_status=self.status)
        binding.rgd_cache_compact(self.cache, self.table, self.prompt_table, self.refs, self.k, self.v, self.live, self.ws,
                                  dev_status=self.status)
        return int(self.live.item())

    def check(self):
        self.torch.cuda.synchronize()
        status = int(self.status.item()) | (int(self.gate_status.item()) & ~binding.RGD_DEV_BAD_TOKEN)
        if status:
            raise RuntimeError(f"device status {status}")


def run(draft=3, steps=8, seed=0, **sizes):
    """Tokens of every row, and the mean number of accepted drafts a step."""
    d = Decoder(draft=draft, seed=seed, **sizes)
    got, accepted = [[] for _ in range(d.R)], 0.0
    for _ in range(steps):
        tokens, acc = d.step()
        accepted += float(acc.float().mean()) / steps
        for r, row in enumerate(tokens.tolist()):
            got[r] += [x for x in row if x >= 0]
    d.check()
    return d, got, accepted


def main():
    d, got, accepted = run()
    for r, row in enumerate(got):
        print(f"row {r} ({'probe' if r % d.rpg == 0 else 'sample'}): {len(row)} tokens, {row[:12]} ...")
    print(f"accepted {accepted:.2f} of {d.K} drafts a step; gate decisions",
          binding.decode_gate_state(d.gate)["decision"].tolist())
    d.fork(0, 1)
    d.step()
    live = d.end([2])
    d.step()
    d.check()
    print(f"row 1 forked from row 0, row 2 ended: {live} of {d.pages} pages in use")


if __name__ == "__main__":
    main()
