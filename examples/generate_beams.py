"""Beam search with merged experts: the block of generate_block.py, several continuations of every request over one paged cache.

The prompts are stored once.  Every step is one lory_kv_plan (places of the new tokens), one lory_qk_rope_cache, one lory_prefix_attn
(the prompt is read once for all beams of a request), the merged FFN (the beams of a request are the tokens of one sequence: they share
its merged parameters), lory_beam_select, lory_kv_fork (the cache's rows go on as the chosen beams) and lory_kv_copy.  Weights are
random; the embedding is the head's transpose.

    python examples/generate_beams.py [--beams 4] [--steps 32]
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from generate_block import Block, Requests, next_input, prefill  # noqa: E402
from paper_2405_03133_amd import binding as lb  # noqa: E402


class Beams:
    """A cache of `requests` whose rows are beams, and the second set of table, lengths and count that a fork writes."""

    def __init__(self, requests, lens, prompts, beams, pages):
        self.r, self.K, self.pages, self.prompts = requests, beams, pages, prompts
        i32 = lambda *shape: torch.zeros(*shape, dtype=torch.int32, device="cuda")
        n, W = prompts * beams, requests.table.shape[1]
        self.shared = lens.clone()
        self.table_new, self.copies, self.status = i32(n, W) - 1, i32(3, n), i32(1)
        self.fork(torch.arange(prompts, device="cuda", dtype=torch.int32).repeat_interleave(beams))
        self.table_new = i32(n, W) - 1
        requests.cu = i32(n + 1)

    def fork(self, src):
        """The cache's rows go on as rows src; src < 0 ends one."""
        r = self.r
        lens_new = torch.empty(src.shape[0], dtype=torch.int32, device="cuda")
        lb.lory_kv_fork(r.lens, src, r.table, r.free, r.count, r.page, self.pages, lens_new, self.table_new, r.count_new, self.copies,
                        self.status)
        lb.lory_kv_copy(r.k, r.v, self.copies)
        r.table, self.table_new = self.table_new, r.table
        r.lens, r.lens_new = lens_new, torch.empty_like(lens_new)
        r.count, r.count_new = r.count_new, r.count


def decode(block, beams, x, merged):
    """x [requests * beams, d] of the beams' tokens -> [requests * beams, d].  Every row has a token, so tokens are rows."""
    r, H, Hkv, D = beams.r, block.H, block.Hkv, block.D
    n = x.shape[0]
    positions, slots, _ = r.plan(torch.ones(n, dtype=torch.int32, device="cuda"), n)
    q, k, v = (t.unflatten(1, (-1, D)) for t in (x @ block.Wqkv).split([H * D, Hkv * D, Hkv * D], 1))
    q = lb.lory_qk_rope_cache(q, k, v, positions, block.freq, r.k, r.v, slots, wq=block.wq, wk=block.wk)
    h = x + lb.lory_prefix_attn(q, r.k, r.v, r.table, r.lens, beams.shared).flatten(1) @ block.Wo
    y = lb.lory_dense_ffn_fwd(h.view(beams.prompts, beams.K, -1), merged, block.d_ff)
    return h + y.view(n, -1)


def search(block, prompts, lens, head, K, steps, page=16):
    """The K best continuations of every prompt (prompts [B, L, d], `lens` tokens each) by `steps` tokens: (score [B, K], tokens
    [B, K, steps], status of the last plan and fork, free pages).  head [d, vocab]."""
    B, L, _ = prompts.shape
    longest = L + steps
    pages = B * -(-L // page) + B * K * (-(-steps // page) + 2)
    requests = Requests(block, B, pages, page, longest)
    h, merged = prefill(block, requests, prompts, lens)
    h = next_input(h[torch.arange(B, device="cuda"), lens.long() - 1])
    score, token, _ = lb.lory_beam_select(h @ head, torch.zeros(B, 1, device="cuda"), K)
    beams = Beams(requests, lens, B, K, pages)
    tokens = token[:, :, None]
    for _ in range(steps - 1):
        x = next_input(head.T[token.view(-1).long()].contiguous())
        h = next_input(decode(block, beams, x, merged))
        score, token, parent = lb.lory_beam_select(h @ head, score, K)
        beams.fork(parent.view(-1))
        tokens = torch.cat([tokens.flatten(0, 1)[parent.long()], token[:, :, None]], 2)
    return score, tokens, (requests.status, beams.status), requests.count


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--requests", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=512)
    ap.add_argument("--beams", type=int, default=4)
    ap.add_argument("--steps", type=int, default=32, help="at least 2")
    ap.add_argument("--vocab", type=int, default=32000)
    args = ap.parse_args()
    torch.manual_seed(0)
    block, B = Block(), args.requests
    head = (torch.randn(block.d, args.vocab, device="cuda") * block.d ** -0.5).to(block.dtype)
    lens = torch.linspace(1, args.prompt, B, device="cuda").int()
    prompts = torch.randn(B, args.prompt, block.d, device="cuda").to(block.dtype)
    search(block, prompts, lens, head, args.beams, 2)   # loads kernels
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    score, tokens, status, count = search(block, prompts, lens, head, args.beams, args.steps)
    torch.cuda.synchronize()
    print(f"{B} requests, {args.beams} beams, {args.steps} steps and the prompts in {(time.perf_counter() - t0) * 1e3:.1f} ms; best scores "
          f"{[round(s, 2) for s in score[:, 0].tolist()]}, status {[s.item() for s in status]}, {count.item()} pages free")


if __name__ == "__main__":
    main()
