"""A transformer block that generates with merged experts: the attention operators and prompt-only routing together.

Requests with prompts of different lengths enter a step, generate token by token over a paged cache, and some end while
the others go on.  Every step is one lory_kv_plan (pages, positions, slots), one lory_qk_rope_cache (head norms,
rotation, store), one lory_paged_attn, and the merged FFN of each request (lory_prompt_merge on its prompt, then
lory_dense_ffn_fwd).  The projections are plain matrix products.  Weights and hidden states are random.

    python examples/generate_block.py [--steps 32]
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2405_03133_amd import binding as lb  # noqa: E402


class Block:
    """Weights of one block; everything in `dtype` (bf16 or fp32) on the GPU."""

    def __init__(self, d=1024, heads=16, kv_heads=4, head_dim=64, d_ff=2816, experts=8, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def normal(*shape, sigma=0.02):
            return (torch.randn(*shape, generator=g, device="cuda") * sigma).to(dtype)

        self.d, self.H, self.Hkv, self.D, self.d_ff, self.dtype = d, heads, kv_heads, head_dim, d_ff, dtype
        self.Wqkv, self.Wo = normal(d, (heads + 2 * kv_heads) * head_dim), normal(heads * head_dim, d)
        self.wq, self.wk = 1 + normal(head_dim, sigma=0.1), 1 + normal(head_dim, sigma=0.1)
        self.R = normal(d, experts, sigma=d ** -0.5)
        self.Wg, self.Wu, self.Wd = normal(experts, d, d_ff), normal(experts, d, d_ff), normal(experts, d_ff, d)
        self.freq = 10000.0 ** (-2.0 * torch.arange(head_dim // 2, device="cuda", dtype=torch.float64) / head_dim)


class Requests:
    """The paged cache of a block and what a step's plan needs: two sets of lengths and counts that change places."""

    def __init__(self, block, rows, pages, page, longest):
        i32 = lambda *shape: torch.zeros(*shape, dtype=torch.int32, device="cuda")
        self.page = page
        self.k, self.v = (torch.zeros(pages, block.Hkv, page, block.D, dtype=block.dtype, device="cuda") for _ in range(2))
        self.table = torch.full((rows, -(-longest // page)), -1, dtype=torch.int32, device="cuda")
        self.free = torch.arange(pages, dtype=torch.int32, device="cuda")
        self.lens, self.lens_new, self.cu, self.status = i32(rows), i32(rows), i32(rows + 1), i32(1)
        self.count, self.count_new = i32(1) + pages, i32(1)

    def plan(self, add, room):
        """Places `room` tokens at most; returns their positions and slots, and the request of each."""
        positions = torch.empty(room, dtype=torch.int32, device="cuda")
        slots = torch.empty(room, dtype=torch.int64, device="cuda")
        lb.lory_kv_plan(self.lens, add, self.table, self.free, self.count, self.page, self.lens_new, self.cu, positions, slots,
                        self.count_new, self.status)
        self.lens, self.lens_new = self.lens_new, self.lens
        self.count, self.count_new = self.count_new, self.count
        row = torch.searchsorted(self.cu[1:], torch.arange(room, device="cuda", dtype=torch.int32), right=True)
        return positions, slots, row.clamp_(max=add.shape[0] - 1)


def attention(block, requests, x, positions, slots, row):
    """x [tokens, d] of the step's tokens -> [tokens, d].  A token sees its request's cache up to itself, so a step may
    hold prompts as well as single tokens; places that no token fills (slot -1) are rows without a token."""
    H, Hkv, D = block.H, block.Hkv, block.D
    q, k, v = (t.unflatten(1, (-1, D)) for t in (x @ block.Wqkv).split([H * D, Hkv * D, Hkv * D], 1))
    q = lb.lory_qk_rope_cache(q, k, v, positions, block.freq, requests.k, requests.v, slots, wq=block.wq, wk=block.wk)
    seen = torch.where(slots >= 0, positions + 1, 0)
    out = lb.lory_paged_attn(q, requests.k, requests.v, requests.table[row], seen)
    return out.flatten(1) @ block.Wo


def prefill(block, requests, prompts, lens):
    """prompts [B, L, d], padded, of `lens` tokens -> (hidden states [B, L, d], the requests' merged FFN weights)."""
    B, L, d = prompts.shape
    _, merged = lb.lory_prompt_merge(prompts, block.R, block.Wg, block.Wu, block.Wd, prompt_len=lens)
    positions, slots, row = requests.plan(lens, B * L)
    at = row * L + positions                                 # the token's place among the padded ones
    x = prompts.reshape(B * L, d)
    y = attention(block, requests, x[at], positions, slots, row)
    filled = slots >= 0
    h = x.clone()
    h[at[filled]] += y[filled]
    h = h.view(B, L, d)
    return h + lb.lory_dense_ffn_fwd(h.contiguous(), merged, block.d_ff), merged


def decode(block, requests, x, active, merged):
    """One token for every active request: x [B, d] -> [B, d] (rows that are not active stay)."""
    B = x.shape[0]
    positions, slots, row = requests.plan(torch.where(active, 1, -1).int(), B)
    y = attention(block, requests, x[row], positions, slots, row)
    filled = (slots >= 0)[:, None]
    h = x.index_add(0, row, torch.where(filled, y, torch.zeros_like(y)))
    y = h + lb.lory_dense_ffn_fwd(h.view(B, 1, -1), merged, block.d_ff).view(B, -1)
    return torch.where(active[:, None], y, x)


def next_input(h):
    """In place of the model's head and embedding: the hidden state, scaled to what a prompt's tokens have."""
    return (h.float() * h.float().square().mean(-1, keepdim=True).rsqrt()).to(h.dtype)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--requests", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=512)
    ap.add_argument("--steps", type=int, default=32, help="at least 2")
    args = ap.parse_args()
    torch.manual_seed(0)
    block, B = Block(), args.requests
    page, longest = 16, args.prompt + args.steps
    requests = Requests(block, B, B * -(-longest // page), page, longest)
    lens = torch.linspace(1, args.prompt, B, device="cuda").int()
    prompts = torch.randn(B, args.prompt, block.d, device="cuda").to(block.dtype)
    h, merged = prefill(block, requests, prompts, lens)
    x = next_input(h[torch.arange(B, device="cuda"), lens.long() - 1])
    active = torch.ones(B, dtype=torch.bool, device="cuda")
    t0 = 0.0
    for step in range(args.steps):
        if step == 1:   # the first step also loads kernels
            torch.cuda.synchronize()
            t0 = time.perf_counter()
        if step == args.steps // 2:
            active = active & (torch.arange(B, device="cuda") % 4 != 3)   # every fourth request ends; its pages come back
        x = next_input(decode(block, requests, x, active, merged))
    torch.cuda.synchronize()
    ms = (time.perf_counter() - t0) / (args.steps - 1) * 1e3
    print(f"{B} requests, {args.steps} steps, {ms:.2f} ms a step; lengths {requests.lens.tolist()}, "
          f"{requests.count.item()} pages free, status {requests.status.item()}")


if __name__ == "__main__":
    main()
