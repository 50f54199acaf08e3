"""From a batch of prompts to caches a verify step can read.

Host glue only: a PromptPass holds the device buffers of one model's pass over
a batch of prompts and issues its two calls on one stream:

  ipd_rope_append  rotary positions of the prompts' queries and keys, and the
                   write of their K/V rows into the model's paged cache
  ipd_prompt_attn  causal attention of the packed prompts

What lies between passes (projections, the LM head) is the caller's; the next
tokens come from ipd.sample_trunc on the last positions' logits, and from then
on the model proposes or verifies through VerifyStep over the same cache.
"""
from __future__ import annotations

import math
from typing import Optional, Sequence

import torch

from . import ipd


class PromptPass:
    """Buffers and calls of one model's pass over new prompts.

    cache: the model's ipd.KVCache; table: its rotary table ([max_pos, rot / 2,
    2], see ipd.rope_table); lens: the prompts' lengths (host ints, 0 allowed);
    page_table: [R, max_pages] int32 with the pages of every prompt, as a verify
    step takes it; num_q_heads: query heads.  The prompts start at position 0.
    """

    def __init__(self, cache: ipd.KVCache, table: torch.Tensor, lens: Sequence[int],
                 page_table: torch.Tensor, num_q_heads: int, layout: int = ipd.ROPE_HALF,
                 scale: float = 1.0 / math.sqrt(128.0), want_lse: bool = False, device="cuda"):
        lens = [int(n) for n in lens]
        if any(n < 0 for n in lens):
            raise ValueError("a prompt's length is negative")
        if lens and max(lens) > table.shape[0]:
            raise ValueError(f"a prompt of {max(lens)} tokens is longer than the rotary table")
        if page_table.shape[0] != len(lens):
            raise ValueError("one row of the page table a prompt")
        if lens and max(lens) > 16 * page_table.shape[1]:
            raise ValueError(f"a prompt of {max(lens)} tokens does not fit the page table's row")
        dev = torch.device(device)
        self.cache, self.table, self.layout, self.scale = cache, table, layout, scale
        self.lens, self.total, self.max_len = lens, sum(lens), max(lens, default=0)
        cu = torch.zeros(len(lens) + 1, dtype=torch.int32)
        cu[1:] = torch.tensor(lens, dtype=torch.int64).cumsum(0).to(torch.int32)
        self.cu = cu.to(dev)
        self.seq_len = torch.tensor(lens, dtype=torch.int32).to(dev)
        self.page_table = page_table.to(torch.int32).contiguous().to(dev)
        # positions of the prompts' last tokens among the packed rows (-1: empty)
        self.last = torch.tensor([int(c) - 1 if n else -1 for c, n in zip(cu[1:], lens)],
                                 dtype=torch.int64)
        bf = dict(dtype=torch.bfloat16, device=dev)
        self.q = torch.empty(self.total, num_q_heads, 128, **bf)
        self.k = torch.empty(self.total, cache.num_kv_heads, 128, **bf)
        self.out = torch.empty_like(self.q)
        self.lse: Optional[torch.Tensor] = (
            torch.empty(num_q_heads, self.total, dtype=torch.float32, device=dev) if want_lse else None)

    def run(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, stream=None) -> torch.Tensor:
        """The two calls on the prompts' projected rows (q [total, Hq, 128], k and
        v [total, Hkv, 128], before the rotation; views into one projection
        output are fine).  Returns the attention's output ([total, Hq, 128])."""
        ipd.rope_append(self.cache, q, self.q, k, v, self.cu, self.seq_len, self.page_table,
                        self.table, layout=self.layout, k_out=self.k, stream=stream)
        ipd.prompt_attn(self.q, self.k, v, self.cu, self.max_len, self.out, self.scale,
                        lse=self.lse, stream=stream)
        return self.out
