"""State of a service around ``LagaBlock``: a pool of cache pages shared by a fixed number of request rows.

One token's entry is its normalised latent and its rotated shared key, 576 bf16 channels for all heads together.  The
tables are the same for every layer, so one ``LatentCache`` serves a stack of layers: ``pages[layer]`` is what a layer's
calls read and write.  Everything lives on the device and is updated there (laga_cache_plan); nothing here waits for the GPU.
"""
from __future__ import annotations

import torch

from . import laga


class CacheStep(laga.CachePlan):
    """A plan of a LatentCache.  Beside the plan's tensors, for the calls in which row b is request b's one new token: row_slots and
    row_lens (int32 [n_requests]), the plan's slots and lengths, -1 in rows that are not (see `rows_are_requests`)."""

    row_slots = row_lens = None


def rows_are_requests(step: laga.CachePlan, ranks: torch.Tensor):
    """(row_slots, row_lens) of a plan; ranks: int32 0 .. n_requests.  Token b of the step is request b's only one where b tokens come
    before the request's and b + 1 before the next: a request with none or with several moves those behind it to other rows."""
    n = ranks.numel() - 1
    same = step.cu_new_lens == ranks
    yes = same[1:] & same[:-1]
    return torch.where(yes, step.slots[:n], -1), torch.where(yes, step.seq_lens, -1)


class LatentCache:
    """n_pages pages of page_size tokens (a power of two from 16 to 1024) in each of n_layers layers; n_requests rows, each with
    room for max_tokens tokens (in whole pages: a plan takes up to ceil(max_tokens / page_size) * page_size)."""

    ROW = 576

    def __init__(self, n_pages: int, n_requests: int, max_tokens: int, page_size: int = 64, n_layers: int = 1, device="cuda"):
        if min(n_pages, n_requests, max_tokens, n_layers) < 1 or n_requests > 8192:
            raise ValueError("LatentCache: sizes must be at least 1, and n_requests at most 8192")
        if page_size not in (16, 32, 64, 128, 256, 512, 1024):
            raise ValueError(f"LatentCache: page_size must be a power of two from 16 to 1024, got {page_size}")
        i32 = dict(dtype=torch.int32, device=device)
        self.page_size, self.columns = page_size, -(-max_tokens // page_size)
        self.pages = [torch.zeros(n_pages, page_size, self.ROW, dtype=torch.bfloat16, device=device) for _ in range(n_layers)]
        self.block_table = torch.zeros(n_requests, self.columns, **i32)
        self.seq_lens = torch.zeros(n_requests, **i32)
        self.free_pages = torch.zeros(n_pages + 1, **i32)          # a stack; the last entry only absorbs what `release` drops
        self.free_pages[:n_pages] = torch.arange(n_pages - 1, -1, -1, **i32)
        self.n_free = torch.full((1,), n_pages, **i32)
        self._ranks = torch.arange(n_requests + 1, **i32)

    def plan(self, new_lens: torch.Tensor, max_tokens: int) -> CacheStep:
        """Places new_lens[b] (int32 [n_requests], on the device) tokens for each request and makes the result the cache's
        state.  A step that does not fit takes nothing and gives every row slot -1: ``laga.check_status(plan.status)`` tells."""
        step = CacheStep._make(laga.cache_plan(self.seq_lens, new_lens, self.block_table, self.free_pages, self.n_free, self.page_size,
                                               max_tokens))
        self.seq_lens.copy_(step.seq_lens)
        self.n_free.copy_(step.n_free)
        if max_tokens >= self.seq_lens.numel():                     # (once a step here, not once a layer in `LagaBlock.decode`)
            step.row_slots, step.row_lens = rows_are_requests(step, self._ranks)
        return step

    def release(self, request: int) -> None:
        """Gives a request's pages back and empties its row."""
        column = torch.arange(self.columns, device=self.seq_lens.device)
        held = (self.seq_lens[request] + self.page_size - 1) // self.page_size
        # behind the top of the stack; columns the request does not hold go to the spare last entry
        at = torch.where(column < held, self.n_free + column, self.free_pages.numel() - 1)
        self.free_pages.scatter_(0, at, self.block_table[request])
        self.n_free += held
        self.seq_lens[request] = 0
