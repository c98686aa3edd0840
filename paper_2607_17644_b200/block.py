"""Algorithm 1 of the paper as one differentiable block for SP degree 1 (no exchange steps), with every
step executed by the library's kernels:

  step 1   q = W_q(h);  latent, k_pe = W_kv_a(h);  latent = LayerNorm(latent)      laga_linear x2, laga_layernorm
  step 4-5 K_nope/V up-projection of the head shard and causal softmax attention   laga_fwd / laga_bwd
  step 7   W_o(reshape(out))                                                        laga_linear

Steps 2, 3 and 6 are the sequence-parallel exchanges (``sp.py``); with one rank they are the identity.
This module is torch.autograd plumbing only: ``autograd.Function``s that hand tensors to the C ABI
entry points and a module that owns the block's weights.  As in Algorithm 1, q_rope and k_pe are taken as
the projections deliver them (the paper's algorithm has no rotary step of its own) unless the block is given a
rotation (``rope``, from ``laga.rope_plan``): then step 1 ends with laga_rope on the queries, and laga_latent_norm_rope
takes the latent's norm and the key's rotation in one pass over what W_kv_a delivers.

In service the block keeps, per token, the normalised latent and the rotated key in a paged cache (``serving.LatentCache``):
``prefill`` runs prompts through the path above and fills the cache, ``decode`` adds one token per request and attends
to the cache through laga_paged_decode.

Weights are stored as [in_features, out_features] (y = x W), the layout ``W_kv_b`` already has.  Weight
gradients leave the kernels in fp32 and are handed to autograd in the weight's dtype.
"""
from __future__ import annotations

import torch

from . import laga
from .autograd import first_order, laga_attention
from .serving import rows_are_requests


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w):
        y, status = laga.linear(x, w)
        ctx.save_for_backward(x, w)
        return y

    @staticmethod
    @first_order
    def backward(ctx, dy):
        x, w = ctx.saved_tensors
        dx, dw, _ = laga.linear_backward(dy.contiguous(), x, w)
        return dx, dw.to(w.dtype)


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gamma, beta, eps):
        y, mean, rstd = laga.layernorm(x, gamma, beta, eps)
        ctx.save_for_backward(x, gamma, mean, rstd)
        ctx.has_beta = beta is not None
        return y

    @staticmethod
    @first_order
    def backward(ctx, dy):
        x, gamma, mean, rstd = ctx.saved_tensors
        dx, dgamma, dbeta = laga.layernorm_backward(dy.contiguous(), x, gamma, mean, rstd, with_beta=ctx.has_beta)
        return dx, dgamma.to(gamma.dtype), (dbeta.to(gamma.dtype) if ctx.has_beta else None), None


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, positions, rope):
        ctx.save_for_backward(positions, rope.freqs)
        ctx.mscale, ctx.interleaved = rope.mscale, rope.interleaved
        return laga.rope(x, positions, rope)

    @staticmethod
    @first_order
    def backward(ctx, dy):
        positions, freqs = ctx.saved_tensors
        return laga.rope(dy.contiguous(), positions, laga.RopePlan(freqs, ctx.mscale, ctx.interleaved), inverse=True), None, None


class _LatentNormRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, kv_a, gamma, beta, positions, rope, eps):
        latent, k_pe, mean, rstd = laga.latent_norm_rope(kv_a, gamma, beta, positions, rope, eps)
        ctx.save_for_backward(kv_a, gamma, mean, rstd, positions, rope.freqs)
        ctx.mscale, ctx.interleaved, ctx.has_beta = rope.mscale, rope.interleaved, beta is not None
        return latent, k_pe

    @staticmethod
    @first_order
    def backward(ctx, dlatent, dk_pe):
        kv_a, gamma, mean, rstd, positions, freqs = ctx.saved_tensors
        dkv_a, dgamma, dbeta = laga.latent_norm_rope_backward(dlatent.contiguous(), dk_pe.contiguous(), kv_a, gamma, mean, rstd, positions,
                                                              laga.RopePlan(freqs, ctx.mscale, ctx.interleaved),
                                                              with_beta=ctx.has_beta)
        return dkv_a, dgamma.to(gamma.dtype), (dbeta.to(gamma.dtype) if ctx.has_beta else None), None, None, None


def rotary(x: torch.Tensor, positions: torch.Tensor, rope) -> torch.Tensor:
    """The last channels of every head of x [S, h, d] rotated, through laga_rope (differentiable in x)."""
    return _Rotary.apply(x, positions, rope)


def latent_norm_rope(kv_a, gamma, beta, positions, rope, eps: float = 1e-5):
    """(latent, k_pe) from the output of W_kv_a, through laga_latent_norm_rope / laga_latent_norm_rope_backward."""
    return _LatentNormRope.apply(kv_a, gamma, beta, positions, rope, eps)


def linear(x: torch.Tensor, w: torch.Tensor) -> torch.Tensor:
    """y[M, N] = x[M, K] . w[K, N] through laga_linear / laga_linear_backward (bf16 CUDA tensors)."""
    return _Linear.apply(x, w)


def layernorm(x: torch.Tensor, gamma: torch.Tensor, beta=None, eps: float = 1e-5) -> torch.Tensor:
    """LayerNorm over the last axis through laga_layernorm / laga_layernorm_backward (bf16 CUDA tensors)."""
    return _LayerNorm.apply(x, gamma, beta, eps)


class LagaBlock(torch.nn.Module):
    """hidden [S, d_model] -> [S, d_model]: Algorithm 1 with P = 1 for ``n_heads`` heads of the DeepSeek-V3
    geometry (d_nope 128, d_rope 64, d_v 128, d_c 512).  ``forward(hidden, cu_seqlens=None)``: with
    ``cu_seqlens`` the rows are packed sequences and attention stays inside each.  ``rope``: the rotation of the rope bands
    (``laga.rope_plan``); None takes them as the projections deliver them, and the block then has no prefill / decode.
    ``softmax_scale``: the factor on the scores in training and service (default 192^-0.5).  YaRN's factor is one on whole scores, and a
    plan's mscale reaches the 64 rotated channels of the 192 alone: with it give the plan mscale_weight 0 and the block
    192^-0.5 * (0.1 ln(factor) + 1)^2."""

    D_NOPE, D_ROPE, D_V, D_C = 128, 64, 128, 512

    def __init__(self, d_model: int, n_heads: int, eps: float = 1e-5, device="cuda", seed: int = 0, rope=None, softmax_scale=None):
        super().__init__()
        self.rope, self.softmax_scale = rope, softmax_scale
        g = torch.Generator().manual_seed(seed)

        def weight(k, n):     # variance-preserving draw, rounded once to bf16
            return torch.nn.Parameter((torch.randn(k, n, generator=g) * k ** -0.5).to(torch.bfloat16).to(device))

        d_qk = self.D_NOPE + self.D_ROPE
        self.n_heads, self.eps = n_heads, eps
        self.w_q = weight(d_model, n_heads * d_qk)
        self.w_kv_a = weight(d_model, self.D_C + self.D_ROPE)
        self.w_kv_b = weight(self.D_C, n_heads * (self.D_NOPE + self.D_V))
        self.w_o = weight(n_heads * self.D_V, d_model)
        self.ln_gamma = torch.nn.Parameter(torch.ones(self.D_C, dtype=torch.bfloat16, device=device))
        self.ln_beta = torch.nn.Parameter(torch.zeros(self.D_C, dtype=torch.bfloat16, device=device))

    @staticmethod
    def positions(n_tokens: int, cu_seqlens=None, device="cuda") -> torch.Tensor:
        """int32 [n_tokens]: each token's place in its sequence (the rows are one sequence without cu_seqlens)."""
        pos = torch.arange(n_tokens, dtype=torch.int32)
        for begin, end in zip(cu_seqlens[:-1], cu_seqlens[1:]) if cu_seqlens is not None else ():
            pos[int(begin):int(end)] -= int(begin)
        return pos.to(device, non_blocking=True)

    def _project(self, hidden, positions):
        """Step 1: queries, latent and shared key."""
        S = hidden.shape[0]
        q = linear(hidden, self.w_q).view(S, self.n_heads, self.D_NOPE + self.D_ROPE)
        kv_a = linear(hidden, self.w_kv_a)
        if self.rope is None:
            latent = layernorm(kv_a[:, :self.D_C].contiguous(), self.ln_gamma, self.ln_beta, self.eps)
            return q, latent, kv_a[:, self.D_C:].contiguous()
        return (rotary(q, positions, self.rope),
                *latent_norm_rope(kv_a, self.ln_gamma, self.ln_beta, positions, self.rope, self.eps))

    def forward(self, hidden: torch.Tensor, cu_seqlens=None, causal: bool = True, positions=None) -> torch.Tensor:
        """positions (int32 [S] on the device, only with ``rope``): by default each token's place in its sequence, which
        the call then copies from the host (give them to capture a step in a graph)."""
        S = hidden.shape[0]
        if self.rope is not None and positions is None:
            positions = self.positions(S, cu_seqlens, hidden.device)
        q, latent, k_pe = self._project(hidden, positions)                                        # step 1
        out = laga_attention(q, latent, k_pe, self.w_kv_b, causal=causal, softmax_scale=self.softmax_scale,
                             cu_seqlens=cu_seqlens)                                               # steps 4-5
        return linear(out.reshape(S, self.n_heads * self.D_V), self.w_o)                          # step 7

    def _service(self):
        if self.rope is None:
            raise ValueError("prefill and decode need the block's rotation: LagaBlock(..., rope=laga.rope_plan(64))")

    @staticmethod
    def _not_these_prompts(step, positions, slots, cu_seqlens) -> torch.Tensor:
        """A truth value on the device: the plan was not placed, or its rows are not prompts with these boundaries from position 0 on (rows
        without a slot are padding).  Where it is so, the plan's status says it (detail 0x50000005)."""
        row = wanted = torch.arange(positions.numel(), dtype=torch.int32, device=positions.device)
        if cu_seqlens is not None:
            cu = torch.as_tensor(cu_seqlens, dtype=torch.int32).to(positions.device, non_blocking=True)
            wanted = row - cu[torch.searchsorted(cu, row, right=True) - 1]
        refused = ((positions != wanted) & (slots >= 0)).any() | (step.status[0] != 0)
        step.status.masked_fill_(refused & (step.status == 0), 0x50000005)
        return refused

    @torch.no_grad()
    def prefill(self, hidden: torch.Tensor, pages: torch.Tensor, step, cu_seqlens, workspace=None) -> torch.Tensor:
        """Prompts of requests that have nothing in the cache yet, packed: hidden [T, d_model], cu_seqlens their host
        boundaries (the same lengths that ``step``, a plan of ``LatentCache.plan``, was made for), pages one layer's
        cache [n_pages, page_size, 576].  Returns the block's output [T, d_model]; the cache holds the prompts afterwards.
        workspace (``laga.fwd_varlen_workspace_bytes``): give one to have the attention's status, as for ``decode``.
        A step that is not that -- a request held tokens already, other lengths, a plan that could not be placed -- is refused on the
        device: nothing enters the cache, the output is NaN, and ``laga.check_status(step.status)`` raises LAGA_ERR_CACHE_PLAN."""
        self._service()
        T = hidden.shape[0]
        q = laga.linear(hidden, self.w_q)[0].view(T, self.n_heads, self.D_NOPE + self.D_ROPE)
        kv_a = laga.linear(hidden, self.w_kv_a)[0]
        positions, slots = step.positions[:T], step.slots[:T]
        refused = self._not_these_prompts(step, positions, slots, cu_seqlens)
        slots, gamma = torch.where(refused, -1, slots), torch.where(refused, float("nan"), self.ln_gamma)
        laga.rope(q, positions, self.rope, y=q)
        latent, k_pe, _, _ = laga.latent_norm_rope(kv_a, gamma, self.ln_beta, positions, self.rope, self.eps, cache=pages, slots=slots)
        out = laga.fwd(q, latent, k_pe, self.w_kv_b, softmax_scale=self.softmax_scale, workspace=workspace, cu_seqlens=cu_seqlens)[0]
        return laga.linear(out.view(T, self.n_heads * self.D_V), self.w_o)[0]

    @torch.no_grad()
    def decode(self, hidden: torch.Tensor, pages: torch.Tensor, step, block_table: torch.Tensor, workspace=None, requests=None) -> torch.Tensor:
        """One new token for each of B requests: hidden [B, d_model], ``step`` a plan that gives every request one token,
        block_table the plan's table [B, columns].  After a plan that does not, rows that are not their request's one token are refused
        on the device: nothing of them enters the cache, their attention is zeros, the workspace's status LAGA_ERR_DEVICE_CHECK.
        Where the plan gave only some requests a token, ``requests`` (int64 [B], on the device, ascending) names them; rows of
        ``hidden`` behind the plan's tokens are padding (any request's number, results to be ignored).
        Appends the tokens' latents and keys to ``pages`` and attends to each request's whole cache, the new token included.  Every call reads lengths and tables on the device, so a step can be captured in a
        graph (with a workspace of its own, ``laga.paged_decode_workspace_bytes``) and replayed.  A page number outside the cache or a
        length outside the table shows only in the workspace's status: give one, and ``laga.check_status(workspace)`` raises
        (with no workspace given, nothing of it is left to ask)."""
        self._service()
        B = hidden.shape[0]
        q = laga.linear(hidden, self.w_q)[0].view(B, self.n_heads, self.D_NOPE + self.D_ROPE)
        kv_a = laga.linear(hidden, self.w_kv_a)[0]
        positions = step.positions[:B]
        if requests is not None:
            slots, block_table, lens = step.slots[:B], block_table.index_select(0, requests), step.seq_lens.index_select(0, requests)
        elif getattr(step, "row_lens", None) is not None:
            slots, lens = step.row_slots, step.row_lens
        else:                                    # a plan of laga.cache_plan itself
            slots, lens = rows_are_requests(step, torch.arange(B + 1, dtype=torch.int32, device=hidden.device))
        laga.rope(q, positions, self.rope, y=q)
        laga.cache_append(kv_a, self.ln_gamma, self.ln_beta, positions, self.rope, slots, pages, eps=self.eps)
        out = laga.paged_decode(q, self.w_kv_b, pages, block_table, lens, softmax_scale=self.softmax_scale, workspace=workspace)[0]
        return laga.linear(out.view(B, self.n_heads * self.D_V), self.w_o)[0]
