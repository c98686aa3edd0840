"""The operators around one MLA attention layer in service and in training, each in its plain form and as the
library computes it: the rotary positions of the queries, the latent's norm with the shared key's rotation (dense for
training, written into a paged cache for serving), the page tables and slot maps of that cache, and the attention of
one new token over it.

``run`` computes in elementary torch operations where ``own`` is false and through the package's entry points where
it is true; ``exact`` is the definition in float64.
"""
import math

import torch

own = False

D_NOPE, D_ROPE, D_V, D_C = 128, 64, 128, 512        # the head geometry of this repository's configurations
ROW = D_C + D_ROPE                                  # one cached token: latent, then the shared rotated key
BF16 = torch.bfloat16
DEV = "cuda"


# ---- cases -------------------------------------------------------------------------------------------------
def listed():
    return [
        # One decode step of a small batch at far positions: a launch, nothing else.
        {"name": "rope decode 8x16", "op": "rope", "tokens": 8, "heads": 16, "far": 131072, "interleaved": True,
         "scaled": False, "inverse": False, "strided": False},
        # The queries of the per-rank training shard (16 heads of 16384 tokens).
        {"name": "rope train 16384x16", "op": "rope", "tokens": 16384, "heads": 16, "far": 0, "interleaved": True,
         "scaled": False, "inverse": False, "strided": False},
        # Backward of the rotation over all 128 heads (one rank, no sequence parallelism), half layout, long context.
        {"name": "rope backward 8192x128", "op": "rope", "tokens": 8192, "heads": 128, "far": 0, "interleaved": False,
         "scaled": True, "inverse": True, "strided": False},
        # Between W_kv_a and the attention of a training step, forward and backward.
        {"name": "latent forward 16384", "op": "latent", "tokens": 16384, "beta": True, "interleaved": True,
         "scaled": False},
        {"name": "latent backward 16384", "op": "latent_bwd", "tokens": 16384, "beta": True, "interleaved": True,
         "scaled": False},
        # One decode step of 61 requests in a batch padded to 64: the new tokens enter the cache.
        {"name": "append decode 64", "op": "append", "tokens": 64, "pad": 3, "page": 64, "pages": 2048,
         "interleaved": True, "scaled": True, "beta": True},
        # A prompt of 65536 tokens enters the cache.
        {"name": "append prompt 65536", "op": "append", "tokens": 65536, "pad": 0, "page": 64, "pages": 1152,
         "interleaved": True, "scaled": True, "beta": False},
        # Tables of a decode step: one token for each of 48 requests.
        {"name": "plan decode 48", "op": "plan", "requests": 48, "longest": 8192, "new_most": 1, "page": 64},
        # Tables of a step that mixes prompts and decodes: 1024 requests, some 130 thousand new tokens.
        {"name": "plan mixed 1024", "op": "plan", "requests": 1024, "longest": 4000, "new_most": 255, "page": 16},
        # One request, 16 heads, a short context: latency.
        {"name": "decode 1x511 h16", "op": "decode", "requests": 1, "shortest": 511, "longest": 511, "heads": 16, "page": 32},
        # A serving batch of the 16-head shard, ragged.
        {"name": "decode 64x8192 h16", "op": "decode", "requests": 64, "shortest": 1, "longest": 8192, "heads": 16, "page": 64},
        # All 128 heads on one GPU over long contexts.
        {"name": "decode 8x65536 h128", "op": "decode", "requests": 8, "shortest": 30001, "longest": 65536, "heads": 128,
         "page": 64},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "latent", "latent_bwd", "append", "plan", "decode", "decode", "decode"])
    if op == "rope":
        heads = rng.choice([1, 2, 3, 4, 8, 16, 32, 64, 128])
        return {"op": op, "tokens": _log(rng, 1, min(65536, 8192 * 128 // heads)), "heads": heads,
                "far": rng.choice([0, 4096, 131072, 4000000]), "interleaved": rng.random() < 0.5,
                "scaled": rng.random() < 0.5, "inverse": rng.random() < 0.5, "strided": heads == 1}
    if op in ("latent", "latent_bwd"):
        return {"op": op, "tokens": _log(rng, 1, 65536), "beta": rng.random() < 0.5, "interleaved": rng.random() < 0.5,
                "scaled": rng.random() < 0.5}
    page = rng.choice([16, 32, 64, 128, 256])
    if op == "append":
        tokens = _log(rng, 1, 65536)
        return {"op": op, "tokens": tokens, "pad": rng.randint(0, tokens // 8), "page": page,
                "pages": -(-tokens // page) + rng.randint(1, 64), "interleaved": rng.random() < 0.5,
                "scaled": rng.random() < 0.5, "beta": rng.random() < 0.5}
    if op == "plan":
        requests = _log(rng, 1, 2000)
        return {"op": op, "requests": requests, "longest": _log(rng, 1, 8192),
                "new_most": _log(rng, 1, min(8192, 131072 // requests)), "page": page}
    requests = _log(rng, 1, 256)
    longest = _log(rng, 1, min(65536, 524288 // requests))
    return {"op": op, "requests": requests, "shortest": rng.randint(0, longest), "longest": longest,
            "heads": rng.choice([1, 2, 4, 8, 16, 16, 24, 32, 64, 96, 128]), "page": page}


# ---- inputs ------------------------------------------------------------------------------------------------
def _inverse_frequencies(scaled):
    """Angles per position of the 32 rotated pairs, float64: base 10000; scaled: the long-context form that divides
    the slow pairs' frequencies by 40 and leaves the fast pairs', with a ramp between them and a factor on cos and sin."""
    i = torch.arange(D_ROPE // 2, dtype=torch.float64)
    fast = 10000.0 ** (-2 * i / D_ROPE)
    if not scaled:
        return fast, 1.0

    def pair_of(turns):                             # the pair that makes so many turns in 4096 positions
        return D_ROPE * math.log(4096 / (turns * 2 * math.pi)) / (2 * math.log(10000.0))

    low, high = math.floor(pair_of(32)), math.ceil(pair_of(1))
    slow_part = ((i - low) / (high - low)).clamp(0, 1)
    return fast * (1 - slow_part) + fast / 40 * slow_part, 0.1 * math.log(40.0) + 1.0


def _rotary(case, tokens, g, far=0):
    freqs, mscale = _inverse_frequencies(case["scaled"])
    positions = torch.arange(tokens, dtype=torch.int32)
    if far:
        positions = torch.randint(0, far, (tokens,), generator=g, dtype=torch.int32)
    return {"freqs": freqs.to(DEV), "mscale": mscale, "interleaved": case["interleaved"], "positions": positions.to(DEV)}


def _lengths(case, g):
    """The requests' lengths: spread evenly from the shortest to the longest, in an order of the seed's."""
    n, lo, hi = case["requests"], case["shortest"], case["longest"]
    lens = [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]
    return torch.tensor(lens, dtype=torch.int32)[torch.randperm(n, generator=g)]


def _latent_inputs(case, g, gd):
    """The output of W_kv_a: rows of order one with an offset and a spread of their own; gamma near one, beta near zero."""
    m = case["tokens"]
    x = torch.randn(m, ROW, generator=gd, device=DEV)
    x = x * (0.5 + 2 * torch.rand(m, 1, generator=gd, device=DEV)) + torch.randn(m, 1, generator=gd, device=DEV)
    beta = (0.1 * torch.randn(D_C, generator=g)).to(BF16).to(DEV)
    return {"kv_a": x.to(BF16), "gamma": (1 + 0.2 * torch.randn(D_C, generator=g)).to(BF16).to(DEV),
            "beta": beta if case["beta"] else None, "eps": 1e-5}


def prepare(case, seed):
    g = torch.Generator().manual_seed(seed)
    gd = torch.Generator(device=DEV).manual_seed(seed)
    op = case["op"]
    s = {"op": op}
    if op == "rope":
        s |= _rotary(case, case["tokens"], g, case["far"])
        s["inverse"] = case["inverse"]
        if case["strided"]:                         # the shared key where W_kv_a left it: a column slice
            s["x"] = torch.randn(case["tokens"], ROW, generator=gd, device=DEV).to(BF16)[:, D_C:].unsqueeze(1)
        else:
            s["x"] = torch.randn(case["tokens"], case["heads"], D_NOPE + D_ROPE, generator=gd, device=DEV).to(BF16)
    elif op in ("latent", "latent_bwd"):
        s |= _latent_inputs(case, g, gd) | _rotary(case, case["tokens"], g)
        if op == "latent_bwd":
            s["dlatent"] = torch.randn(case["tokens"], D_C, generator=gd, device=DEV).to(BF16)
            s["dk_pe"] = torch.randn(case["tokens"], D_ROPE, generator=gd, device=DEV).to(BF16)
            x = s["kv_a"][:, :D_C].double()         # what the forward kept
            s["mean"] = x.mean(1).float()
            s["rstd"] = (x.var(1, unbiased=False) + s["eps"]).rsqrt().float()
    elif op == "append":
        s |= _latent_inputs(case, g, gd) | _rotary(case, case["tokens"], g, 131072 if case["tokens"] <= 4096 else 0)
        n = case["tokens"] - case["pad"]
        if case["tokens"] <= 4096:                  # decodes: slots all over the cache
            slots = torch.randperm(case["pages"] * case["page"], generator=g)[:n]
        else:                                       # a prompt: whole pages in the order they were free
            pages = torch.randperm(case["pages"], generator=g)
            t = torch.arange(n)
            slots = pages[t // case["page"]] * case["page"] + t % case["page"]
        s["slots"] = torch.cat([slots, torch.full((case["pad"],), -1)]).to(torch.int32).to(DEV)
        s["cache"] = torch.randn(case["pages"], case["page"], ROW, generator=gd, device=DEV, dtype=BF16)
    elif op == "plan":
        n, page = case["requests"], case["page"]
        lens = torch.randint(0, case["longest"] + 1, (n,), generator=g, dtype=torch.int32)
        new = torch.randint(min(1, case["new_most"] - 1), case["new_most"] + 1, (n,), generator=g, dtype=torch.int32)
        columns = -(-(case["longest"] + case["new_most"]) // page)
        held = (lens + page - 1) // page
        more = int(((lens + new + page - 1) // page - held).sum())
        pool = torch.randperm(int(held.sum()) + more + 7, generator=g).to(torch.int32)
        table = torch.full((n, columns), -1, dtype=torch.int32)
        table[torch.arange(columns) < held[:, None]] = pool[: int(held.sum())]
        free = pool[int(held.sum()):]
        s |= {"seq_lens": lens.to(DEV), "new_lens": new.to(DEV), "block_table": table.to(DEV), "free_pages": free.to(DEV),
              "n_free": torch.tensor([len(free)], dtype=torch.int32, device=DEV), "page": page,
              "max_tokens": n * case["new_most"]}
    else:
        n, page, h = case["requests"], case["page"], case["heads"]
        lens = _lengths(case, g)
        columns = max(1, -(-case["longest"] // page))
        held = (lens + page - 1) // page
        pool = torch.randperm(int(held.sum()) + 5, generator=g).to(torch.int32)
        table = torch.zeros(n, columns, dtype=torch.int32)
        table[torch.arange(columns) < held[:, None]] = pool[: int(held.sum())]
        s |= {"q": torch.randn(n, h, D_NOPE + D_ROPE, generator=gd, device=DEV).to(BF16),
              "w_kv_b": (torch.randn(D_C, h * (D_NOPE + D_V), generator=gd, device=DEV) * D_C ** -0.5).to(BF16),
              "cache": torch.randn(len(pool), page, ROW, generator=gd, device=DEV, dtype=BF16),
              "block_table": table.to(DEV), "seq_lens": lens.to(DEV), "scale": (D_NOPE + D_ROPE) ** -0.5}
    return s


# ---- one pass ----------------------------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _PLAIN[s["op"]](s)


def _run_own(s):
    from paper_2607_17644_b200 import laga
    op = s["op"]
    if op == "plan":
        p = laga.cache_plan(s["seq_lens"], s["new_lens"], s["block_table"], s["free_pages"], s["n_free"],
                            page_size=s["page"], max_tokens=s["max_tokens"])
        return {"slots": p.slots, "positions": p.positions, "cu_new": p.cu_new_lens, "seq_lens": p.seq_lens,
                "n_free": p.n_free, "block_table": s["block_table"]}
    if op == "decode":
        return laga.paged_decode(s["q"], s["w_kv_b"], s["cache"], s["block_table"], s["seq_lens"],
                                 softmax_scale=s["scale"])[0]
    rope = laga.RopePlan(s["freqs"], s["mscale"], s["interleaved"])
    if op == "rope":
        return laga.rope(s["x"], s["positions"], rope, inverse=s["inverse"])
    if op == "latent":
        latent, k_pe, mean, rstd = laga.latent_norm_rope(s["kv_a"], s["gamma"], s["beta"], s["positions"], rope, eps=s["eps"])
        return {"latent": latent, "k_pe": k_pe, "mean": mean, "rstd": rstd}
    if op == "latent_bwd":
        dkv_a, dgamma, dbeta = laga.latent_norm_rope_backward(s["dlatent"], s["dk_pe"], s["kv_a"], s["gamma"], s["mean"],
                                                              s["rstd"], s["positions"], rope, with_beta=s["beta"] is not None)
        return {"dkv_a": dkv_a, "dgamma": dgamma, "dbeta": dbeta}
    return laga.cache_append(s["kv_a"], s["gamma"], s["beta"], s["positions"], rope, s["slots"], s["cache"], eps=s["eps"])


def _rotated(x, s, inverse=False):
    """The last 64 channels of x rotated (x in 32 bits; angles in 64: positions reach millions)."""
    angle = s["positions"].double()[:, None] * s["freqs"]
    cos, sin = (angle.cos() * s["mscale"]).float(), (angle.sin() * s["mscale"]).float()
    if inverse:
        sin = -sin
    shape = (x.shape[0],) + (1,) * (x.dim() - 2) + (D_ROPE // 2,)
    cos, sin = cos.view(shape), sin.view(shape)
    y = x.clone()
    r = y[..., x.shape[-1] - D_ROPE:]
    if s["interleaved"]:
        a, b = x[..., -D_ROPE::2], x[..., 1 - D_ROPE::2]
        r[..., 0::2], r[..., 1::2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., -D_ROPE:-D_ROPE // 2], x[..., -D_ROPE // 2:]
        r[..., : D_ROPE // 2], r[..., D_ROPE // 2:] = a * cos - b * sin, b * cos + a * sin
    return y


def _plain_rope(s):
    return _rotated(s["x"].float(), s, s["inverse"]).to(BF16)


def _norm(s):
    x = s["kv_a"][:, :D_C].float()
    mean = x.mean(1)
    rstd = 1 / ((x - mean[:, None]).square().mean(1) + s["eps"]).sqrt()
    y = (x - mean[:, None]) * rstd[:, None] * s["gamma"].float()
    return (y if s["beta"] is None else y + s["beta"].float()), mean, rstd


def _plain_latent(s):
    y, mean, rstd = _norm(s)
    return {"latent": y.to(BF16), "k_pe": _rotated(s["kv_a"][:, D_C:].float(), s).to(BF16), "mean": mean, "rstd": rstd}


def _plain_latent_bwd(s):
    dy = s["dlatent"].float()
    xhat = (s["kv_a"][:, :D_C].float() - s["mean"][:, None]) * s["rstd"][:, None]
    g = dy * s["gamma"].float()
    dx = s["rstd"][:, None] * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    return {"dkv_a": torch.cat([dx, _rotated(s["dk_pe"].float(), s, inverse=True)], 1).to(BF16),
            "dgamma": (dy * xhat).sum(0), "dbeta": None if s["beta"] is None else dy.sum(0)}


def _plain_append(s):
    rows = torch.cat([_norm(s)[0], _rotated(s["kv_a"][:, D_C:].float(), s)], 1).to(BF16)
    kept = s["slots"] >= 0
    s["cache"].view(-1, ROW)[s["slots"][kept].long()] = rows[kept]
    return s["cache"]


def _plain_plan(s):
    page, lens, new = s["page"], s["seq_lens"].long(), s["new_lens"].long()
    after = lens + new
    held, need = (lens + page - 1) // page, (after + page - 1) // page
    taken_before = (need - held).cumsum(0) - (need - held)
    table = s["block_table"]
    column = torch.arange(table.shape[1], device=DEV)
    fresh = (column >= held[:, None]) & (column < need[:, None])
    nth = taken_before[:, None] + column - held[:, None]
    top = s["n_free"].long() - 1
    page_of = s["free_pages"][(top - nth).clamp(0, s["free_pages"].numel() - 1)]
    table.copy_(torch.where(fresh, page_of, table))
    cu = torch.cat([torch.zeros(1, dtype=torch.long, device=DEV), new.cumsum(0)])
    t = torch.arange(s["max_tokens"], device=DEV)
    live = t < cu[-1]
    request = torch.searchsorted(cu[1:], t, right=True).clamp(max=lens.numel() - 1)
    position = lens[request] + t - cu[request]
    slot = table[request, (position // page).clamp(0, table.shape[1] - 1)].long() * page + position % page
    i32 = torch.int32
    return {"slots": torch.where(live, slot, -1).to(i32), "positions": torch.where(live, position, 0).to(i32),
            "cu_new": cu.to(i32), "seq_lens": after.to(i32), "n_free": (s["n_free"].long() - (need - held).sum()).to(i32),
            "block_table": table}


def _plain_decode(s):
    q, lens = s["q"].float(), s["seq_lens"].long()
    n, h = q.shape[:2]
    w = s["w_kv_b"].float().view(D_C, h, D_NOPE + D_V)
    held = torch.arange(s["block_table"].shape[1], device=DEV) * s["cache"].shape[1] < lens[:, None]
    rows = s["cache"][torch.where(held, s["block_table"], 0).long()].view(n, -1, ROW).float()
    q_lat = torch.cat([torch.einsum("bhn,chn->bhc", q[..., :D_NOPE], w[..., :D_NOPE]), q[..., D_NOPE:]], 2)
    scores = torch.matmul(q_lat, rows.transpose(1, 2)) * s["scale"]
    there = torch.arange(rows.shape[1], device=DEV) < lens[:, None]
    scores = torch.where(there[:, None], scores, -math.inf)
    top = scores.amax(2, keepdim=True)
    p = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(2, keepdim=True)
    o = torch.matmul(p, rows[..., :D_C]) / torch.where(total == 0, 1.0, total)
    return torch.einsum("bhc,chv->bhv", o, w[..., D_NOPE:]).to(BF16)


_PLAIN = {"rope": _plain_rope, "latent": _plain_latent, "latent_bwd": _plain_latent_bwd, "append": _plain_append,
          "plan": _plain_plan, "decode": _plain_decode}


# ---- the definitions in float64 ----------------------------------------------------------------------------
def _turned(v, s, back):
    """v [tokens, ..., 64] as 32 complex numbers for each head, each times mscale * exp(+-i * position * frequency)."""
    v = v.double()
    z = torch.view_as_complex(v.unflatten(-1, (-1, 2)).contiguous()) if s["interleaved"] else torch.complex(
        v[..., :D_ROPE // 2].contiguous(), v[..., D_ROPE // 2:].contiguous())
    phase = torch.outer(s["positions"].double(), s["freqs"]) * (-1.0 if back else 1.0)
    turn = torch.polar(torch.full_like(phase, s["mscale"]), phase)
    z = z * turn.reshape((v.shape[0],) + (1,) * (v.dim() - 2) + (-1,))
    return torch.view_as_real(z).flatten(-2) if s["interleaved"] else torch.cat([z.real, z.imag], -1)


def exact(case, seed):
    if case["op"] == "plan":                        # whole numbers
        return None
    s = prepare(case, seed)
    op = s["op"]
    if op == "rope":
        x = s["x"].double()
        return torch.cat([x[..., :-D_ROPE], _turned(x[..., -D_ROPE:], s, s["inverse"])], -1)
    if op == "decode":
        return _exact_decode(s)
    x = s["kv_a"][:, :D_C].double()
    gamma = s["gamma"].double()
    if op == "latent_bwd":
        # the Jacobian of the normalisation at the statistics that the forward kept
        xhat = (x - s["mean"].double()[:, None]) * s["rstd"].double()[:, None]
        dy = s["dlatent"].double()
        g = dy * gamma
        project = g - (g.sum(1, keepdim=True) + xhat * (xhat * g).sum(1, keepdim=True)) / D_C
        return {"dkv_a": torch.cat([project * s["rstd"].double()[:, None], _turned(s["dk_pe"], s, True)], 1),
                "dgamma": torch.einsum("mc,mc->c", dy, xhat), "dbeta": None if s["beta"] is None else dy.sum(0)}
    var, mean = torch.var_mean(x, 1, correction=0)
    rstd = (var + s["eps"]).pow(-0.5)
    y = torch.addcmul(torch.zeros_like(gamma) if s["beta"] is None else s["beta"].double(),
                      (x - mean[:, None]) * rstd[:, None], gamma)
    k_pe = _turned(s["kv_a"][:, D_C:], s, False)
    if op == "latent":
        return {"latent": y, "k_pe": k_pe, "mean": mean, "rstd": rstd}
    cache = s["cache"].double().view(-1, ROW)
    n = int((s["slots"] >= 0).sum())
    cache.index_copy_(0, s["slots"][:n].long(), torch.cat([y, k_pe], 1)[:n])
    return cache.view(s["cache"].shape)


def _exact_decode(s):
    """The explicit form, one request at a time: keys and values of every head from the latent, then softmax."""
    n, h = s["q"].shape[:2]
    page = s["cache"].shape[1]
    w = s["w_kv_b"].double().view(D_C, h, D_NOPE + D_V).permute(1, 0, 2)
    out = torch.zeros(n, h, D_V, dtype=torch.float64, device=DEV)
    for b in range(n):
        t = int(s["seq_lens"][b])
        if t == 0:
            continue
        pages = s["block_table"][b, : -(-t // page)].long()
        rows = s["cache"][pages].reshape(-1, ROW)[:t].double()
        most = max(1, (1 << 30) // (t * (D_NOPE + D_V) * 8))       # heads at a time: about 1 GB of keys and values
        for i in range(0, h, most):
            kv = rows[:, :D_C] @ w[i:i + most]                     # [heads, t, 256]
            q = s["q"][b, i:i + most].double()
            z = (torch.einsum("hn,htn->ht", q[:, :D_NOPE], kv[..., :D_NOPE]) + q[:, D_NOPE:] @ rows[:, D_C:].T) * s["scale"]
            out[b, i:i + most] = torch.einsum("ht,htv->hv", z.softmax(1), kv[..., D_NOPE:])
    return out


# ---- what a pass cannot do without -------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op == "rope":
        width = D_ROPE if case["strided"] else case["heads"] * (D_NOPE + D_ROPE)
        m = case["tokens"]
        return {"bytes": m * width * 4 + m * 4, "flops": m * case["heads"] * D_ROPE * 3}
    if op in ("latent", "append"):
        m = case["tokens"]
        return {"bytes": m * (ROW * 4 + (12 if op == "latent" else 8)) + 4 * D_C, "flops": m * (8 * D_C + 3 * D_ROPE)}
    if op == "latent_bwd":
        m = case["tokens"]
        return {"bytes": m * (ROW * 6 + 12) + 10 * D_C, "flops": m * (14 * D_C + 3 * D_ROPE)}
    if op == "plan":
        n, new = case["requests"], case["requests"] * (case["new_most"] + min(1, case["new_most"] - 1)) // 2
        return {"bytes": n * 16 + 8 * (new // case["page"]) + 8 * n * case["new_most"], "flops": 0}
    n, h = case["requests"], case["heads"]
    tokens = case["longest"] if n == 1 else n * (case["shortest"] + case["longest"]) // 2
    return {"bytes": tokens * (ROW * 2 + 4 / case["page"]) + n * h * (D_NOPE + D_ROPE + D_V) * 2 + D_C * h * (D_NOPE + D_V) * 2,
            "flops": tokens * h * 2 * (ROW + D_C) + n * h * 2 * D_C * (D_NOPE + D_V)}
