"""The paged latent cache held in 8 bits, each operator in its plain form and as the library computes it: tokens quantised as they
enter the cache, rows read back from it, and the attention of one new token over it.

A page of n tokens is n * 644 bytes: n rows of 640 e4m3 codes, then the rows' n fp32 scales.  A row holds the 512 latent channels,
the 64 channels of the rotated key, and 64 codes of what the key's first codes left: latent = scale * code, key = scale * (code +
second code).  The scale is the smallest power of two, 2^-32 at least, that brings every channel within 448.

``run`` computes in elementary torch operations where ``own`` is false and through the package's entry points where
it is true; ``exact`` is the definition in float64.
"""
import math

import torch

own = False

D_NOPE, D_ROPE, D_V, D_C = 128, 64, 128, 512        # the head geometry of this repository's configurations
ROW, CODES, TOKEN = D_C + D_ROPE, D_C + 2 * D_ROPE, D_C + 2 * D_ROPE + 4
BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn
DEV = "cuda"


# ---- cases -------------------------------------------------------------------------------------------------
def listed():
    return [
        # One decode step of 61 requests in a batch padded to 64: the new tokens enter the cache, and what it holds of them comes back.
        {"name": "write decode 64", "op": "write", "tokens": 64, "pad": 3, "page": 64, "pages": 2048, "interleaved": True, "beta": True},
        # A packed batch of prompts of 16384 tokens enters the cache, and is read back for its attention.
        {"name": "write prompt 16384", "op": "write", "tokens": 16384, "pad": 0, "page": 64, "pages": 1152, "interleaved": True,
         "beta": True},
        # A long prompt, half layout of the rotated pairs, small pages.
        {"name": "write prompt 65535", "op": "write", "tokens": 65535, "pad": 0, "page": 16, "pages": 4352, "interleaved": False,
         "beta": False},
        # A short request read back to move it elsewhere.
        {"name": "read 511", "op": "read", "tokens": 511, "pad": 1, "page": 32, "pages": 256},
        # A batch of requests read back: some 130 thousand tokens.
        {"name": "read 131072", "op": "read", "tokens": 131072, "pad": 5, "page": 64, "pages": 2176},
        # One request, 16 heads, a short context: latency.
        {"name": "decode 1x511 h16", "op": "decode", "requests": 1, "shortest": 511, "longest": 511, "heads": 16, "page": 32},
        # A serving batch of the 16-head shard, ragged.
        {"name": "decode 64x8192 h16", "op": "decode", "requests": 64, "shortest": 1, "longest": 8192, "heads": 16, "page": 64},
        # A shard of 32 heads, contexts of nearly one length.
        {"name": "decode 200x2048 h32", "op": "decode", "requests": 200, "shortest": 1900, "longest": 2048, "heads": 32, "page": 128},
        # Many short requests, 64 heads, small pages.
        {"name": "decode 250x600 h64", "op": "decode", "requests": 250, "shortest": 0, "longest": 600, "heads": 64, "page": 16},
        # All 128 heads on one GPU over long contexts.
        {"name": "decode 8x65536 h128", "op": "decode", "requests": 8, "shortest": 30001, "longest": 65536, "heads": 128,
         "page": 64},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["write", "read", "decode", "decode", "decode"])
    page = rng.choice([16, 32, 64, 128, 256])
    if op in ("write", "read"):
        tokens = _log(rng, 1, 65536 if op == "write" else 131072)
        case = {"op": op, "tokens": tokens, "pad": rng.randint(0, tokens // 8), "page": page, "pages": -(-tokens // page) + rng.randint(1, 64)}
        if op == "write":
            case |= {"interleaved": rng.random() < 0.5, "beta": rng.random() < 0.5}
        return case
    requests = _log(rng, 1, 256)
    longest = _log(rng, 1, min(65536, 524288 // requests))
    return {"op": op, "requests": requests, "shortest": rng.randint(0, longest), "longest": longest,
            "heads": rng.choice([1, 2, 4, 8, 16, 16, 24, 32, 64, 96, 128]), "page": page}


# ---- the cache's rows ----------------------------------------------------------------------------------------
def _planes(cache):
    """(codes [pages, page, 640], scales fp32 [pages, page]) of a cache, as views."""
    page = cache.shape[1] // TOKEN
    return cache[:, : page * CODES].unflatten(1, (page, CODES)), cache[:, page * CODES:].view(torch.float32)


def _encode(rows):
    """rows fp32 [n, 576] -> (codes uint8 [n, 640], scales fp32 [n])."""
    mantissa, exponent = torch.frexp(rows.abs().amax(1))
    exponent = (exponent - 9 + (mantissa > 0.875)).clamp(min=-32)
    scale = torch.ldexp(torch.ones_like(mantissa), exponent)
    x = rows / scale[:, None]
    code = x.to(E4M3)
    rest = (x[:, D_C:] - code[:, D_C:].float()).to(E4M3)
    return torch.cat([code.view(torch.uint8), rest.view(torch.uint8)], 1), scale


def _decode(codes, scales):
    """codes uint8 [..., 640], scales [...] -> rows fp32 [..., 576]."""
    x = codes.view(E4M3).float()
    return torch.cat([x[..., :D_C], x[..., D_C:ROW] + x[..., ROW:]], -1) * scales[..., None]


# ---- inputs ------------------------------------------------------------------------------------------------
def _random_cache(n_pages, page, gd):
    """A cache of normalised latents with a gain of their own each, and keys."""
    cache = torch.empty(n_pages, page * TOKEN, dtype=torch.uint8, device=DEV)
    codes, scales = _planes(cache)
    step = max(1, (1 << 20) // page)                # some million rows at a time
    for i in range(0, n_pages, step):
        n = min(step, n_pages - i) * page
        rows = torch.randn(n, ROW, generator=gd, device=DEV) * (0.5 + torch.rand(n, 1, generator=gd, device=DEV))
        c, s = _encode(rows)
        codes[i:i + step], scales[i:i + step] = c.view(-1, page, CODES), s.view(-1, page)
    return cache


def _slots(case, g):
    """Rows all over the cache where few, whole pages in a random order where many; the padding at the end has none."""
    n = case["tokens"] - case["pad"]
    if case["tokens"] <= 4096:
        slots = torch.randperm(case["pages"] * case["page"], generator=g)[:n]
    else:
        pages, t = torch.randperm(case["pages"], generator=g), torch.arange(n)
        slots = pages[t // case["page"]] * case["page"] + t % case["page"]
    return torch.cat([slots, torch.full((case["pad"],), -1)]).to(torch.int32).to(DEV)


def prepare(case, seed):
    g = torch.Generator().manual_seed(seed)
    gd = torch.Generator(device=DEV).manual_seed(seed)
    op, page = case["op"], case["page"]
    s = {"op": op}
    if op in ("write", "read"):
        s |= {"slots": _slots(case, g), "cache": _random_cache(case["pages"], page, gd)}
    if op == "write":                               # what W_kv_a delivers: rows of order one with an offset and a spread of their own
        m = case["tokens"]
        x = torch.randn(m, ROW, generator=gd, device=DEV)
        x = x * (0.5 + 2 * torch.rand(m, 1, generator=gd, device=DEV)) + torch.randn(m, 1, generator=gd, device=DEV)
        beta = (0.1 * torch.randn(D_C, generator=g)).to(BF16).to(DEV)
        positions = torch.randint(0, 131072, (m,), generator=g) if m <= 4096 else torch.arange(m)
        s |= {"kv_a": x.to(BF16), "gamma": (1 + 0.2 * torch.randn(D_C, generator=g)).to(BF16).to(DEV),
              "beta": beta if case["beta"] else None, "eps": 1e-5, "positions": positions.to(torch.int32).to(DEV),
              "freqs": (10000.0 ** (-torch.arange(0, D_ROPE, 2, dtype=torch.float64) / D_ROPE)).to(DEV),
              "interleaved": case["interleaved"]}
    elif op == "decode":
        n, h = case["requests"], case["heads"]
        lo, hi = case["shortest"], case["longest"]  # lengths spread evenly, in an order of the seed's
        lens = torch.tensor([hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)], dtype=torch.int32)
        lens = lens[torch.randperm(n, generator=g)]
        held = (lens + page - 1) // page
        pool = torch.randperm(int(held.sum()) + 5, generator=g).to(torch.int32)
        table = torch.zeros(n, max(1, -(-hi // page)), dtype=torch.int32)
        table[torch.arange(table.shape[1]) < held[:, None]] = pool[: int(held.sum())]
        s |= {"q": torch.randn(n, h, D_NOPE + D_ROPE, generator=gd, device=DEV).to(BF16),
              "w_kv_b": (torch.randn(D_C, h * (D_NOPE + D_V), generator=gd, device=DEV) * D_C ** -0.5).to(BF16),
              "cache": _random_cache(len(pool), page, gd), "block_table": table.to(DEV), "seq_lens": lens.to(DEV),
              "scale": (D_NOPE + D_ROPE) ** -0.5}
    return s


# ---- one pass ----------------------------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _PLAIN[s["op"]](s)


def _run_own(s):
    from paper_2607_17644_b200 import laga
    if s["op"] == "decode":
        return laga.paged_decode(s["q"], s["w_kv_b"], s["cache"], s["block_table"], s["seq_lens"], softmax_scale=s["scale"])[0]
    if s["op"] == "write":
        laga.cache_append(s["kv_a"], s["gamma"], s["beta"], s["positions"], laga.RopePlan(s["freqs"], 1.0, s["interleaved"]),
                          s["slots"], s["cache"], eps=s["eps"])
    latent, k_pe = laga.cache_read(s["cache"], s["slots"])
    return {"latent": latent, "k_pe": k_pe}


def _plain_read(s):
    codes, scales = _planes(s["cache"])
    page, slot = codes.shape[1], s["slots"].long().clamp(min=0)
    rows = _decode(codes[slot // page, slot % page], scales[slot // page, slot % page])
    rows = torch.where(s["slots"][:, None] >= 0, rows, 0.0)          # a row without a slot is zeros
    return {"latent": rows[:, :D_C].to(BF16), "k_pe": rows[:, D_C:].to(BF16)}


def _plain_write(s):
    x = s["kv_a"].float()
    c = x[:, :D_C] - x[:, :D_C].mean(1, keepdim=True)
    y = c / (c.square().mean(1, keepdim=True) + s["eps"]).sqrt() * s["gamma"].float()
    if s["beta"] is not None:
        y = y + s["beta"].float()
    angle = s["positions"].double()[:, None] * s["freqs"]            # (in 64 bits: positions are far)
    cos, sin = angle.cos().float(), angle.sin().float()
    if s["interleaved"]:
        a, b = x[:, D_C::2], x[:, D_C + 1::2]
        key = torch.stack([a * cos - b * sin, b * cos + a * sin], 2).flatten(1)
    else:
        a, b = x[:, D_C:D_C + D_ROPE // 2], x[:, D_C + D_ROPE // 2:]
        key = torch.cat([a * cos - b * sin, b * cos + a * sin], 1)
    code, scale = _encode(torch.cat([y, key], 1))
    codes, scales = _planes(s["cache"])
    kept = s["slots"] >= 0
    slot, page = s["slots"][kept].long(), codes.shape[1]
    codes[slot // page, slot % page], scales[slot // page, slot % page] = code[kept], scale[kept]
    return _plain_read(s)


def _plain_decode(s):
    q, lens = s["q"].float(), s["seq_lens"].long()
    n, h = q.shape[:2]
    w = s["w_kv_b"].float().view(D_C, h, D_NOPE + D_V)
    codes, scales = _planes(s["cache"])
    held = torch.arange(s["block_table"].shape[1], device=DEV) * codes.shape[1] < lens[:, None]
    pages = torch.where(held, s["block_table"], 0).long()
    rows = _decode(codes[pages], scales[pages]).flatten(1, 2)
    q_lat = torch.cat([torch.einsum("bhn,chn->bhc", q[..., :D_NOPE], w[..., :D_NOPE]), q[..., D_NOPE:]], 2)
    scores = torch.matmul(q_lat, rows.transpose(1, 2)) * s["scale"]
    there = torch.arange(rows.shape[1], device=DEV) < lens[:, None]
    scores = torch.where(there[:, None], scores, -math.inf)
    top = scores.amax(2, keepdim=True)
    p = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(2, keepdim=True)
    o = torch.matmul(p, rows[..., :D_C]) / torch.where(total == 0, 1.0, total)
    return torch.einsum("bhc,chv->bhv", o, w[..., D_NOPE:]).to(BF16)


_PLAIN = {"write": _plain_write, "read": _plain_read, "decode": _plain_decode}


# ---- the definitions in float64 ----------------------------------------------------------------------------
def _value_of(code):
    """The numbers that e4m3 codes stand for, from their bits: sign, four bits of exponent (bias 7), three of mantissa."""
    code = code.to(torch.int64)
    e, m = (code >> 3) & 15, (code & 7).double()
    x = torch.where(e > 0, (8 + m) * torch.exp2((e - 10).double()), m * 2.0 ** -9)
    return torch.where(code >= 128, -x, x)


def _nearest(x):
    """x to the nearest number of four binary digits, of multiples of 2^-9 near zero, ties to even."""
    digit = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / digit) * digit


def _held(cache, slots):
    page = cache.shape[1] // TOKEN
    at = slots.long()
    bytes_ = cache.view(-1)
    first = (at // page) * (page * TOKEN)
    code = bytes_[(first + (at % page) * CODES)[:, None] + torch.arange(CODES, device=DEV)]
    scale = bytes_[(first + page * CODES + (at % page) * 4)[:, None] + torch.arange(4, device=DEV)].view(torch.float32).double()
    x = _value_of(code) * scale
    return torch.cat([x[:, :D_C], x[:, D_C:ROW] + x[:, ROW:]], 1)


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "decode":
        return _exact_decode(s)
    rows = torch.zeros(case["tokens"], ROW, dtype=torch.float64, device=DEV)
    n = case["tokens"] - case["pad"]
    if s["op"] == "read":
        rows[:n] = _held(s["cache"], s["slots"][:n])
    else:
        x = s["kv_a"][:n].double()
        var, mean = torch.var_mean(x[:, :D_C], 1, correction=0)
        y = (x[:, :D_C] - mean[:, None]) * (var + s["eps"]).pow(-0.5)[:, None] * s["gamma"].double()
        y = y if s["beta"] is None else y + s["beta"].double()
        k = x[:, D_C:]                              # 32 complex numbers, each times exp(i * position * frequency)
        z = torch.view_as_complex(k.unflatten(1, (-1, 2)).contiguous()) if s["interleaved"] else torch.complex(
            k[:, :D_ROPE // 2].contiguous(), k[:, D_ROPE // 2:].contiguous())
        phase = torch.outer(s["positions"][:n].double(), s["freqs"])
        z = z * torch.polar(torch.ones_like(phase), phase)
        k = torch.view_as_real(z).flatten(1) if s["interleaved"] else torch.cat([z.real, z.imag], 1)
        most = torch.maximum(y.abs().amax(1), k.abs().amax(1))
        scale = torch.exp2(torch.ceil(torch.log2(most / 448)).clamp(min=-32))[:, None]
        first = _nearest(k / scale)
        rows[:n] = torch.cat([_nearest(y / scale), first + _nearest(k / scale - first)], 1) * scale
    return {"latent": rows[:, :D_C], "k_pe": rows[:, D_C:]}


def _exact_decode(s):
    """The explicit form, one request at a time: keys and values of every head from the latent, then softmax."""
    n, h = s["q"].shape[:2]
    page = s["cache"].shape[1] // TOKEN
    w = s["w_kv_b"].double().view(D_C, h, D_NOPE + D_V).permute(1, 0, 2)
    out = torch.zeros(n, h, D_V, dtype=torch.float64, device=DEV)
    for b in range(n):
        t = int(s["seq_lens"][b])
        if t == 0:
            continue
        at = torch.arange(t, device=DEV)
        rows = _held(s["cache"], s["block_table"][b].long()[at // page] * page + at % page)
        most = max(1, (1 << 30) // (t * (D_NOPE + D_V) * 8))       # heads at a time: about 1 GB of keys and values
        for i in range(0, h, most):
            kv = rows[:, :D_C] @ w[i:i + most]                     # [heads, t, 256]
            q = s["q"][b, i:i + most].double()
            z = (torch.einsum("hn,htn->ht", q[:, :D_NOPE], kv[..., :D_NOPE]) + q[:, D_NOPE:] @ rows[:, D_C:].T) * s["scale"]
            out[b, i:i + most] = torch.einsum("ht,htv->hv", z.softmax(1), kv[..., D_NOPE:])
    return out


# ---- what a pass cannot do without -------------------------------------------------------------------------
def work(case):
    m = case.get("tokens", 0)
    if case["op"] == "read":
        return {"bytes": m * (TOKEN + ROW * 2 + 4), "flops": m * CODES}
    if case["op"] == "write":                       # the rows in; codes and what comes back of them out
        return {"bytes": m * (ROW * 4 + TOKEN + 8) + 4 * D_C, "flops": m * (12 * D_C + 6 * D_ROPE)}
    n, h = case["requests"], case["heads"]
    tokens = case["longest"] if n == 1 else n * (case["shortest"] + case["longest"]) // 2
    return {"bytes": tokens * (TOKEN + 4 / case["page"]) + n * h * (D_NOPE + D_ROPE + D_V) * 2 + D_C * h * (D_NOPE + D_V) * 2,
            "flops": tokens * h * 2 * (ROW + D_C) + n * h * 2 * D_C * (D_NOPE + D_V)}
