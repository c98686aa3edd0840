"""Plain float64 references (CPU) of the rotary, latent-norm, page-table and decode operators, with the error bounds
their kernels are held to.  U is half a step of bf16: the most one rounding to it can be off, relative to the value."""
import math

import torch

U = float(torch.finfo(torch.bfloat16).eps) / 2       # 2^-8


def rotate(x, positions, freqs, mscale, interleaved, inverse=False, begin=None):
    """x [M, ..., d] float64; channels [begin, begin + 2 len(freqs)) rotated.  Returns (y, bound on the error of a kernel
    that rounds y to bf16 and has sine and cosine to 2^-20 absolute: the special-function unit's 2^-21 and the fp32 products)."""
    n = freqs.numel()
    d = x.shape[-1]
    begin = d - 2 * n if begin is None else begin
    ang = positions.double()[:, None] * freqs.double()
    ang = ang.view((x.shape[0],) + (1,) * (x.dim() - 2) + (n,))
    c, s = ang.cos() * mscale, ang.sin() * mscale * (-1 if inverse else 1)
    y, slack = x.clone(), torch.zeros_like(x)
    if interleaved:
        ia = torch.arange(n) * 2 + begin
        ib = ia + 1
    else:
        ia = torch.arange(n) + begin
        ib = ia + n
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    slack[..., ia] = slack[..., ib] = (a.abs() + b.abs()) * mscale * 2.0 ** -20
    bound = slack + U * (y.abs() + slack)
    bound[..., :begin] = 0                             # copied channels are exact
    bound[..., begin + 2 * n:] = 0
    return y, bound


def norm(x, gamma, beta, eps):
    """LayerNorm in float64: (y, mean, rstd, bound): bf16 rounding of y, plus fp32 statistics and arithmetic (sums of D terms:
    at most D 2^-24 of the mean magnitude, which reaches y through xhat)."""
    mean = x.mean(1, keepdim=True)
    rstd = ((x - mean).square().mean(1, keepdim=True) + eps).rsqrt()
    xhat = (x - mean) * rstd
    y = xhat * gamma + (0 if beta is None else beta)
    f32 = x.shape[1] * 2.0 ** -24 * (1 + x.abs().mean(1, keepdim=True) * rstd + xhat.abs()) * gamma.abs() + 2.0 ** -22 * y.abs()
    return y, mean[:, 0], rstd[:, 0], f32 + U * (y.abs() + f32)


def norm_backward(dy, x, gamma, mean, rstd):
    """(dx, dgamma, dbeta, bound of dx, sums of magnitudes of dgamma's and dbeta's terms) at given statistics."""
    xhat = (x - mean[:, None]) * rstd[:, None]
    g = dy * gamma
    dx = rstd[:, None] * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    f32 = (x.shape[1] * 2.0 ** -24) * rstd[:, None] * (g.abs() + g.abs().mean(1, keepdim=True) +
                                                   xhat.abs() * (g * xhat).abs().mean(1, keepdim=True))
    # xhat itself is formed in fp32 from x - mean: an error of 2^-23 (|x| + |mean|) rstd
    rough = 2.0 ** -22 * (x.abs() + mean.abs()[:, None]) * rstd[:, None]
    f32 = f32 + rstd[:, None] * rough * (g * xhat).abs().mean(1, keepdim=True) * 2
    return dx, (dy * xhat).sum(0), dy.sum(0), f32 + U * (dx.abs() + f32), ((dy * xhat).abs() + dy.abs() * rough).sum(0), dy.abs().sum(0)


def plan(seq_lens, new_lens, table, free_pages, n_free, page, max_tokens):
    """The step's tables by the obvious loops; None where it cannot be placed."""
    n, columns = len(seq_lens), len(table[0])
    table = [list(r) for r in table]
    if any(v < 0 for v in list(seq_lens) + list(new_lens)) or any(s + a > columns * page for s, a in zip(seq_lens, new_lens)):
        return None
    slots, positions, cu, top = [], [], [0], n_free
    for b in range(n):
        for i in range(new_lens[b]):
            p = seq_lens[b] + i
            if p % page == 0:
                if top == 0:
                    return None
                top -= 1
                table[b][p // page] = free_pages[top]
            slots.append(table[b][p // page] * page + p % page)
            positions.append(p)
        cu.append(len(slots))
    if len(slots) > max_tokens:
        return None
    pad = max_tokens - len(slots)
    return {"slots": slots + [-1] * pad, "positions": positions + [0] * pad, "cu": cu, "lens": [s + a for s, a in zip(seq_lens, new_lens)],
            "n_free": top, "table": table}


def decode(q, w, cache, table, lens, scale, heads=None):
    """Explicit form in float64, one request at a time.  Returns (out, lse, bound_out, bound_lse): the bounds follow the four
    roundings to bf16 that the path makes -- of W_uk q, of the probabilities, of the latent-space output and of the result --
    each taken at its worst for every element at once."""
    B, h, _ = q.shape
    d_c = w.shape[0]
    w3 = w.double().view(d_c, h, 256)
    out, lse = torch.zeros(B, h, 128, dtype=torch.float64), torch.full((B, h), -math.inf, dtype=torch.float64)
    b_out, b_lse = torch.zeros(B, h, 128, dtype=torch.float64), torch.zeros(B, h, dtype=torch.float64)
    page = cache.shape[1]
    for b in range(B):
        t = int(lens[b])
        if t == 0:
            continue
        rows = cache[table[b, : -(-t // page)].long()].reshape(-1, cache.shape[2])[:t].double()
        c, kpe = rows[:, :d_c], rows[:, d_c:]
        for i in range(h):
            qn, qr = q[b, i, :128].double(), q[b, i, 128:].double()
            k = c @ w3[:, i, :128]
            v = c @ w3[:, i, 128:]
            s = (k @ qn + kpe @ qr) * scale
            p = s.softmax(0)
            out[b, i] = p @ v
            lse[b, i] = s.logsumexp(0)
            q_abs = w3[:, i, :128] @ qn
            # fp32 accumulation over 576 products adds at most 576 * 2^-24 of the magnitudes (tensor cores may truncate: twice)
            mag = c.abs() @ q_abs.abs() + kpe.abs() @ qr.abs()
            e = float((scale * (U * (c.abs() @ q_abs.abs()) + 576 * 2.0 ** -23 * mag)).max()) + 2.0 ** -20 * float(s.abs().max() + 1)
            rho = math.exp(2 * e) * (1 + U) / (1 - U) - 1 + t * 2.0 ** -24 + 2.0 ** -12
            lat = (p @ c).abs()
            d_lat = rho * (p @ c.abs())
            d = (U * lat + d_lat * (1 + U)) @ w3[:, i, 128:].abs()
            b_out[b, i] = d + U * (out[b, i].abs() + d)
            b_lse[b, i] = e + 1e-5 + 2.0 ** -22 * abs(float(lse[b, i]))
    return out, lse, b_out, b_lse
