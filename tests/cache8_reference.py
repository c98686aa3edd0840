"""Plain float64 references (CPU) of the latent cache in 8 bits: its format, and the attention over it with the error bound of the parts
that queries and probabilities are carried in.  E is half a step of e4m3, the most one rounding to it can be off, relative to the value."""
import math

import torch
import torch.nn.functional as F

import serving_reference as ref

E = float(torch.finfo(torch.float8_e4m3fn).eps) / 2      # 2^-4
LEAST = 2.0 ** -10                                       # half of the smallest e4m3 number: the most that a small one can be off
TOKEN, CODES = 644, 640


def scale_of(amax):
    """The smallest power of two, 2^-32 at least, that brings amax (float64) within 448."""
    m, e = torch.frexp(amax)
    return torch.ldexp(torch.ones_like(amax), torch.where(amax == 0, -32, e - 9 + (m > 0.875)).clamp(min=-32))


def nearest(x):
    """x (float64) to e4m3, ties to even; within 448."""
    digit = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / digit) * digit


def byte_of(value):
    """The codes (uint8) of numbers that e4m3 holds."""
    return value.to(torch.float32).to(torch.float8_e4m3fn).view(torch.uint8)


def value_of(code):
    return code.view(torch.float8_e4m3fn).to(torch.float64)


def encode(rows):
    """rows float64 [n, 576] -> (codes uint8 [n, 640], scales fp32 [n])."""
    s = scale_of(rows.abs().amax(1))
    x = rows / s[:, None]
    first = nearest(x)
    rest = nearest(x[:, 512:] - first[:, 512:])
    return torch.cat([byte_of(first), byte_of(rest)], 1), s.float()


def decode_rows(codes, scales):
    """(codes [..., 640], scales [...]) -> rows float64 [..., 576]."""
    x = value_of(codes)
    return torch.cat([x[..., :512], x[..., 512:576] + x[..., 576:]], -1) * scales.double()[..., None]


def planes(pages):
    """(codes uint8 [n, page, 640], scales fp32 [n, page]) of pages uint8 [n, page * 644], as views."""
    page = pages.shape[1] // TOKEN
    return pages[:, : page * CODES].unflatten(1, (page, CODES)), pages[:, page * CODES:].view(torch.float32)


def empty_pages(n, page, fill=0xff):
    """fill 0xff: every code a NaN, every scale too."""
    return torch.full((n, page * TOKEN), fill, dtype=torch.uint8)


def decode(q, w, pages, table, lens, scale):
    """As serving_reference.decode over the rows that the pages stand for.  Returns (out, lse, bound_out, bound_lse).  The bound takes every
    rounding at its worst for every element at once: q W_uk and the rotated queries in two e4m3 parts (E^2 of the value, taken of its fp16 rounding,
    and LEAST of the power of two r that brings the 576 channels within 448); the probabilities in two parts (E^2; over 32 heads, where the
    first is e5m2, 2 E^2), with what both parts leave of the smallest: LEAST / 32 in units in which a tile's largest is 2^-3 at least, so 2^-12 of
    that (over 32 heads LEAST, and 2^0: 2^-10).  What is held in those parts, and what a tile's largest is one of, is the probability times its
    token's scale, p_t s_t, and what multiplies it the token's codes, c_t / s_t.  The joined output and the result as there."""
    B, h, _ = q.shape
    codes, scales = planes(pages)
    w3 = w.double().view(512, h, 256)
    many = h > 32
    two = E * E * (1 + 2.0 ** -4)
    p_two, p_floor = (2 * two, 2.0 ** -10) if many else (two, 2.0 ** -12)
    out, lse = torch.zeros(B, h, 128, dtype=torch.float64), torch.full((B, h), -math.inf, dtype=torch.float64)
    b_out, b_lse = torch.zeros(B, h, 128, dtype=torch.float64), torch.zeros(B, h, dtype=torch.float64)
    page = codes.shape[1]
    for b in range(B):
        t = int(lens[b])
        if t == 0:
            continue
        at = table[b, : -(-t // page)].long()
        rows = decode_rows(codes[at], scales[at]).reshape(-1, 576)[:t]
        s_t = scales[at].reshape(-1)[:t].double()
        s_t = torch.where(s_t == 0, 1.0, s_t)
        c, kpe = rows[:, :512], rows[:, 512:]
        v_all = torch.einsum("tc,chv->htv", c, w3[..., 128:])
        q_abs = torch.einsum("chn,hn->hc", w3[..., :128], q[b, :, :128].double())
        q_all = torch.cat([q_abs, q[b, :, 128:].double()], 1)
        s = q_all @ rows.T * scale
        p = s.softmax(1)
        out[b] = torch.einsum("ht,htv->hv", p, v_all)
        lse[b] = s.logsumexp(1)
        r = scale_of(q_all.abs().amax(1))
        size = rows.abs()                                # (the key's two codes: their sizes add up to 1 + E of the key's at most)
        size = torch.cat([size[:, :512], size[:, 512:] * (1 + 2 * E)], 1)
        mag = q_all.abs() @ size.T
        e = scale * (two * mag + LEAST * r[:, None] * size.sum(1) + 2 * 640 * 2.0 ** -23 * mag).amax(1) + 2.0 ** -20 * (s.abs().amax(1) + 1)
        near = F.max_pool1d((p * s_t)[:, None], 255, 1, 127)[:, 0]       # the largest of any tile that a key can be in
        off = p * ((torch.exp(2 * e) * (1 + p_two) - 1 + t * 2.0 ** -24 + 2.0 ** -12)[:, None])
        d_lat = off @ c.abs() + p_floor * torch.exp(2 * e)[:, None] * (near @ (c.abs() / s_t[:, None]))
        lat = (p @ c).abs()
        d = torch.einsum("hc,chv->hv", 2.0 ** -15 * lat + d_lat, w3[..., 128:].abs())
        b_out[b] = d + ref.U * (out[b].abs() + d)
        b_lse[b] = e + 1e-5 + 2.0 ** -22 * lse[b].abs()
    return out, lse, b_out, b_lse
