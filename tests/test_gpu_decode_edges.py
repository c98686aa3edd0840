"""One-token attention over the paged latent cache at the edges of softmax: requests that nothing is left of."""
import math

import pytest
import torch

from test_gpu_decode import BF16, case, check, laga, run  # noqa: F401  (laga: the fixture)

pytestmark = pytest.mark.gpu
KEY = 3                                                # the rope channel through which the tests set scores


def keyed(lens, h, page, of, value, seed=31):
    """A case in which every token of the requests `of` has `value` in channel KEY of its key, and every query a positive number there."""
    q, w, cache, table, n = case(lens, h, page, seed=seed, fill=0.0)
    q[..., 128 + KEY] = 0.5
    for b in of:
        cache[table[b, : -(-lens[b] // page)].long(), :, 512 + KEY] = value
    return q, w, cache, table, n


# one piece; many pieces over several CTAs; pieces of both kinds next to one another; two requests in a row; 64 heads a CTA
@pytest.mark.parametrize("lens,h,of", [([100, 70], 16, [0]), ([20000, 300, 5], 4, [0]), ([300, 20000, 5], 16, [1]), ([64, 1, 1, 9000], 24, [1, 2]),
                                       ([100, 70, 129], 64, [2]), ([9000, 40], 128, [0]), ([33] * 40, 16, list(range(0, 40, 3)))])
def test_requests_whose_every_key_is_minus_infinity(laga, lens, h, of):  # noqa: F811
    """Nothing weighs anything: zeros and an LSE of minus infinity, as for a request without tokens; its neighbours are not touched."""
    q, w, cache, table, n = keyed(lens, h, 16, of, -math.inf)
    out, lse = run(laga, (q, w, cache, table, n))
    assert bool((out[of] == 0).all()) and bool((lse[of] == -math.inf).all())
    live = [b for b in range(len(lens)) if b not in of]
    check((q[live], w, cache, table[live], n[live]), out[live], lse[live])


def test_nan_among_keys_of_minus_infinity_is_not_hidden(laga):  # noqa: F811
    q, w, cache, table, n = keyed([100, 70], 16, 16, [0], -math.inf)
    cache[table[0, 2].long(), 4, 512 + KEY + 1] = math.nan
    out, lse = run(laga, (q, w, cache, table, n))
    assert bool(out[0].isnan().all()) and bool(lse[0].isnan().all()) and bool(out[1].isfinite().all())


LOWEST = float(torch.finfo(BF16).min)


def plain_scores(q, of, heads):
    """Queries that see channel KEY alone, so that scores are exactly query * key in any arithmetic."""
    q[of] = 0
    q[of, :, 128 + KEY] = torch.tensor([0.5, 0.25, 1.0, 0.0078125])[torch.arange(heads) % 4].to(BF16)


def uniform(w, rows):
    """(mean of the rows' values, bound): equal weights leave the fp32 sum of t latents, the joined latent's two bf16 parts (2^-16 relative,
    with the product's fp32 sums under it) and the result's rounding."""
    h = w.shape[1] // 256
    w_uv = w.double().view(512, h, 256)[..., 128:]
    want = torch.einsum("c,chv->hv", rows.double().mean(0), w_uv)
    d = (2.0 ** -15 + len(rows) * 2.0 ** -23) * torch.einsum("c,chv->hv", rows.double().abs().mean(0), w_uv.abs())
    return want, d + 2.0 ** -8 * (want.abs() + d)


def latents(cache, table, b, at, page=16):
    at = torch.as_tensor(at)
    return cache[table[b, at // page].long(), at % page, :512]


@pytest.mark.parametrize("value", [LOWEST, -1e30, 3e37])
@pytest.mark.parametrize("lens,h,of", [([100, 70], 16, [0]), ([20000, 300], 4, [0]), ([300, 9000], 40, [0]), ([60, 9000], 128, [0])])
def test_requests_whose_every_score_is_the_same_huge_value(laga, lens, h, of, value):  # noqa: F811
    """Masked tokens given the type's lowest value where nothing else is left (and any other score of that size): as for all equal scores
    the mean of the values.  A rounded maximum taken from unrounded scores would leave 2^100 in the exponent."""
    q, w, cache, table, n = keyed(lens, h, 16, of, value)
    plain_scores(q, of, h)
    out, lse = run(laga, (q, w, cache, table, n))
    for b in of:
        want, bound = uniform(w, latents(cache, table, b, range(lens[b])))
        assert float(((out[b].double().cpu() - want).abs() - bound).max()) <= 0
        score = q[b, :, 128 + KEY].double() * float(torch.tensor(value).to(BF16)) * 192 ** -0.5
        assert float(((lse[b].double().cpu() - score) / score).abs().max()) <= 2.0 ** -20      # (log t is nothing beside it)
    live = [b for b in range(len(lens)) if b not in of]
    check((q[live], w, cache, table[live], n[live]), out[live], lse[live])


@pytest.mark.parametrize("h", [16, 64])
def test_tokens_of_the_lowest_value_beside_others(laga, h):  # noqa: F811
    """Such tokens weigh nothing beside ordinary ones, also where they are all that a CTA has of the request; and beside one token of a huge
    score nothing else weighs anything."""
    lens = [20000, 100]
    q, w, cache, table, n = case(lens, h, 16, seed=33, fill=0.0)
    q[..., 128 + KEY] = q[..., 128 + KEY].abs().clamp_min(0.125)
    rows = cache[table[0].long()].reshape(-1, 576)[:20000]
    at = torch.arange(20000)
    out_of = (at < 2048) | ((at // 64) % 2 == 0) | (at % 64 == 11) | (at >= 19000)
    rows[out_of, 512 + KEY] = LOWEST
    cache[table[0].long()] = rows.view(-1, 16, 576)
    kept = cache.clone()
    left = rows[~out_of]
    count = -(-len(left) // 16)
    kept[table[0, :count].long()] = torch.nn.functional.pad(left, (0, 0, 0, 16 * count - len(left))).view(-1, 16, 576)
    out, lse = run(laga, (q, w, cache, table, n))
    check((q, w, kept, table, torch.tensor([len(left), 100], dtype=torch.int32)), out, lse)
    plain_scores(q, [0], h)
    places = [77, 9000, 9001, 19999]                   # four tokens of one huge score
    cache[table[0].long(), :, 512 + KEY] = 1.0
    for t in places:
        cache[int(table[0, t // 16]), t % 16, 512 + KEY] = 1e37
    out, lse = run(laga, (q, w, cache, table, n))
    want, bound = uniform(w, latents(cache, table, 0, places))
    assert float(((out[0].double().cpu() - want).abs() - bound).max()) <= 0
