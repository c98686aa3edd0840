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
