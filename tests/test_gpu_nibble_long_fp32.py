"""The 4-bit cache's attention with fp32 rows over caches that a warp takes many tiles of: errors do not grow with the number of tiles."""
import math

import numpy as np
import pytest

from oracle import nibble_cache as N
from paper_2511_05534_b200 import binding as F

import nibble_util as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("U,n", [(200, 16000), (400, 9000)])
def test_errors_do_not_grow_with_the_length(D, U, n):
    """Units that share one sequence's pages, values above zero.  Root mean square of the error, relative to the output:
    16 rows' products are two matrix instructions, each within 2^-23 of their sum; n / 16 such sums are added one after the other, to the nearest, each within 2^-24 of
    what the sum has grown to by then, independent of one another: sqrt(n / 16) / 3 of that for the last one's size; the sum of weights is no worse, hence twice both; weights, independent
    of one another too, joining and the quotient 2^-21."""
    rng = np.random.default_rng(D + n)
    H, G, page = 4, 1, 64
    one, n_pages = T.random_table(rng, [n], page)
    pool = T.random_pool(rng, n_pages, H, page, D, [n], one, scales=(88, 104))
    pool[1] &= 0x77
    q = rng.standard_normal((U, H * G, D)).astype(np.float32)
    p = T.params(U, H * G, H, D, page, n_pages, one.shape[1], dtype=F.F32)
    got, status = T.attend(p, q, pool, np.repeat(one, U, 0), np.full(U, n))
    assert status == 0
    k, v = N.load(pool[0], pool[2], one[0], n), N.load(pool[1], pool[3], one[0], n)
    w = np.exp(q.astype(np.float64).transpose(1, 0, 2) @ k.transpose(0, 2, 1) / math.sqrt(D))      # [H, U, n]: logits of one or two
    want = (w @ v / w.sum(2, keepdims=True)).transpose(1, 0, 2)
    assert (want > 0).all()
    error = math.sqrt(np.mean((got / want - 1) ** 2))
    assert error <= 2 * (2 * 2.0 ** -23 + math.sqrt(n / 16) / 3 * 2.0 ** -24) + 2.0 ** -21, error
