"""The 4-bit cache's attention with fp32 rows, by the root mean square of its errors: a bound that an implementation without the second halves of its
queries or weights does not keep (worst-case bounds leave it room)."""
import math

import numpy as np
import pytest

from oracle import nibble_cache as N
from paper_2511_05534_b200 import binding as F

import nibble_util as T

CASES = [(1, 64), (2, 64), (33, 128), (218, 128), (700, 64), (3000, 128)]


def _case(n, D, group=4):
    """Scales of 2^-3 to 2^-1, so that logits are about as large as one."""
    rng = np.random.default_rng(n + D)
    rows = np.array([n, max(1, n - 1), n], np.int32)
    table, n_pages = T.random_table(rng, rows, 32)
    pool = T.random_pool(rng, n_pages, 2, 32, D, rows, table, scales=(96, 112))
    q = rng.standard_normal((3, 2 * group, D)).astype(np.float32).astype(np.float64)
    return q, pool, table, rows


def _by_hand(q, pool, table, rows, weight=lambda w: w, query=lambda q: q):
    """(out, rss, logits): with weights, relative to the largest, and queries passed through a rounding; rss[u, hq, d] = the root of
    sum_j w_j^2 v_jd^2 over sum_j w_j, logits = mean over keys of scale * sum_d |q_d k_jd|."""
    U, Hq, D = q.shape
    H = pool[0].shape[1]
    out, rss, logits = np.zeros(q.shape), np.zeros(q.shape), np.zeros((U, Hq))
    for u in range(U):
        k, v = N.load(pool[0], pool[2], table[u], rows[u]), N.load(pool[1], pool[3], table[u], rows[u])
        for g in range(Hq):
            h = g // (Hq // H)
            z = k[h] @ query(q[u, g]) / math.sqrt(D)
            w = np.exp(z - z.max())
            out[u, g], rss[u, g] = weight(w) @ v[h] / w.sum(), np.sqrt(w ** 2 @ v[h] ** 2) / w.sum()
            logits[u, g] = np.mean(np.abs(k[h]) @ np.abs(q[u, g])) / math.sqrt(D)
    return out, rss, logits


def _allowed(rss, logits, n, D):
    """The root mean square of the error.  A logit: D products in steps of 16, twice (the query's two halves), each step's 17 summands cut off within 2^-23 of a
    sum that is no larger than the sum of sizes: the root of as many errors; the query's halves within 2^-21.  A weight: its exponent, up to 32 in size, in fp32 by two roundings,
    2 * 2^-20 at most, the exponential 2^-21, the second half 2^-21.  Sums over keys: the root of n errors of 2^-23.  Weights' errors are independent of one another, so the output's is
    that of a weight times rss; the denominator's is no larger: twice that."""
    of_logit = math.sqrt(2 * D / 16 * 17) * 2.0 ** -23 * logits + 2.0 ** -21 * logits
    weight = of_logit + 2 * 2.0 ** -20 + 2 * 2.0 ** -21 + math.sqrt(n) * 2.0 ** -23
    return 2 * math.sqrt(np.mean((weight[..., None] * rss) ** 2))


@pytest.mark.gpu
@pytest.mark.parametrize("n,D", CASES)
def test_fp32_attention(n, D):
    q, pool, table, rows = _case(n, D)
    p = T.params(3, 8, 2, D, 32, pool[0].shape[0], table.shape[1], dtype=F.F32)
    got, status = T.attend(p, q, pool, table, rows)
    assert status == 0
    want, rss, logits = _by_hand(q, pool, table, rows)
    error = math.sqrt(np.mean((got - want) ** 2))
    assert error <= _allowed(rss, logits, n, D), error / _allowed(rss, logits, n, D)


def _fp16(x):
    scale = 2.0 ** 14 / np.abs(x).max()
    return (x * scale).astype(np.float16).astype(np.float64) / scale


@pytest.mark.parametrize("n,D", [c for c in CASES if c[0] > 1])
@pytest.mark.parametrize("lost", ["weights", "queries"])
def test_the_bound_sees_a_lost_half(n, D, lost):
    """The oracle with weights, or queries, of one fp16 number is outside the bound."""
    q, pool, table, rows = _case(n, D)
    want, rss, logits = _by_hand(q, pool, table, rows)
    off = _by_hand(q, pool, table, rows, **{"weight" if lost == "weights" else "query": _fp16})[0]
    assert math.sqrt(np.mean((off - want) ** 2)) > 2 * _allowed(rss, logits, n, D)
