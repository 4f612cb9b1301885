"""Paged caches for the tests: pools with bytes of any kind in them, and the calls of the binding."""
import numpy as np
import torch

from oracle import paged_cache as P
from paper_2511_05534_b200 import binding as F


def params(U, Hq, Hkv, D, page, n_pages, wide, n_rows=1, dtype=F.BF16, **kw):
    return F.CacheParams(U, Hq, Hkv, D, page, n_pages, wide, n_rows, dtype=dtype, **kw)


def random_table(rng, rows, page, spare=3, wide=None):
    """(block table, n_pages): pages in random order, numbers out of range behind a unit's last page."""
    count = [P.pages(int(n), page) for n in rows]
    n_pages = sum(count) + spare
    order = rng.permutation(n_pages)
    table = np.full((len(rows), wide or max(1, max(count))), 1 << 30, np.int32)
    at = 0
    for u, c in enumerate(count):
        table[u, :c] = order[at:at + c]
        at += c
    return table, n_pages


def random_pool(rng, n_pages, H, page, D, rows, table, exponents=(-3, 3)):
    """(codes uint8, scales float32): no NaN in rows that units hold, any byte elsewhere, NaN among them."""
    codes = rng.integers(0, 256, (n_pages, H, page, D)).astype(np.uint8)
    for u, n in enumerate(rows):
        for j in range(P.pages(int(n), page)):
            there = codes[table[u, j], :, :min(page, int(n) - j * page)]
            there[there & 127 == 127] -= 1
    return codes, (2.0 ** rng.integers(exponents[0], exponents[1] + 1, (n_pages, H))).astype(np.float32)


def dev(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t if dtype is None else t.to(F.torch_dtype(dtype))


def attend(p, q, codes_k, codes_v, ks, vs, table, rows, ws=None):
    """flowmm_cache_attention on numpy arrays; (out float64, device status)."""
    ws = F.alloc_cache_workspace(p) if ws is None else ws
    out = torch.full((p.n_units, p.n_q_heads, p.head_dim), float("nan"), device="cuda")
    F.flowmm_cache_attention(p, dev(q, p.dtype), dev(codes_k), dev(codes_v), dev(ks), dev(vs), dev(table), dev(np.asarray(rows, np.int32)), out, ws)
    status = F.flowmm_last_device_status(ws)
    return out.cpu().numpy().astype(np.float64), status


def attention_bound(size, logits, n, D):
    """How far an fp32 implementation may be from the 64-bit one, per output.  Logits: D products and their sum in fp32, the scale
    and the scale of the page, each within 2^-23 (a tensor core that truncates), plus a bf16 query as two e4m3 numbers, exact but for
    elements 2^13 times smaller than the largest, 2^-18 covers it; weights: exp2 within 2^-21 and a split into four e4m3 numbers, 2^-16;
    sums of n weights and products, each within 2^-23.  Numerator and denominator both carry the weights' error.  The split: a weight x, 256 for the
    largest, is rounded to e4m3 four times, its rest times 16 each time; a rest is at most 2^-4 of what was rounded, so four leave 2^-16 of x,
    unless a rest falls below e4m3's least normal number: then half a step of the last piece, 2^-10 * 16^-3 = 2^-22, is left, 2^-30 of the
    largest weight: 2^-16 of one 2^-14 times the largest, which `size` counts weights as at least (oracle.paged_cache.attention)."""
    rel = (D + 16) * 2.0 ** -23 * logits + 2.0 ** -18 * logits + 2.0 ** -16 + 2.0 ** -20 + (n + 16) * 2.0 ** -23
    return 2 * rel[:, None] * size + 1e-30
