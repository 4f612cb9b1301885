"""The paged 4-bit cache in numpy and 64 bits, from the definitions in include/flowmm.h.  Pools are held as the values of their codes
[n_pages, H, page, D] and of their scales [n_pages, H, page, D / 16]."""
import math

import numpy as np

E2M1 = np.array([(-1.0) ** (c >> 3) * ((1 + (c & 1) / 2) * 2.0 ** ((c >> 1 & 3) - 1) if c >> 1 & 3 else (c & 1) / 2) for c in range(16)])
SCALE = np.array([(math.nan if b & 7 else math.inf) if b >> 3 == 31 else (1 + (b & 7) / 8) * 2.0 ** ((b >> 3) - 15) if b >> 3 else (b & 7) * 2.0 ** -17
                  for b in range(256)])
LEAST, MOST, NAN = 8, 226, 255        # bytes of the scales that a store writes


def nearest(x, grid):
    """Places in the ascending grid of what is nearest to x, ties to the even place."""
    hi = np.minimum(np.searchsorted(grid, x), len(grid) - 1)
    lo = np.maximum(hi - 1, 0)
    up, down = np.abs(grid[hi] - x), np.abs(x - grid[lo])
    return np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)


def quantise(x):
    """(codes, bytes of scales) of rows x [..., D]; codes 0 .. 15, not packed."""
    g = x.astype(np.float64).reshape(*x.shape[:-1], -1, 16)
    fine = np.isfinite(g).all(-1)
    g = np.where(fine[..., None], g, 0.0)
    size = np.abs(g).max(-1) / 6
    byte = LEAST + nearest(size, SCALE[LEAST:MOST + 1])
    code = nearest(np.minimum(np.abs(g) / SCALE[byte][..., None], 6.0), E2M1[:8])
    code = np.where(fine[..., None], code + 8 * np.signbit(g), 0)
    return code.reshape(x.shape), np.where(fine, byte, NAN)


def pack(codes):
    return (codes[..., ::2] | codes[..., 1::2] << 4).astype(np.uint8)


def unpack(pages):
    out = np.empty((*pages.shape[:-1], 2 * pages.shape[-1]), np.int64)
    out[..., ::2], out[..., 1::2] = pages & 15, pages >> 4
    return out


def pages(n, page):
    return -(-n // page)


def store(x, slots, page_bytes, scale_bytes):
    """The bytes of a pool and its scales after rows x [U, H, T, D] went to slots [U, T]."""
    page_bytes, scale_bytes = page_bytes.copy(), scale_bytes.copy()
    page = page_bytes.shape[2]
    codes, scale = quantise(x)
    codes = pack(codes)
    for u, t in zip(*np.nonzero(slots >= 0)):
        p, at = divmod(int(slots[u, t]), page)
        page_bytes[p, :, at], scale_bytes[p, :, at] = codes[u, :, t], scale[u, :, t]
    return page_bytes, scale_bytes


def load(page_bytes, scale_bytes, table, n):
    """[H, n, D]: the rows of a unit with this row of the block table."""
    ids = table[:pages(n, page_bytes.shape[2])]
    x = E2M1[unpack(page_bytes[ids])] * np.repeat(SCALE[scale_bytes[ids]], 16, -1)
    return np.moveaxis(x, 1, 0).reshape(x.shape[1], -1, x.shape[3])[:, :n]


def attention(q, pool, table, rows, softmax_scale=0.0, least=2.0 ** -18):
    """(out, size, logits): q [U, Hq, D], pool: pages and scales of K, then V, as bytes, in the order k, v, k scale, v scale.
    size[u, hq, d] = sum_j max(w_j, least * max_i w_i) |v_jd| / sum_j w_j, logits[u, hq] = the largest scale * sum_d |q_d k_jd|: by both of these the
    rounding errors go of an implementation that holds weights w with a relative error down to `least` of the largest, and with the absolute error that
    belongs to that below."""
    U, Hq, D = q.shape
    kp, vp, ks, vs = pool
    H = kp.shape[1]
    c = softmax_scale or 1 / math.sqrt(D)
    out, size, logits = np.zeros((U, Hq, D)), np.zeros((U, Hq, D)), np.zeros((U, Hq))
    for u in range(U):
        if rows[u] == 0:
            continue
        k, v = load(kp, ks, table[u], rows[u]), load(vp, vs, table[u], rows[u])
        for g in range(Hq):
            h = g // (Hq // H)
            z = c * (k[h] @ q[u, g])
            w = np.exp(z - np.max(z))
            out[u, g], size[u, g] = w @ v[h] / w.sum(), np.maximum(w, least) @ np.abs(v[h]) / w.sum()
            logits[u, g] = c * np.max(np.abs(k[h]) @ np.abs(q[u, g]))
    return out, size, logits
