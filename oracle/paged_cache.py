"""The paged 8-bit cache in numpy and 64 bits, one unit, page and head at a time, from the definitions in include/flowmm.h."""
import math

import numpy as np

LOWEST = -96          # exponent of the smallest scale that a store writes

E4M3 = np.array([(-1.0) ** (c >> 7) * (np.nan if c & 127 == 127 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3 & 15) - 7) if c >> 3 & 15 else (c & 7) * 2.0 ** -9)
                 for c in range(256)])


def to_e4m3(x: np.ndarray) -> np.ndarray:
    """The codes' values nearest to x, ties to the even code; x at most 448 in size; what is not finite becomes NaN."""
    grid = E4M3[:127]                                                    # ascending, an even code at every even place
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    assert (a <= 448).all()
    hi = np.searchsorted(grid, a)                                        # grid[hi] >= a
    lo = np.maximum(hi - 1, 0)
    up, down = grid[hi] - a, a - grid[lo]
    take = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return np.where(np.isfinite(x), np.copysign(grid[take], x), np.nan)


def scale_for(size: float) -> float:
    e = LOWEST
    if size > 0:
        e = max(LOWEST, math.frexp(size)[1] - 10)
        while 448 * 2.0 ** e < size:
            e += 1
    return 2.0 ** e


def pages(n: int, page: int) -> int:
    return -(-n // page)


def plan(grow, rows, ring, state, table, page, n_rows, with_slots=True):
    """(rows_out, state_out, table, ring, slots, units refused); the arguments are left alone."""
    ring, table = ring.copy(), table.copy()
    head, count = (int(x) for x in state)
    n, wide = len(ring), table.shape[1]
    out, slots, refused = rows.copy(), np.full((len(rows), n_rows), -1, np.int32), []
    asked = taken = 0
    back = []
    for u in range(len(rows)):
        r, g = int(rows[u]), int(grow[u])
        new = max(0, r + g)
        if not 0 <= r <= wide * page or new > wide * page or (with_slots and g > n_rows):
            refused.append(u)
            continue
        held, want = pages(r, page), pages(new, page)
        if want > held:
            asked += want - held
            if asked > count:
                refused.append(u)
                continue
            for j in range(held, want):
                table[u, j] = ring[(head + taken) % n]
                taken += 1
        back += [int(x) for x in table[u, want:held]]
        for t in range(max(0, g)) if with_slots else ():
            slots[u, t] = table[u, (r + t) // page] * page + (r + t) % page
        out[u] = new
    for i, x in enumerate(back):
        ring[(head + count + i) % n] = x
    return out, np.array([(head + taken) % n, count - taken + len(back)], np.int32), table, ring, slots, refused


def store(x, slots, values, scale):
    """Values (codes as numbers) and scales of a pool after rows x [U, H, T, D] went to slots; values [n_pages, H, page, D]."""
    values, scale = values.copy(), scale.astype(np.float64)
    page = values.shape[2]
    U, H, T, _ = x.shape
    for u in range(U):
        t = 0
        while t < T and slots[u, t] >= 0:
            p, at = divmod(int(slots[u, t]), page)
            n = 1
            while t + n < T and at + n < page and slots[u, t + n] >= 0:
                n += 1
            for h in range(H):
                rows = x[u, h, t:t + n].astype(np.float64)
                s = scale_for(np.max(np.abs(rows[np.isfinite(rows)]), initial=0.0))
                if at:
                    s = max(s, scale[p, h])
                    values[p, h, :at] = to_e4m3(values[p, h, :at] * (scale[p, h] / s))
                values[p, h, at:at + n] = to_e4m3(rows / s)
                scale[p, h] = s
            t += n
    return values, scale


def load(values, scale, table, n):
    """[H, n, D]: the rows of a unit with this row of the block table."""
    page = values.shape[2]
    ids = table[:pages(n, page)]
    x = values[ids] * scale[ids][:, :, None, None]
    return np.moveaxis(x, 1, 0).reshape(x.shape[1], -1, x.shape[3])[:, :n]


def attention(q, k_values, v_values, k_scale, v_scale, table, rows, softmax_scale=0.0, least=2.0 ** -14):
    """(out, size, logits): q [U, Hq, D]; size[u, hq, d] = sum_j max(w_j, least * max_i w_i) |code_jd| with w_j = p_j sv_j, a key's weight and V's
    scale, logits[u, hq] = the largest scale * sum_d |q_d k_jd|: by both of these the rounding errors go of an implementation that holds weights w with
    a relative error down to `least` of the largest, and with the absolute error that belongs to that below."""
    U, Hq, D = q.shape
    H = k_values.shape[1]
    c = softmax_scale or 1 / math.sqrt(D)
    out, size, logits = np.zeros((U, Hq, D)), np.zeros((U, Hq, D)), np.zeros((U, Hq))
    for u in range(U):
        if rows[u] == 0:
            continue
        k, v = load(k_values, k_scale, table[u], rows[u]), load(v_values, v_scale, table[u], rows[u])
        for g in range(Hq):
            h = g // (Hq // H)
            z = c * (k[h] @ q[u, g])
            w = np.exp(z - np.max(z))
            sv = np.repeat(v_scale[table[u, :pages(int(rows[u]), v_values.shape[2])], h], v_values.shape[2])[:rows[u]].astype(np.float64)
            weight = np.maximum(w * sv, least * np.max(w * sv)) / sv
            out[u, g], size[u, g] = w @ v[h] / w.sum(), weight @ np.abs(v[h]) / w.sum()
            logits[u, g] = c * np.max(np.abs(k[h]) @ np.abs(q[u, g]))
    return out, size, logits
