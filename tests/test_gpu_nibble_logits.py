"""The 4-bit cache's attention where one key, or all of them alike, decide the output: logits of any size, and answers that do not hang on how they are rounded."""
import numpy as np
import pytest
import torch

from oracle import nibble_cache as N
from paper_2511_05534_b200 import binding as F

import nibble_util as T

pytestmark = pytest.mark.gpu
ONE = 120                                      # the byte of the scale 1
# units, KV heads, longest, width of the table in rows: a row, a tile, warps of a block, blocks (cut heads), two heads a block, heads in line
SHAPES = [(2, 2, 1, 16), (2, 2, 40, 64), (2, 2, 700, 704), (2, 2, 9000, 9216), (38, 8, 300, 320), (75, 8, 130, 160)]


def _pool(rng, U, H, D, rows, codes, wide, page=32):
    """Keys [units, H, rows, D] of these codes and scales of 1, random values."""
    table, n_pages = T.random_table(rng, rows, page, wide=wide // page if wide >= page else None)
    pool = T.random_pool(rng, n_pages, H, page, D, rows, table)
    for u, n in enumerate(rows):
        at = np.arange(n)
        where = (table[u, at // page], slice(None), at % page)
        pool[0][where] = N.pack(codes[u][:, :n]).swapaxes(0, 1)
        pool[2][where] = ONE
    return table, pool


def _rows(rng, U, most):
    rows = rng.integers(max(1, most // 2), most + 1, U).astype(np.int32)
    rows[0] = most
    return rows


def _one_channel(U, Hq, D, channel, value):
    q = np.zeros((U, Hq, D))
    q[:, :, channel] = value
    return q


def _attend(rng, U, H, G, D, rows, codes, wide, q, dtype):
    table, pool = _pool(rng, U, H, D, rows, codes, wide)
    p = T.params(U, H * G, H, D, 32, pool[0].shape[0], table.shape[1], dtype=dtype, softmax_scale=1.0)
    got, status = T.attend(p, q, pool, table, rows)
    assert status == 0
    return got, [N.load(pool[1], pool[3], table[u], rows[u]) for u in range(U)]


def _relative(dtype, n):
    """Equal weights, or one: a weight in fp16 2^-11 of itself (fp32: in two, 2^-21), exponentials 2^-21 each, sums of n products and of n weights 2^-23 a
    term, the quotient 2^-21; a bf16 output half a step, 2^-8, of what it is by then."""
    inner = (2.0 ** -11 if dtype == F.BF16 else 2.0 ** -21) + 2 * 2.0 ** -21 + 2 * (n + 8) * 2.0 ** -23 + 2.0 ** -21
    return inner if dtype == F.F32 else inner + 2.0 ** -8 * (1 + inner)


@pytest.mark.parametrize("dtype", [F.BF16, F.F32])
@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("U,H,most,wide", SHAPES)
@pytest.mark.parametrize("exponent", [20, 28, 30, 34, 120])
def test_one_key_takes_all(dtype, D, U, H, most, wide, exponent):
    """A key whose logit is ahead by a twelfth of its size or more: the output is its value.  Positive logits in the even query heads, negative ones in the odd."""
    rng = np.random.default_rng(exponent + most + D)
    G, channel = 4, int(rng.integers(0, D))
    rows = _rows(rng, U, most)
    codes = [np.zeros((H, n, D), np.int64) for n in rows]
    best = [rng.integers(0, n, (H, 2)) for n in rows]                      # of the positive logits, of the negative ones
    for u, n in enumerate(rows):
        codes[u][:, :, channel] = rng.integers(2, 7, (H, n))               # 1 to 4
        for h in range(H):
            if u % 3 == 0:
                best[u][h] = [0, n - 1] if h % 2 else [n - 1, 0]
            if n > 1 and best[u][h, 0] == best[u][h, 1]:
                best[u][h, 1] = (best[u][h, 0] + 1) % n
            codes[u][h, best[u][h, 1], channel] = 1                        # 0.5
            codes[u][h, best[u][h, 0], channel] = 7                        # 6
    q = _one_channel(U, H * G, D, channel, 2.0 ** exponent)
    q[:, 1::2] *= -1
    q[:, 2:] /= 4                                                          # (heads of a group differ)
    got, v = _attend(rng, U, H, G, D, rows, codes, wide, q, dtype)
    for u in range(U):
        for g in range(H * G):
            want = v[u][g // G, best[u][g // G, g % 2]]
            assert (np.abs(got[u, g] - want) <= _relative(dtype, 1) * np.abs(want)).all(), (u, g)


@pytest.mark.parametrize("dtype", [F.BF16, F.F32])
@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("U,H,most,wide", SHAPES)
@pytest.mark.parametrize("exponent", [-130, 0, 26, 30, 120])
def test_equal_keys_give_the_mean(dtype, D, U, H, most, wide, exponent):
    rng = np.random.default_rng(exponent + 200 + most + D)
    G, channel = 3, int(rng.integers(0, D))
    rows = _rows(rng, U, most)
    codes = [np.zeros((H, n, D), np.int64) for n in rows]
    for c in codes:
        c[:, :, channel] = 5                                               # 3
    q = _one_channel(U, H * G, D, channel, 1.25 * 2.0 ** exponent)
    q[:, 1::2] *= -1
    got, v = _attend(rng, U, H, G, D, rows, codes, wide, q, dtype)
    for u in range(U):
        want, size = v[u].mean(1), np.abs(v[u]).mean(1)
        for g in range(H * G):
            assert (np.abs(got[u, g] - want[g // G]) <= _relative(dtype, rows[u]) * size[g // G]).all(), (u, g)


@pytest.mark.parametrize("dtype", [F.BF16, F.F32])
@pytest.mark.parametrize("exponent", [26, 30, 34])
def test_the_largest_comes_late_or_early(dtype, exponent):
    """Logits that rise or fall from row to row, so that the maximum is set again in every tile, or never again."""
    rng = np.random.default_rng(exponent)
    n, D = 1500, 64
    rows = np.array([n, n], np.int32)
    codes = [np.zeros((1, n, D), np.int64) for _ in rows]
    for u in range(2):
        digits = (np.arange(n) if u == 0 else np.arange(n)[::-1])[:, None] // 4 ** np.arange(6) % 4
        codes[u][0, :, :6] = np.array([0, 2, 4, 5])[digits]               # 0, 1, 2 and 3
    q = np.zeros((2, 1, D))
    q[:, 0, :6] = 2.0 ** exponent * 4.0 ** np.arange(6) / 4 ** 5
    got, v = _attend(rng, 2, 1, 1, D, rows, codes, 1504, q, dtype)
    for u, best in ((0, n - 1), (1, 0)):
        want = v[u][0, best]
        assert (np.abs(got[u, 0] - want) <= _relative(dtype, 1) * np.abs(want)).all(), u
