"""The paged cache's attention where a bound for both paths is too wide, or where one path's own limits lie; its calls in the build with index checks."""
import numpy as np
import pytest
import torch

from oracle import paged_cache as P
from paper_2511_05534_b200 import binding as F
from paper_2511_05534_b200 import build, inputs

import paged_util as T

pytestmark = pytest.mark.gpu


def _case(rng, U, Hq, H, D, page, rows, dtype, path=F.PATH_AUTO, exponents=(-3, 1)):
    table, n_pages = T.random_table(rng, rows, page)
    p = T.params(U, Hq, H, D, page, n_pages, table.shape[1], dtype=dtype, path=path)
    ck, ks = T.random_pool(rng, n_pages, H, page, D, rows, table, (-9, -6))
    cv, vs = T.random_pool(rng, n_pages, H, page, D, rows, table, exponents)
    return p, ck, cv, ks, vs, table


def simt_bound(size, logits, n, D):
    """How far the SIMT kernel may be from 64 bits, per output.  A logit: scale (1 / sqrt, times log2 e: 4 roundings) times query (1), 16 fused
    multiply-adds, 3 additions across lanes and the page's scale: 25 roundings of sums of at most `logits`; less the maximum, a difference of at most twice
    `logits`, here and where maxima change: 4 more; one spare.  A weight: exp2 within 2^-22, and as often again as its maximum changes: a step of at least 32 keys, the
    block's groups, the join (4).  Sums: 4 rows a step, up to 32 groups, a record for 64 keys or more.  Scales are powers of two.  Numerator and denominator."""
    steps = -(-n // 32)
    rel = 30 * 2.0 ** -24 * logits + (steps + 4) * (2.0 ** -22 + 2.0 ** -24) + (4 * steps + 36 + n / 64) * 2.0 ** -24
    return 2 * rel[:, None] * size + 1e-30


@pytest.mark.parametrize("dtype,path", [(F.F32, F.PATH_AUTO), (F.BF16, F.PATH_SIMT)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,H", [(3, 3), (8, 2), (7, 1)])
def test_simt_attention_has_fp32_errors_only(dtype, path, D, Hq, H):
    rng = np.random.default_rng(Hq + D + dtype)
    for page, scale, rows in ((16, 0.05, [1, 2, 31, 33, 64, 200]), (64, 1.0, [1, 63, 65, 129, 500, 3000]), (128, 0.3, [7, 0, 256, 90, 1, 1000])):
        rows = np.array(rows)
        p, ck, cv, ks, vs, table = _case(rng, len(rows), Hq, H, D, page, rows, dtype, path)
        q = (scale * rng.standard_normal((len(rows), Hq, D))).astype(np.float32)
        if dtype == F.BF16:
            q = inputs.round_to_bf16(q)
        got, status = T.attend(p, q, ck, cv, ks, vs, table, rows)
        want, size, logits = P.attention(q, P.E4M3[ck], P.E4M3[cv], ks, vs, table, rows, least=0.0)
        assert status == 0
        for u, n in enumerate(rows):
            bound = simt_bound(size[u], logits[u], int(n), D)
            assert (np.abs(got[u] - want[u]) <= bound).all(), (page, u, np.max(np.abs(got[u] - want[u]) / bound))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,H", [(2, 2), (8, 2), (8, 1)])
def test_queries_with_elements_far_apart(D, Hq, H):
    """Channels where queries are 2^6 to 2^20 times larger than elsewhere, and keys are zero, so that the small elements make the logits.  Tensor cores: an element is
    two e4m3 numbers, the second one 16 times finer, of the query scaled to a largest element in [128, 256): steps of 2^-13 at least, so each is
    within 2^-14 of 2^7, 2^-21 of the largest; SIMT: as any other."""
    rng = np.random.default_rng(D + Hq)
    rows, page = np.array([300, 40, 129]), 32
    p, ck, cv, ks, vs, table = _case(rng, 3, Hq, H, D, page, rows, F.BF16)
    ck[..., ::16] = 0
    for far in (6, 10, 13, 16, 20):
        q = rng.standard_normal((3, Hq, D))
        q[..., ::16] *= 2.0 ** far
        q = inputs.round_to_bf16(q.astype(np.float32))
        for path in (F.PATH_AUTO, F.PATH_SIMT):
            p.path = path
            got, status = T.attend(p, q, ck, cv, ks, vs, table, rows)
            want, size, logits = P.attention(q, P.E4M3[ck], P.E4M3[cv], ks, vs, table, rows)
            assert status == 0
            for u, n in enumerate(rows):
                if path == F.PATH_SIMT:
                    bound = simt_bound(size[u], logits[u], int(n), D)
                else:
                    keys = np.abs(P.load(P.E4M3[ck], ks, table[u], int(n))).sum(2).max(1)           # [H]
                    off = 2.0 ** -21 * np.abs(q[u]).max(1) * D ** -0.5 * np.repeat(keys, Hq // H)
                    # (a weight that is off by a factor of e^off, up or down)
                    bound = T.attention_bound(size[u], logits[u], int(n), D) + 2 * np.expm1(2 * off)[:, None] * size[u]
                assert (np.abs(got[u] - want[u]) <= bound).all(), (far, path, u, np.max(np.abs(got[u] - want[u]) / bound))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("path", [F.PATH_AUTO, F.PATH_SIMT])
@pytest.mark.parametrize("Hq,H", [(2, 2), (8, 2), (7, 1)])
def test_logits_of_any_size(path, D, Hq, H):
    """Queries of one element, 2^6 to 2^70, either sign: the largest logit is a key's, or two keys' alike, and so far above the others that they have all the
    weight; every logit is exact, so that of the bound the errors of weights and sums are left (paged_util.attention_bound without logits)."""
    rng = np.random.default_rng(D + Hq)
    rows, page = np.array([300, 40, 1500, 128]), 32
    p, ck, cv, ks, vs, table = _case(rng, 4, Hq, H, D, page, rows, F.BF16, path, exponents=(-6, 6))
    ks[:] = 2.0 ** -8
    ck[..., 5] = rng.integers(0x08, 0x58, ck.shape[:3])               # 2^-6 .. 15
    for u, n in enumerate(rows):
        for h in range(H):
            top = rng.choice(n, 2, replace=False)
            for sign, at in ((0, top[:1 + h % 2]), (0x80, rng.choice(np.setdiff1d(np.arange(n), top), 2, replace=False))):
                ck[table[u, at // page], h, at % page, 5] = sign | 0x7E    # 448, -448
    for e in (6, 10, 16, 20, 22, 24, 25, 26, 28, 31, 40, 70):
        for sign in (1, -1):
            q = np.zeros((4, Hq, D), np.float32)
            q[..., 5] = sign * 2.0 ** (e + 3)                          # (largest logit: 448 * 2^-8 * 2^(e + 3) / sqrt(D))
            got, status = T.attend(p, q, ck, cv, ks, vs, table, rows)
            want, size, _ = P.attention(q, P.E4M3[ck], P.E4M3[cv], ks, vs, table, rows)
            assert status == 0
            for u, n in enumerate(rows):
                bound = T.attention_bound(size[u], np.zeros(Hq), int(n), D)
                assert (np.abs(got[u] - want[u]) <= bound).all(), (e, sign, u, np.max(np.abs(got[u] - want[u]) / bound))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("path", [F.PATH_AUTO, F.PATH_SIMT])
@pytest.mark.parametrize("U,Hq,H", [(1, 8, 2), (3, 40, 40)])
def test_nan_in_a_head_that_is_cut(path, D, U, Hq, H):
    """Records of a range with a NaN among others: the head's outputs that it belongs to, bit for bit nothing else."""
    rng = np.random.default_rng(D + U)
    rows, page, G = np.array([9000, 8100, 7000])[:U], 64, Hq // H
    p, ck, cv, ks, vs, table = _case(rng, U, Hq, H, D, page, rows, F.BF16, path)
    q = inputs.round_to_bf16(rng.standard_normal((U, Hq, D)).astype(np.float32))
    clean, status = T.attend(p, q, ck, cv, ks, vs, table, rows)
    assert status == 0 and np.isfinite(clean).all()
    for at in (0, 4444, int(rows[0]) - 1):
        bad = ck.copy()
        bad[table[0, at // page], 1, at % page, 7] = 127
        got, status = T.attend(p, q, bad, cv, ks, vs, table, rows)
        assert status == 0 and np.isnan(got[0, G:2 * G]).all()
        got[0, G:2 * G] = clean[0, G:2 * G]
        assert np.array_equal(got, clean), at
        bad = cv.copy()
        bad[table[0, at // page], 0, at % page, D - 1] = 255
        got, status = T.attend(p, q, ck, bad, ks, vs, table, rows)
        assert status == 0 and np.isnan(got[0, :G, D - 1]).all()
        got[0, :G, D - 1] = clean[0, :G, D - 1]
        assert np.array_equal(got, clean), at


def test_the_build_with_index_checks(monkeypatch):
    """libflowmm_debug.so: the four calls give what the release library gives, and report what it reports."""
    rng = np.random.default_rng(3)
    U, Hq, H, D, page, n = 4, 8, 2, 64, 16, 21
    held = np.array([0, 3, 16, 40])
    rows = held + n
    table, n_pages = T.random_table(rng, rows, page)
    codes, scale = T.random_pool(rng, n_pages, H, page, D, held, table)
    pos = held[:, None] + np.arange(n)
    slots = (np.take_along_axis(table, pos // page, 1) * page + pos % page).astype(np.int32)
    k = T.dev(rng.standard_normal((U, H, n, D)).astype(np.float32), F.BF16)
    q = T.dev(rng.standard_normal((U, Hq, D)).astype(np.float32), F.BF16)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")

    def all_calls(table, slots):
        results = []
        for path in (F.PATH_AUTO, F.PATH_SIMT):
            p = T.params(U, Hq, H, D, page, n_pages, table.shape[1], n, path=path)
            ws, grow, out_rows, left, new = F.alloc_cache_workspace(p), i32(U), i32(U), i32(2), i32(U, n)
            held_d, t = T.dev(held.astype(np.int32)), T.dev(table)
            F.flowmm_cache_plan(p, grow, held_d, out_rows, i32(n_pages), i32(2), left, t, new, ws)
            pool = [T.dev(codes), T.dev(codes), T.dev(scale), T.dev(scale)]
            F.flowmm_cache_store(p, k, k, T.dev(slots), *pool, ws)
            out, rows_d = torch.zeros((U, Hq, D), device="cuda"), T.dev(rows.astype(np.int32))
            F.flowmm_cache_attention(p, q, *pool, t, rows_d, out, ws)
            dense = [torch.zeros_like(k) for _ in "kv"]
            F.flowmm_cache_load(p, *pool, t, rows_d, *dense, ws)
            results.append((F.flowmm_last_device_status(ws), [x.float().cpu().nan_to_num() for x in (out_rows, left, new, *pool, out, *dense)]))
        return results

    wrong = table.copy()
    wrong[3, 2] = n_pages
    gap = slots.copy()
    gap[1, 4] = -1
    release = [all_calls(t, s) for t, s in ((table, slots), (wrong, slots), (table, gap))]
    assert [[status for status, _ in r] for r in release] == [[0, 0], [10, 10], [10, 10]]
    monkeypatch.setattr(F, "LIB_PATH", build.build(debug=True))
    monkeypatch.setattr(F, "_lib", None)
    F.load()
    assert F.flowmm_debug_build()
    for (t, s), want in zip(((table, slots), (wrong, slots), (table, gap)), release):
        for (status, arrays), (status_r, arrays_r) in zip(all_calls(t, s), want):
            assert status == status_r and all(torch.equal(a, b) for a, b in zip(arrays, arrays_r))
