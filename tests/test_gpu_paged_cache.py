"""The paged 8-bit cache on the GPU against its 64-bit oracle: plans and codes are equal, dense rows too (a code times a power of two is a
bf16 number), attention within the bound that paged_util derives."""
import numpy as np
import pytest
import torch

from oracle import paged_cache as P
from paper_2511_05534_b200 import binding as F
from paper_2511_05534_b200 import inputs

import paged_util as T

pytestmark = pytest.mark.gpu


# ---- plan ----------------------------------------------------------------------------------------

def _plan_case(rng, U, page, wide, n_rows, spare, grow):
    rows = rng.integers(0, wide * page + 1, U).astype(np.int32)
    if U > 2:
        rows[0], rows[1] = 0, wide * page
    held = [P.pages(int(r), page) for r in rows]
    n_pages = sum(held) + spare
    order = rng.permutation(n_pages).astype(np.int32)
    table = np.full((U, wide), -7, np.int32)
    at = 0
    for u, h in enumerate(held):
        table[u, :h] = order[at:at + h]
        at += h
    head = int(rng.integers(0, n_pages))
    ring = np.full(n_pages, -9, np.int32)
    for i, x in enumerate(order[at:]):
        ring[(head + i) % n_pages] = x
    return rows, grow(rows), ring, np.array([head, spare], np.int32), table


def _plan(p, rows, grow, ring, state, table, slots=True):
    d = dict(grow=T.dev(grow), rows=T.dev(rows), rows_out=torch.full((p.n_units,), -5, dtype=torch.int32, device="cuda"), ring=T.dev(ring),
             state=T.dev(state), state_out=torch.full((2,), -5, dtype=torch.int32, device="cuda"), table=T.dev(table),
             slots=torch.full((p.n_units, p.n_rows), -5, dtype=torch.int32, device="cuda") if slots else None)
    ws = F.alloc_cache_workspace(p)
    F.flowmm_cache_plan(p, d["grow"], d["rows"], d["rows_out"], d["ring"], d["state"], d["state_out"], d["table"], d["slots"], ws)
    status = F.flowmm_last_device_status(ws)
    assert torch.equal(d["rows"].cpu(), torch.from_numpy(rows)) and torch.equal(d["state"].cpu(), torch.from_numpy(state))
    return [None if t is None else t.cpu().numpy() for t in (d["rows_out"], d["state_out"], d["table"], d["ring"], d["slots"])], status


@pytest.mark.parametrize("U,page,wide,n_rows,spare", [(1, 16, 1, 1, 1), (1, 64, 27, 1690, 27), (7, 32, 9, 5, 3), (48, 64, 40, 1, 30), (513, 16, 12, 3, 200),
                                                      (320, 64, 8, 400, 1500), (1700, 128, 3, 257, 900)])
@pytest.mark.parametrize("slots", [True, False])
def test_plan_equals_oracle(U, page, wide, n_rows, spare, slots):
    """Growing, shrinking, ending and waiting units, with pools and tables that are too small for some."""
    rng = np.random.default_rng(U + page)
    for kind in range(3):
        def grow(rows):
            if kind == 0:
                return np.ones_like(rows)
            g = rng.integers(-wide * page, n_rows + 3, U).astype(np.int32)
            if kind == 2:
                g = np.where(rng.random(U) < 0.5, -rows, np.where(rng.random(U) < 0.3, 0, g % (n_rows + 1)))
            return g.astype(np.int32)
        rows, g, ring, state, table = _plan_case(rng, U, page, wide, n_rows, spare, grow)
        p = T.params(U, 1, 1, 128, page, len(ring), wide, n_rows)
        got, status = _plan(p, rows, g, ring, state, table, slots)
        want = P.plan(g, rows, ring, state, table, page, n_rows, slots)
        for name, a, b in zip(("rows", "state", "table", "ring"), got, want):
            assert np.array_equal(a, b), (kind, name)
        if slots:
            assert np.array_equal(got[4], want[4]), kind
        assert status == (11 if want[5] else 0), (kind, status)


def test_plan_without_slots_takes_any_growth_and_none():
    """n_rows = 0, slots NULL: pages are given out and taken back, whatever the growth."""
    rng = np.random.default_rng(5)
    rows, g, ring, state, table = _plan_case(rng, 6, 16, 50, 1, 120, lambda r: np.array([300, -5, 0, 90, -10000, 1], np.int32))
    got, status = _plan(T.params(6, 1, 1, 128, 16, len(ring), 50, 0), rows, g, ring, state, table, slots=False)
    want = P.plan(g, rows, ring, state, table, 16, 0, False)
    assert status == (11 if want[5] else 0) and all(np.array_equal(a, b) for a, b in zip(got[:4], want[:4]))


def test_a_plan_thrown_away_is_made_again():
    """The same step planned twice gives the same, and so does another one planned between."""
    rng = np.random.default_rng(6)
    rows, g, ring, state, table = _plan_case(rng, 40, 32, 30, 5, 90, lambda r: rng.integers(-400, 6, 40).astype(np.int32))
    p = T.params(40, 1, 1, 128, 32, len(ring), 30, 5)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    d = [T.dev(x) for x in (g, rows, ring, state, table)]
    ws, results = F.alloc_cache_workspace(p), []
    for grow in (d[0], torch.ones_like(d[0]), d[0]):
        out, left, slots = i32(40), i32(2), i32(40, 5)
        F.flowmm_cache_plan(p, grow, d[1], out, d[2], d[3], left, d[4], slots, ws)
        held = (out.cpu().numpy() + 31) // 32
        results.append([out.cpu(), left.cpu(), slots.cpu(), [d[4].cpu()[u, :held[u]] for u in range(40)]])
    for a, b in zip(results[0][:3], results[2][:3]):
        assert torch.equal(a, b)
    assert all(torch.equal(a, b) for a, b in zip(results[0][3], results[2][3]))


def test_plan_of_unsound_state_changes_nothing():
    """Numbers out of range where the call reads lengths or the ring's state: reported, and nothing is taken."""
    rng = np.random.default_rng(3)
    rows, g, ring, state, table = _plan_case(rng, 5, 16, 4, 2, 6, np.ones_like)
    p = T.params(5, 1, 1, 128, 16, len(ring), 4, 2)
    for bad in ([-1, 3], [len(ring), 3], [0, -1], [0, len(ring) + 1]):
        got, status = _plan(p, rows, g, ring, np.array(bad, np.int32), table)
        assert status == 10 and np.array_equal(got[0], rows) and got[1].tolist() == bad
        assert np.array_equal(got[2], table) and np.array_equal(got[3], ring) and (got[4] == -1).all()
    for wrong in (-3, 65):
        rows2 = rows.copy()
        rows2[2] = wrong
        got, status = _plan(p, rows2, np.where(np.arange(5) == 2, 1, 0).astype(np.int32), ring, state, table)
        assert status == 10 and np.array_equal(got[0], rows2) and np.array_equal(got[2], table)
    far = g.copy()
    far[1], far[3] = 2 ** 31 - 1, -2 ** 31                          # (sums that pass 32 bits)
    got, status = _plan(p, rows, far, ring, state, table)
    want = P.plan(far, rows, ring, state, table, 16, 2)
    assert status == 11 and all(np.array_equal(a, b) for a, b in zip(got, want))


def test_plan_reports_bad_page_numbers_and_makes_no_slots_of_them():
    """Numbers out of range in the table (of a page that is held, of one given back) and in the ring."""
    page, n_pages = 16, 6
    rows, grow = np.array([20, 20, 20], np.int32), np.array([2, 2, -20], np.int32)
    table, ring, state = np.array([[0, 1], [2, 3], [4, 5]], np.int32), np.zeros(n_pages, np.int32), np.array([0, 0], np.int32)
    p = T.params(3, 1, 1, 128, page, n_pages, 2, 2)
    got, status = _plan(p, rows, grow, ring, state, table)
    assert status == 0 and got[4].tolist() == [[20, 21], [52, 53], [-1, -1]]
    for bad in (-1, n_pages, 1 << 28, (1 << 28) + 1, 2 ** 31 - 1, -2 ** 31):      # (2^28 pages of 16: slots that would wrap to pages 0 and 1)
        wrong = table.copy()
        wrong[0, 1] = bad
        got, status = _plan(p, rows, grow, ring, state, wrong)
        assert status == 10 and got[4].tolist() == [[-1, -1], [52, 53], [-1, -1]] and got[0].tolist() == [22, 22, 0]
        wrong = table.copy()
        wrong[2, 0] = bad
        got, status = _plan(p, rows, grow, ring, state, wrong)
        assert status == 10 and got[4].tolist() == [[20, 21], [52, 53], [-1, -1]]
        got, status = _plan(p, np.array([16, 16, 0], np.int32), np.array([1, 1, 0], np.int32), np.array([bad, 5, 0, 0, 0, 0], np.int32),
                            np.array([0, 2], np.int32), table)
        assert status == 10 and got[4].tolist() == [[-1, -1], [80, -1], [-1, -1]]


# ---- store and load ------------------------------------------------------------------------------

def _store(p, k, v, slots, codes_k, codes_v, ks, vs):
    d = [T.dev(codes_k), T.dev(codes_v), T.dev(ks), T.dev(vs)]
    ws = F.alloc_cache_workspace(p)
    F.flowmm_cache_store(p, k, v, T.dev(slots), *d, ws)
    return [t.cpu().numpy() for t in d], F.flowmm_last_device_status(ws)


def _rows(rng, shape, dtype):
    """Rows with sizes from page to page 2^-20 to 2^20, zeros, and values that fall under the codes' range."""
    x = rng.standard_normal(shape) * 2.0 ** rng.integers(-20, 21, shape[:3])[..., None] * 2.0 ** -rng.integers(0, 14, shape)
    x[..., ::9] = 0
    x = x.astype(np.float32)
    return inputs.round_to_bf16(x) if dtype == F.BF16 else x


@pytest.mark.parametrize("dtype", [F.F32, F.BF16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("n", [1, 2, 15, 17, 131])
def test_store_equals_oracle(dtype, D, page, n):
    rng = np.random.default_rng(1000 * page + n + D + dtype)
    U, H = 5, 3
    held = np.array([0, 1, page - 1, page, 2 * page + page // 2 + 3])
    fresh = np.array([n, max(0, n - 1), n, n // 2, n])              # (padded: the last slots of some units are -1)
    table, n_pages = T.random_table(rng, held + n, page)
    codes_k, ks = T.random_pool(rng, n_pages, H, page, D, held, table)
    codes_v, vs = T.random_pool(rng, n_pages, H, page, D, held, table, (-20, 20))
    slots = np.full((U, n), -1, np.int32)
    for u in range(U):
        pos = held[u] + np.arange(fresh[u])
        slots[u, :fresh[u]] = table[u, pos // page] * page + pos % page
    k, v = _rows(rng, (U, H, n, D), dtype), _rows(rng, (U, H, n, D), dtype)
    k[0, 0, 0, 3], k[2, 1, n - 1, 5], v[2, 2, 0, 7] = np.nan, np.inf, -np.inf
    p = T.params(U, H, H, D, page, n_pages, table.shape[1], n, dtype)
    got, status = _store(p, T.dev(k, dtype), T.dev(v, dtype), slots, codes_k, codes_v, ks, vs)
    assert status == 0
    for x, before, s, codes, scale in ((k, codes_k, ks, got[0], got[2]), (v, codes_v, vs, got[1], got[3])):
        want, want_s = P.store(x, slots, P.E4M3[before], s)
        assert np.array_equal(scale.astype(np.float64), want_s)
        assert np.array_equal(P.E4M3[codes], want, equal_nan=True)
        touched = np.zeros((n_pages, page), bool)                   # places that no row went to keep their bytes
        for u in range(U):
            for t in range(fresh[u]):
                touched.reshape(-1)[slots[u, t]] = True
            if fresh[u] and held[u] % page:
                touched[table[u, held[u] // page], :held[u] % page] = True
        assert np.array_equal(np.moveaxis(codes, 2, 1)[~touched], np.moveaxis(before, 2, 1)[~touched])


def test_store_of_strided_rows_and_wild_scales():
    """Rows as views of [units, rows, heads, head_dim]; a page whose scale no store has written."""
    rng = np.random.default_rng(8)
    U, H, n, D, page = 3, 2, 20, 128, 32
    x = inputs.round_to_bf16(rng.standard_normal((U, n, H, D)).astype(np.float32))
    big = T.dev(np.concatenate([x, x[:, :3]], 1), F.BF16)
    k = big[:, :n].transpose(1, 2)
    assert not k.is_contiguous()
    held = np.array([5, 0, 31])
    table, n_pages = T.random_table(rng, held + n, page)
    pos = held[:, None] + np.arange(n)
    slots = (np.take_along_axis(table, pos // page, 1) * page + pos % page).astype(np.int32)
    codes, scale = T.random_pool(rng, n_pages, H, page, D, held, table)
    p = T.params(U, H, H, D, page, n_pages, table.shape[1], n)
    got, status = _store(p, k, k, slots, codes, codes, scale, scale)
    want, want_s = P.store(np.moveaxis(x, 1, 2), slots, P.E4M3[codes], scale)
    assert status == 0 and np.array_equal(got[2], want_s) and np.array_equal(P.E4M3[got[1]], want, equal_nan=True)
    for wild in (np.nan, -1.0, 0.0, np.inf, 1e-40, 3.0):
        s2 = np.full_like(scale, wild)
        got, status = _store(p, k, k, slots, codes, codes, s2, s2)
        s = got[2][table[0, 0]]
        assert status == 0 and (np.log2(s) == np.round(np.log2(s))).all() and (s >= (4.0 if wild == 3.0 else 2.0 ** -96)).all()
        fresh = P.E4M3[got[0][table[0, 0], :, 5:5 + n]] * s[:, None, None]
        ideal = np.moveaxis(x[0], 0, 1)
        step = np.maximum(np.abs(ideal) * 2.0 ** -4, s[:, None, None] * 2.0 ** -10)      # half a step of a code
        assert (np.abs(fresh - ideal) <= step).all()


def test_bad_slots_are_reported_and_write_nothing_else():
    rng = np.random.default_rng(9)
    U, H, n, D, page, n_pages = 4, 2, 6, 64, 16, 8
    x = T.dev(rng.standard_normal((U, H, n, D)).astype(np.float32))
    good = np.array([[u * 32 + t for t in range(n)] for u in range(U)], np.int32)
    p = T.params(U, H, H, D, page, n_pages, 2, n, F.F32)
    codes = rng.integers(0, 256, (n_pages, H, page, D)).astype(np.uint8)
    scale = np.ones((n_pages, H), np.float32)
    for bad in (-2, n_pages * page, 2 ** 31 - 1, -2 ** 31):
        slots = good.copy()
        slots[1, 0] = bad
        got, status = _store(p, x, x, slots, codes, codes, scale, scale)
        assert status == 10 and np.array_equal(got[0][2:4], codes[2:4])
    slots = good.copy()
    slots[2, 3] = 100                                               # not where the row before it says
    got, status = _store(p, x, x, slots, codes, codes, scale, scale)
    assert status == 10 and np.array_equal(got[0][100 // 16][:, 6:], codes[100 // 16][:, 6:]) and np.array_equal(got[0][4, :, 3], codes[4, :, 3])
    slots = np.full_like(good, -1)
    got, status = _store(p, x, x, slots, codes, codes, scale, scale)
    assert status == 0 and np.array_equal(got[0], codes) and np.array_equal(got[2], scale)


@pytest.mark.parametrize("n", [20, 300])
@pytest.mark.parametrize("D,page", [(64, 16), (128, 32), (128, 128)])
def test_rows_behind_one_without_a_place_are_reported(D, page, n):
    """Slots of -1 in front of a unit's rows, or where a page begins: the rows of those pages are not stored, and the call says so."""
    rng = np.random.default_rng(page + n)
    pages = n // page + 2
    x = T.dev(rng.standard_normal((2, 2, n, D)).astype(np.float32))
    p = T.params(2, 2, 2, D, page, 2 * pages, pages, n, F.F32)
    codes, scale = rng.integers(0, 256, (2 * pages, 2, page, D)).astype(np.uint8), np.ones((2 * pages, 2), np.float32)
    good = np.stack([np.arange(n), pages * page + np.arange(n)]).astype(np.int32)
    want, status = _store(p, x, x, good, codes, codes, scale, scale)
    assert status == 0
    for t0, t1 in ((0, 1), (0, 3), (0, n - 1), (n // page * page, n // page * page + 1)):
        if t1 >= n:
            continue                                                # (nothing behind it)
        slots = good.copy()
        slots[0, t0:t1] = -1
        got, status = _store(p, x, x, slots, codes, codes, scale, scale)
        assert status == 10 and np.array_equal(got[0][pages:], want[0][pages:]) and np.array_equal(got[2][pages:], want[2][pages:]), (t0, t1)
        assert np.array_equal(got[0][t0 // page], codes[t0 // page])


@pytest.mark.parametrize("dtype", [F.F32, F.BF16])
@pytest.mark.parametrize("D,page", [(64, 16), (64, 128), (128, 32), (128, 64)])
def test_load_equals_oracle(dtype, D, page):
    rng = np.random.default_rng(D + page + dtype)
    H = 3
    rows = np.array([0, 1, page, page + 1, 5 * page - 2, 333])
    table, n_pages = T.random_table(rng, rows, page)
    codes_k, ks = T.random_pool(rng, n_pages, H, page, D, rows, table)
    codes_v, vs = T.random_pool(rng, n_pages, H, page, D, rows, table)
    for n in (1, page, 200, 400, 900):
        p = T.params(len(rows), H, H, D, page, n_pages, table.shape[1], n, dtype)
        out = torch.full((len(rows), n + 2, H, D), 7.0, dtype=F.torch_dtype(dtype), device="cuda")
        k, v = out[:, :n].transpose(1, 2), torch.full((len(rows), H, n, D), 7.0, dtype=F.torch_dtype(dtype), device="cuda")
        ws = F.alloc_cache_workspace(p)
        F.flowmm_cache_load(p, T.dev(codes_k), T.dev(codes_v), T.dev(ks), T.dev(vs), T.dev(table), T.dev(rows.astype(np.int32)), k, v, ws)
        assert F.flowmm_last_device_status(ws) == 0
        for t, codes, s in ((k, codes_k, ks), (v, codes_v, vs)):
            got = t.float().cpu().numpy()
            for u, r in enumerate(rows):
                m = min(int(r), n)
                assert np.array_equal(got[u, :, :m], P.load(P.E4M3[codes], s, table[u], m)) and (got[u, :, m:] == 7).all(), (n, u)
        assert (out[:, n:] == 7).all()


def test_bad_pages_are_reported(D=64, page=16):
    """Numbers out of range in the block table and in rows, for the two readers."""
    rng = np.random.default_rng(4)
    rows = np.array([40, 20, 33])
    table, n_pages = T.random_table(rng, rows, page)
    codes, s = T.random_pool(rng, n_pages, 2, page, D, rows, table)
    q = rng.standard_normal((3, 2, D)).astype(np.float32)
    p = T.params(3, 2, 2, D, page, n_pages, 3, 40, F.F32)
    good, status = T.attend(p, q, codes, codes, s, s, table, rows)
    assert status == 0
    for bad in (-1, n_pages, 2 ** 31 - 1, -2 ** 31):
        t2 = table.copy()
        t2[1, 1] = bad
        out, status = T.attend(p, q, codes, codes, s, s, t2, rows)
        assert status == 10 and np.array_equal(out[[0, 2]], good[[0, 2]])
        k = torch.zeros((3, 2, 40, D), device="cuda")
        ws = F.alloc_cache_workspace(p)
        F.flowmm_cache_load(p, T.dev(codes), T.dev(codes), T.dev(s), T.dev(s), T.dev(t2), T.dev(rows.astype(np.int32)), k, k.clone(), ws)
        assert F.flowmm_last_device_status(ws) == 10
        assert np.array_equal(k[2, :, :33].cpu().numpy(), P.load(P.E4M3[codes], s, table[2], 33)) and (k[1, :, 16:] == 0).all()
    for bad in (-5, 49, 2 ** 31 - 1):
        r2 = rows.copy()
        r2[1] = bad
        t2 = table.copy()
        t2[1] = table[0]
        out, status = T.attend(p, q, codes, codes, s, s, t2, r2)
        assert status == 10 and np.array_equal(out[[0, 2]], good[[0, 2]])


# ---- attention -----------------------------------------------------------------------------------

def _check(p, rng, rows, page, spare=3, wide=None, exponents=(-3, 1), scale=1.0, softmax_scale=0.0):
    U, Hq, H, D = p.n_units, p.n_q_heads, p.n_kv_heads, p.head_dim
    table, n_pages = T.random_table(rng, rows, page, spare, wide)
    p.n_pages, p.max_pages, p.softmax_scale = n_pages, table.shape[1], softmax_scale
    codes_k, ks = T.random_pool(rng, n_pages, H, page, D, rows, table, (-9, -6))       # (codes go up to 448)
    codes_v, vs = T.random_pool(rng, n_pages, H, page, D, rows, table, exponents)
    q = (scale * rng.standard_normal((U, Hq, D))).astype(np.float32)
    if p.dtype == F.BF16:
        q = inputs.round_to_bf16(q)
    got, status = T.attend(p, q, codes_k, codes_v, ks, vs, table, rows)
    want, size, logits = P.attention(q, P.E4M3[codes_k], P.E4M3[codes_v], ks, vs, table, rows, softmax_scale)
    assert status == 0
    for u in range(U):
        bound = T.attention_bound(size[u], logits[u], int(rows[u]), D)
        assert (np.abs(got[u] - want[u]) <= bound).all(), (u, int(rows[u]), np.max(np.abs(got[u] - want[u]) / bound))
    return got, q, (codes_k, codes_v, ks, vs, table)


@pytest.mark.parametrize("dtype,path", [(F.F32, F.PATH_AUTO), (F.BF16, F.PATH_AUTO), (F.BF16, F.PATH_SIMT)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (2, 1), (6, 2), (8, 2), (5, 1), (28, 4), (8, 1), (32, 32)])
def test_attention_against_oracle(dtype, path, D, Hq, Hkv):
    rng = np.random.default_rng(Hq + 100 * Hkv + D + dtype)
    for page in (16, 32, 64, 128):
        rows = np.array([0, 1, 2, page - 1, page, page + 1, 127, 128, 129, 300, 0])[:4 if Hkv == 32 else None]
        _check(T.params(len(rows), Hq, Hkv, D, page, 1, 1, dtype=dtype, path=path), rng, rows, page)


@pytest.mark.parametrize("path", [F.PATH_AUTO, F.PATH_SIMT])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_of_long_and_many_units(path, D):
    """Ranges of many tiles, units without rows among long ones, more units than a block has threads."""
    rng = np.random.default_rng(D + path)
    _check(T.params(1, 4, 1, D, 64, 1, 1, path=path), rng, np.array([20011]), 64)
    _check(T.params(3, 8, 1, D, 16, 1, 1, path=path), rng, np.array([9001, 0, 5]), 16)
    _check(T.params(500, 2, 1, D, 32, 1, 1, path=path), rng, rng.integers(0, 90, 500), 32)
    _check(T.params(40, 14, 2, D, 128, 1, 1, path=path), rng, rng.integers(0, 2000, 40), 128, wide=64)


@pytest.mark.parametrize("U,Hq,Hkv,lengths", [
    (1, 8, 2, [1700]),                                  # few heads: ranges, a few a head
    (1, 7, 1, [40000]), (1, 1, 1, [9000]),              # ... and up to 64
    (3, 64, 8, [129, 4000, 1]), (30, 28, 4, None), (7, 5, 5, None),
    (37, 32, 8, None), (38, 8, 8, None), (64, 64, 8, None), (64, 9, 9, None), (60, 16, 8, [0, 1700, 0, 900]),   # about and above 296 heads, up to 592: pairs
    (64, 8, 8, [1700]), (48, 8, 8, [5000] + [100] * 47),                                    # ... which would be uneven: pieces
    (70, 16, 8, None), (75, 64, 8, [1, 0, 300]), (300, 1, 1, [30000] + [20] * 299),         # many: pieces, some of a hundred to a head
    (1, 1000, 1000, [40]), (2, 1400, 700, [0, 130]),    # ... and many heads to a piece
    (3, 8, 2, [0]), (40, 8, 8, [0]), (80, 16, 8, [0])]) # nothing at all
def test_every_way_to_share_the_work_out(U, Hq, Hkv, lengths):
    rng = np.random.default_rng(U + Hq)
    rows = rng.integers(0, 1800, U) if lengths is None else np.array([lengths[u % len(lengths)] for u in range(U)])
    _check(T.params(U, Hq, Hkv, 128 if U % 2 else 64, 64, 1, 1), rng, rows, 64)


def test_queries_of_one_sequence_share_its_pages():
    """Several new tokens of a sequence: units with the same row of the block table, each one row longer than the one before."""
    rng = np.random.default_rng(2)
    n, rows = 5, np.array([700])
    table, n_pages = T.random_table(rng, rows, 64)
    codes_k, ks = T.random_pool(rng, n_pages, 2, 64, 128, rows, table, (-9, -6))
    codes_v, vs = T.random_pool(rng, n_pages, 2, 64, 128, rows, table)
    tables, lens = np.repeat(table, n, 0), rows[0] - n + 1 + np.arange(n)
    q = inputs.round_to_bf16(rng.standard_normal((n, 8, 128)).astype(np.float32))
    for path in (F.PATH_AUTO, F.PATH_SIMT):
        got, status = T.attend(T.params(n, 8, 2, 128, 64, n_pages, table.shape[1], path=path), q, codes_k, codes_v, ks, vs, tables, lens)
        want, size, logits = P.attention(q, P.E4M3[codes_k], P.E4M3[codes_v], ks, vs, tables, lens)
        assert status == 0
        for u in range(n):
            assert (np.abs(got[u] - want[u]) <= T.attention_bound(size[u], logits[u], int(lens[u]), 128)).all()


class Guarded:
    """A tensor between two margins that must keep their bytes."""

    def __init__(self, t):
        n = t.numel() * t.element_size()
        self.raw = torch.full((4096 + n + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
        self.t = self.raw[4096:4096 + n].view(t.dtype).view(t.shape)
        self.t.copy_(t)

    def intact(self):
        return bool((self.raw[:4096] == 0xA5).all() and (self.raw[4096 + self.t.numel() * self.t.element_size():] == 0xA5).all())


@pytest.mark.parametrize("D,dtype,path", [(64, F.BF16, F.PATH_AUTO), (128, F.BF16, F.PATH_AUTO), (128, F.BF16, F.PATH_SIMT), (64, F.F32, F.PATH_AUTO)])
def test_nothing_is_written_beside_the_outputs(D, dtype, path):
    """Every array of the four calls, and a workspace of exactly the size that is asked for, between guards; inputs keep their bytes."""
    rng = np.random.default_rng(D + path)
    U, Hq, H, page, n = 9, 21, 3, 32, 77
    rows = np.array([0, 5, 1000, 31, 32, 33, 400, 77, 2000])
    table, n_pages = T.random_table(rng, rows + n, page, spare=50)
    p = T.params(U, Hq, H, D, page, n_pages, table.shape[1], n, dtype, path=path)
    guards = {}

    def guard(name, t):
        guards[name] = Guarded(t)
        return guards[name].t
    ws = guard("ws", F.alloc_cache_workspace(p))
    pool = [guard("pool%d" % i, T.dev(x)) for i, x in enumerate((*(T.random_pool(rng, n_pages, H, page, D, rows, table)[0] for _ in "kv"),
                                                                 *(np.ones((n_pages, H), np.float32) for _ in "kv")))]
    i32 = lambda x: T.dev(np.asarray(x, np.int32))
    ring = guard("ring", i32(np.full(n_pages, 3)))
    fresh = {"rows": guard("rows", i32(rows)), "grow": guard("grow", i32(np.full(U, n))), "state": guard("state", i32([0, 40]))}
    table_d, slots = guard("table", i32(np.where(table < n_pages, table, 0))), guard("slots", i32(np.zeros((U, n))))
    keep = {k: t.clone() for k, t in fresh.items()}
    rows_out, state_out = guard("rows_out", i32(np.zeros(U))), guard("state_out", i32([0, 0]))
    F.flowmm_cache_plan(p, fresh["grow"], fresh["rows"], rows_out, ring, fresh["state"], state_out, table_d, slots, ws)
    assert F.flowmm_last_device_status(ws) in (0, 11)
    pos = rows[:, None] + np.arange(n)
    slots.copy_(i32(np.take_along_axis(table, pos // page, 1) * page + pos % page))
    table_d.copy_(i32(np.where(table < n_pages, table, 0)))
    tdt = F.torch_dtype(dtype)
    k, v = guard("k", torch.randn(U, H, n, D, device="cuda", dtype=tdt)), guard("v", torch.randn(U, H, n, D, device="cuda", dtype=tdt))
    q, out = guard("q", torch.randn(U, Hq, D, device="cuda", dtype=tdt)), guard("out", torch.zeros(U, Hq, D, device="cuda"))
    F.flowmm_cache_store(p, k, v, slots, *pool, ws)
    held = i32(rows + n)
    F.flowmm_cache_attention(p, q, *pool, table_d, held, out, ws)
    F.flowmm_cache_load(p, *pool, table_d, held, k, v, ws)
    assert F.flowmm_last_device_status(ws) == 0 and torch.isfinite(out).all()
    assert all(g.intact() for g in guards.values()), [name for name, g in guards.items() if not g.intact()]
    assert all(torch.equal(t, fresh[k]) for k, t in keep.items())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("path", [F.PATH_AUTO, F.PATH_SIMT])
def test_sharp_and_flat_softmax_and_scales_far_apart(path, D):
    rng = np.random.default_rng(17 + path)
    for scale, soft in ((6.0, 0.0), (1.0, 0.7), (1e-3, 0.0), (0.0, 0.0)):
        _check(T.params(3, 8, 2, D, 64, 1, 1, path=path), rng, np.array([700, 65, 1500]), 64, scale=scale, softmax_scale=soft)
    for exponents in ((-90, -60), (-30, 30), (60, 100)):
        _check(T.params(3, 8, 2, D, 16, 1, 1, path=path), rng, np.array([700, 65, 1500]), 16, exponents=exponents)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype,path", [(F.F32, F.PATH_AUTO), (F.BF16, F.PATH_AUTO), (F.BF16, F.PATH_SIMT)])
def test_nan_reaches_what_it_belongs_to_and_nothing_else(dtype, path, D):
    """A NaN in a row that a unit holds, or in a query: in that unit's outputs, in those heads and (from V) in that place.  (Rows
    behind the last one hold NaN in every test here.)"""
    rng = np.random.default_rng(5)
    rows, page = np.array([200, 130]), 64
    p = T.params(2, 4, 2, D, page, 1, 1, dtype=dtype, path=path)
    clean, q, (ck, cv, ks, vs, table) = _check(p, rng, rows, page)
    ck2 = ck.copy()
    ck2[table[0, 1], 0, 3, 5] = 255
    got, _ = T.attend(p, q, ck2, cv, ks, vs, table, rows)
    assert np.isnan(got[0, :2]).all() and np.array_equal(got[0, 2:], clean[0, 2:]) and np.array_equal(got[1], clean[1])
    cv2 = cv.copy()
    cv2[table[1, 2], 1, 1, 9] = 127
    got, _ = T.attend(p, q, ck, cv2, ks, vs, table, rows)
    assert np.isnan(got[1, 2:, 9]).all() and np.isnan(got).sum() == 2 and np.array_equal(got[0], clean[0])
    for bad in (np.nan, np.inf):
        q2 = q.copy()
        q2[0, 3, 60] = bad
        got, _ = T.attend(p, q2, ck, cv, ks, vs, table, rows)
        assert np.isnan(got[0, 3]).all() and np.isnan(got).sum() == D and np.array_equal(got[0, :3], clean[0, :3])


def test_attention_repeats_bit_by_bit_and_on_any_workspace():
    """Which range of a head ends last has no influence; the workspace may hold anything but in its first 256 bytes."""
    rng = np.random.default_rng(6)
    rows = rng.integers(1, 5000, 9)
    for path in (F.PATH_AUTO, F.PATH_SIMT):
        p = T.params(9, 16, 2, 128, 64, 1, 1, path=path)
        first, q, (ck, cv, ks, vs, table) = _check(p, rng, rows, 64)
        for fill in (0, 255, 1):
            ws = torch.full((F.flowmm_cache_workspace_bytes(p),), fill, dtype=torch.uint8, device="cuda")
            ws[:256] = 0
            for _ in range(3):
                got, status = T.attend(p, q, ck, cv, ks, vs, table, rows, ws)
                assert status == 0 and np.array_equal(got, first)


def test_pool_of_more_than_32_bits():
    """Pages whose place in the pool passes 2^31 and 2^32 bytes."""
    rng = np.random.default_rng(12)
    H, page, D = 8, 128, 128
    n_pages = (1 << 32) // (H * page * D) + 40
    rows = np.array([300, 129])
    codes = torch.zeros((n_pages, H, page, D), dtype=torch.uint8, device="cuda")
    scale = torch.full((n_pages, H), 2.0 ** -7, device="cuda")
    table = np.array([[n_pages - 1, 3, n_pages - 20], [(1 << 31) // (H * page * D) + 1, n_pages - 7, 0]], np.int32)
    small = rng.integers(0, 126, (6, H, page, D)).astype(np.uint8)
    compact = np.arange(6, dtype=np.int32).reshape(2, 3)
    for a, b in zip(table.reshape(-1), range(6)):
        codes[int(a)] = torch.from_numpy(small[b]).cuda()
    q = inputs.round_to_bf16(rng.standard_normal((2, 64, D)).astype(np.float32))
    s6 = np.full((6, H), 2.0 ** -7, np.float32)
    want, size, logits = P.attention(q, P.E4M3[small], P.E4M3[small], s6, s6, compact, rows)
    for path in (F.PATH_AUTO, F.PATH_SIMT):
        p = T.params(2, 64, H, D, page, n_pages, 3, 300, path=path)
        ws = F.alloc_cache_workspace(p)
        out = torch.zeros((2, 64, D), device="cuda")
        rd, td = T.dev(rows.astype(np.int32)), T.dev(table)
        F.flowmm_cache_attention(p, T.dev(q, F.BF16), codes, codes, scale, scale, td, rd, out, ws)
        for u in range(2):
            assert (np.abs(out[u].cpu().numpy() - want[u]) <= T.attention_bound(size[u], logits[u], int(rows[u]), D)).all()
    k = torch.zeros((2, H, 300, D), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    F.flowmm_cache_load(p, codes, codes, scale, scale, td, rd, k, v, ws)
    for u, n in enumerate(rows):
        assert np.array_equal(v[u, :, :n].float().cpu().numpy(), P.load(P.E4M3[small], s6, compact[u], n))
    slots = (np.repeat(table, page, 1) * page + np.tile(np.arange(page), 3))[:, :300].astype(np.int32)
    codes.zero_()
    F.flowmm_cache_store(p, k, k, T.dev(slots), codes, codes.clone(), scale, scale.clone(), ws)
    assert F.flowmm_last_device_status(ws) == 0
    want_c, want_s = P.store(k[1:].float().cpu().numpy(), np.array([[*range(300)]], np.int32), np.zeros((3, H, page, D)), np.ones((3, H)))
    got = codes[torch.from_numpy(table[1]).long().cuda()].cpu().numpy()
    assert np.array_equal(P.E4M3[got][:, :, :44], want_c[:, :, :44]) and np.array_equal(scale[torch.from_numpy(table[1]).long().cuda()].cpu().numpy(), want_s)


# ---- together ------------------------------------------------------------------------------------

class Server:
    """A pool with units in service, as a program keeps them: planned, stored into, attended to; and the same in numpy."""

    def __init__(self, U, Hq, H, D, page, n_pages, wide, dtype, rng):
        self.p = lambda n=1: T.params(U, Hq, H, D, page, n_pages, wide, n, dtype)
        self.ws = F.alloc_cache_workspace(self.p(1690))
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
        self.rows, self.rows_out, self.state, self.state_out = i32(U), i32(U), i32(2), i32(2)
        self.state[1] = n_pages
        self.ring = T.dev(rng.permutation(n_pages).astype(np.int32))
        self.table = i32(U, wide)
        self.pool = [torch.randint(0, 256, (n_pages, H, page, D), dtype=torch.uint8, device="cuda") for _ in "kv"] + [torch.ones((n_pages, H), device="cuda") for _ in "kv"]
        self.mirror = [P.E4M3[t.cpu().numpy()] for t in self.pool[:2]] + [t.cpu().numpy() for t in self.pool[2:]]
        self.book = [self.rows.cpu().numpy(), self.ring.cpu().numpy(), self.state.cpu().numpy(), self.table.cpu().numpy()]
        self.page = page

    def plan(self, grow, n):
        slots = torch.empty((self.rows.numel(), n), dtype=torch.int32, device="cuda")
        F.flowmm_cache_plan(self.p(n), T.dev(grow), self.rows, self.rows_out, self.ring, self.state, self.state_out, self.table, slots, self.ws)
        self.rows, self.rows_out, self.state, self.state_out = self.rows_out, self.rows, self.state_out, self.state
        rows, ring, state, table = self.book
        out, left, table, ring, want, _ = P.plan(grow, rows, ring, state, table, self.page, n)
        self.book = [out, ring, left, table]
        assert np.array_equal(slots.cpu().numpy(), want)
        return slots

    def store(self, k, v, slots):
        F.flowmm_cache_store(self.p(k.shape[2]), k, v, slots, *self.pool, self.ws)
        for i, x in enumerate((k, v)):
            self.mirror[i], self.mirror[2 + i] = P.store(x.float().cpu().numpy(), slots.cpu().numpy(), self.mirror[i], self.mirror[2 + i])

    def attend(self, q):
        out = torch.empty(q.shape, device="cuda")
        F.flowmm_cache_attention(self.p(), q, *self.pool, self.table, self.rows, out, self.ws)
        assert F.flowmm_last_device_status(self.ws) == 0
        rows, _, _, table = self.book
        want, size, logits = P.attention(q.float().cpu().numpy(), *self.mirror, table, rows)
        for u, n in enumerate(rows):
            assert (np.abs(out[u].cpu().numpy() - want[u]) <= T.attention_bound(size[u], logits[u], int(n), q.shape[2])).all(), u
        return out


def test_compress_store_decode_load_and_recompress():
    """The whole use: a layer is compressed and stored, decoded over for some steps while sequences end, read back, re-compressed and stored."""
    rng = np.random.default_rng(21)
    U, Hq, H, D, L, B, W = 3, 8, 2, 128, 512, 60, 16
    gen = lambda *s: T.dev(rng.standard_normal(s).astype(np.float32), F.BF16)
    fp = F.Params(U, Hq, H, D, L, W, B, theta=0.25, tau=8.0, tau_mode=F.TAU_REL)
    q, k, v = gen(U, Hq, W, D), gen(U, H, L, D), gen(U, H, L, D)
    m = T.dev(rng.integers(0, 2, (U, L)).astype(np.uint8))
    c = F.compress_layer_alloc(fp, q, k, v, m)
    s = Server(U, Hq, H, D, 16, 30, 8, F.BF16, rng)
    s.store(c["k_out"], c["v_out"], s.plan(np.full(U, B, np.int32), B))
    s.attend(gen(U, Hq, D))
    for step in range(20):
        grow = np.ones(U, np.int32)
        if step == 9:
            grow[1] = -int(s.book[0][1])                            # the sequence ends, ...
        if step > 9:
            grow[1] = 0                                             # ... and its unit stays empty
        s.store(gen(U, H, 1, D), 4 * gen(U, H, 1, D), s.plan(grow, 1))
        s.attend(gen(U, Hq, D))
    assert s.book[0].tolist() == [B + 20, 0, B + 20]
    n = B + 20
    dense = [torch.zeros((U, H, n, D), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    F.flowmm_cache_load(s.p(n), *s.pool, s.table, s.rows, *dense, s.ws)
    assert np.array_equal(dense[0][0].float().cpu().numpy(), P.load(s.mirror[0], s.mirror[2], s.book[3][0], n))
    rp = F.Params(U, Hq, H, D, n, W, B, theta=0.25, tau=8.0, tau_mode=F.TAU_REL)
    ws = torch.zeros(F.flowmm_recompress_workspace_bytes(rp), dtype=torch.uint8, device="cuda")
    mod = torch.zeros((U, H, n), dtype=torch.uint8, device="cuda")
    ko, vo = (torch.empty((U, H, B, D), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    F.flowmm_recompress(rp, gen(U, Hq, W, D), *dense, mod, ko, vo, torch.empty((U, H, B), dtype=torch.uint8, device="cuda"), ws)
    assert F.flowmm_last_device_status(ws) == 0
    s.plan(-s.book[0], 1)
    s.store(ko, vo, s.plan(np.array([B, 0, B], np.int32), B))
    s.attend(gen(U, Hq, D))


@pytest.mark.parametrize("path", [F.PATH_AUTO, F.PATH_SIMT])
def test_captured_step_with_changing_lengths(path):
    """A decode step captured once (plan, store, attention, lengths carried over) and replayed while lengths grow over pages and tiles;
    a second graph on the same workspace in between."""
    rng = np.random.default_rng(30)
    U, Hq, H, D, page, wide = 3, 8, 2, 128, 16, 20
    s = Server(U, Hq, H, D, page, 60, wide, F.BF16, rng)
    gen = lambda *shape: T.dev(rng.standard_normal(shape).astype(np.float32), F.BF16)
    k0 = gen(U, H, 125, D)
    s.store(k0, k0, s.plan(np.array([125, 0, 7], np.int32), 125))
    k, v, q = gen(U, H, 1, D), gen(U, H, 1, D), gen(U, Hq, D)
    grow, slots, out = torch.ones(U, dtype=torch.int32, device="cuda"), torch.empty((U, 1), dtype=torch.int32, device="cuda"), torch.empty((U, Hq, D), device="cuda")
    p = s.p()
    p.path = path
    rows, state = s.rows.clone(), s.state.clone()
    rows_new, state_new = torch.empty_like(rows), torch.empty_like(state)

    def step():
        F.flowmm_cache_plan(p, grow, rows, rows_new, s.ring, state, state_new, s.table, slots, s.ws)
        F.flowmm_cache_store(p, k, v, slots, *s.pool, s.ws)
        F.flowmm_cache_attention(p, q, *s.pool, s.table, rows_new, out, s.ws)
        rows.copy_(rows_new)
        state.copy_(state_new)

    side = torch.cuda.Stream()
    graphs = []
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                step()
            graphs.append(g)
    torch.cuda.current_stream().wait_stream(side)
    for i in range(8):
        k.copy_(gen(U, H, 1, D)), v.copy_(gen(U, H, 1, D)), q.copy_(gen(U, Hq, D))
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        r, ring, st, table = s.book
        r, st, table, ring, want, _ = P.plan(np.ones(U, np.int32), r, ring, st, table, page, 1)
        s.book = [r, ring, st, table]
        for j, x in enumerate((k, v)):
            s.mirror[j], s.mirror[2 + j] = P.store(x.float().cpu().numpy(), want, s.mirror[j], s.mirror[2 + j])
        ref, size, logits = P.attention(q.float().cpu().numpy(), *s.mirror, table, r)
        assert np.array_equal(rows.cpu().numpy(), r) and np.array_equal(slots.cpu().numpy(), want)
        for u in range(U):
            assert (np.abs(out[u].cpu().numpy() - ref[u]) <= T.attention_bound(size[u], logits[u], int(r[u]), D)).all(), (i, u)
    assert F.flowmm_last_device_status(s.ws) == 0


def test_graphs_of_cut_heads_share_a_workspace():
    """Two captured calls whose heads are cut, of different shapes, on one workspace, replayed in turn with eager calls and other lengths between."""
    rng = np.random.default_rng(33)
    for path in (F.PATH_AUTO, F.PATH_SIMT):
        cases = []
        for U, Hq, H, most in ((2, 16, 2, 9000), (40, 14, 14, 3000)):
            rows = rng.integers(1, most, U)
            p = T.params(U, Hq, H, 128, 64, 1, 1, path=path)
            _, q, arrays = _check(p, rng, rows, 64)
            cases.append((p, q, arrays, T.dev(rows.astype(np.int32)), [T.dev(x) for x in arrays[:4]] + [T.dev(np.where(arrays[4] < 1 << 29, arrays[4], 0))], T.dev(q, F.BF16),
                          torch.empty((U, Hq, 128), device="cuda"), rows))
        ws = torch.full((max(F.flowmm_cache_workspace_bytes(c[0]) for c in cases),), 255, dtype=torch.uint8, device="cuda")
        ws[:256] = 0
        side, graphs = torch.cuda.Stream(), []
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for p, _, _, rows_d, d, qd, out, _ in cases:
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g, stream=side):
                    F.flowmm_cache_attention(p, qd, *d, rows_d, out, ws)
                graphs.append(g)
        torch.cuda.current_stream().wait_stream(side)
        for step in range(6):
            i = step % 2
            p, q, (ck, cv, ks, vs, table), rows_d, d, qd, out, most = cases[i]
            rows = most if step < 2 else rng.integers(0, most + 1)
            rows_d.copy_(T.dev(rows.astype(np.int32)))
            graphs[i].replay()
            if step % 3 == 0:
                F.flowmm_cache_attention(p, qd, *d, rows_d, torch.empty_like(out), ws)
            assert F.flowmm_last_device_status(ws) == 0
            want, size, logits = P.attention(q, P.E4M3[ck], P.E4M3[cv], ks, vs, table, rows)
            for u, n in enumerate(rows):
                assert (np.abs(out[u].cpu().numpy() - want[u]) <= T.attention_bound(size[u], logits[u], int(n), 128)).all(), (step, u)


def test_profile_names_the_kernels():
    rng = np.random.default_rng(1)
    p = T.params(2, 8, 2, 128, 64, 1, 1)
    F.flowmm_profile_enable(True)
    try:
        _check(p, rng, np.array([5000, 70]), 64)
        assert F.flowmm_last_launch_count() == 2
        assert [name for name, ms in F.flowmm_profile_read()] == ["cache_attention_tc", "cache_join"]
    finally:
        F.flowmm_profile_enable(False)


def test_two_streams_with_workspaces_of_their_own():
    rng = np.random.default_rng(31)
    rows = rng.integers(1, 3000, 6)
    p = T.params(6, 8, 2, 128, 64, 1, 1)
    first, q, (ck, cv, ks, vs, table) = _check(p, rng, rows, 64)
    d = [T.dev(x) for x in (ck, cv, ks, vs, table, rows.astype(np.int32))]
    qd = T.dev(q, F.BF16)
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [F.alloc_cache_workspace(p) for _ in streams]
    outs = [[torch.empty((6, 8, 128), device="cuda") for _ in range(20)] for _ in streams]
    torch.cuda.synchronize()
    for i in range(20):
        for st, ws, o in zip(streams, spaces, outs):
            with torch.cuda.stream(st):
                F.flowmm_cache_attention(p, qd, *d, o[i], ws)
    torch.cuda.synchronize()
    for o in outs:
        for t in o:
            assert np.array_equal(t.cpu().numpy().astype(np.float64), first)


def test_binding_refuses_wrong_tensors():
    p = T.params(2, 4, 2, 128, 64, 10, 4, 8)
    ws = F.alloc_cache_workspace(p)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    pool = [torch.zeros((10, 2, 64, 128), dtype=torch.uint8, device="cuda") for _ in "kv"] + [torch.ones((10, 2), device="cuda") for _ in "kv"]
    q, out = torch.zeros((2, 4, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 4, 128), device="cuda")
    k = torch.zeros((2, 2, 8, 128), dtype=torch.bfloat16, device="cuda")
    call = lambda **kw: F.flowmm_cache_attention(*[{**dict(p=p, q=q, a=pool[0], b=pool[1], c=pool[2], d=pool[3], t=i32(2, 4), r=i32(2), o=out, w=ws), **kw}[x] for x in "p q a b c d t r o w".split()])
    call()
    assert (out == 0).all()
    for bad in (dict(q=q.float()), dict(q=q[:, :, :64]), dict(a=pool[0][:9]), dict(c=pool[2].double()), dict(t=i32(2, 5)), dict(r=i32(2).long()), dict(r=i32(3)),
                dict(o=out.bfloat16()), dict(q=torch.zeros((4, 2, 128), dtype=torch.bfloat16, device="cuda").transpose(0, 1)), dict(w=ws.view(torch.int32)),
                dict(r=torch.zeros(2, dtype=torch.int32))):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(ValueError):
        F.flowmm_cache_store(p, k.transpose(2, 3), k, i32(2, 8), *pool, ws)
    with pytest.raises(ValueError):
        F.flowmm_cache_store(p, k, k[:, :, :7], i32(2, 8), *pool, ws)
    with pytest.raises(F.FlowmmError):
        F.flowmm_cache_store(p, k, k, i32(2, 8), *pool, ws[:255])
    fp8 = [t.view(torch.float8_e4m3fn) for t in pool[:2]] + pool[2:]
    F.flowmm_cache_store(p, k, k, torch.full((2, 8), -1, dtype=torch.int32, device="cuda"), *fp8, ws)
    assert F.flowmm_last_device_status(ws) == 0


@pytest.mark.parametrize("dtype", [F.F32, F.BF16])
@pytest.mark.parametrize("D,page,n", [(64, 16, 40), (64, 128, 300), (128, 32, 9), (128, 32, 70), (128, 64, 130), (128, 128, 129)])
def test_a_row_without_a_place_between_rows_is_reported(D, page, n, dtype):
    """A slot of -1 with a good one behind it, wherever in its page: reported; other units' pages are stored, the unit's other rows are where they were to go."""
    rng = np.random.default_rng(page + n + D)
    for held in (0, 5):
        pages = P.pages(held + n, page)
        x = T.dev(rng.standard_normal((2, 2, n, D)).astype(np.float32), dtype)
        p = T.params(2, 2, 2, D, page, 2 * pages, pages, n, dtype)
        codes, scale = rng.integers(0, 256, (2 * pages, 2, page, D)).astype(np.uint8), np.ones((2 * pages, 2), np.float32)
        good = held + np.stack([np.arange(n), pages * page + np.arange(n)]).astype(np.int32)
        want, status = _store(p, x, x, good, codes, codes, scale, scale)
        assert status == 0
        # an inner place, several, the last place of a page, the last but one row, a whole page and more
        for t0, t1 in ((1, 2), (2, 5), (page - held - 1, page - held), (n - 2, n - 1), (page - held, min(n - 1, 2 * page - held)), (1, n - 1)):
            if not 0 < t0 < t1 < n:
                continue
            slots = good.copy()
            slots[0, t0:t1] = -1
            got, status = _store(p, x, x, slots, codes, codes, scale, scale)
            assert status == 10, (held, t0, t1)
            assert all(np.array_equal(a[pages:], b[pages:]) for a, b in zip(got, want)), (held, t0, t1)
            left = np.zeros((pages, page), bool)                    # places in the unit's pages that no row goes to: (page, place)
            left.reshape(-1)[np.setdiff1d(np.arange(pages * page), slots[0])] = True
            left[:, :held] &= np.arange(pages)[:, None] > 0         # (rows held before may be rescaled)
            assert np.array_equal(np.moveaxis(got[0][:pages], 2, 1)[left], np.moveaxis(codes[:pages], 2, 1)[left]), (held, t0, t1)
        slots = good.copy()
        slots[0, n - 1:] = -1                                       # (nothing behind it: no fault)
        assert _store(p, x, x, slots, codes, codes, scale, scale)[1] == 0


def test_units_of_two_lengths_are_recompressed_group_by_group():
    """Compressed to two budgets, grown, read back by units of one length (rows of the block table and of the lengths), compressed again with the rows' modalities that
    the program has kept: what the same rows give that never were in pages."""
    rng = np.random.default_rng(22)
    U, Hq, H, D, L, W, new = 4, 8, 2, 128, 512, 16, 9
    budgets, groups = (60, 44), ([0, 2], [1, 3])
    gen = lambda *shape: T.dev(rng.standard_normal(shape).astype(np.float32), F.BF16)
    s = Server(U, Hq, H, D, 16, 40, 8, F.BF16, rng)
    grow, k, v = np.zeros(U, np.int32), torch.zeros((U, H, max(budgets), D), dtype=torch.bfloat16, device="cuda"), None
    v, kept = torch.zeros_like(k), {}
    for B, units in zip(budgets, groups):
        fp = F.Params(2, Hq, H, D, L, W, B, theta=0.25, tau=8.0, tau_mode=F.TAU_REL)
        modality = T.dev(rng.integers(0, 2, (2, L)).astype(np.uint8))
        c = F.compress_layer_alloc(fp, gen(2, Hq, W, D), gen(2, H, L, D), gen(2, H, L, D), modality)
        k[units, :, :B], v[units, :, :B], grow[units] = c["k_out"], c["v_out"], B
        kept[B] = torch.cat([modality[:, None].expand(2, H, L).gather(2, c["retained"].long()), torch.zeros((2, H, new), dtype=torch.uint8, device="cuda")], 2)
    s.store(k, v, s.plan(grow, max(budgets)))
    k, v = gen(U, H, new, D), gen(U, H, new, D)
    s.store(k, v, s.plan(np.full(U, new, np.int32), new))
    for B, units in zip(budgets, groups):
        n = B + new
        p = T.params(2, Hq, H, D, 16, 40, 8, n)
        dense = [torch.zeros((2, H, n, D), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
        F.flowmm_cache_load(p, *s.pool, s.table[units].contiguous(), s.rows[units].contiguous(), *dense, s.ws)
        want = [T.dev(np.stack([P.load(s.mirror[i], s.mirror[2 + i], s.book[3][u], n) for u in units]).astype(np.float32), F.BF16) for i in range(2)]
        assert all(torch.equal(a, b) for a, b in zip(dense, want))
        rp = F.Params(2, Hq, H, D, n, W, 40, theta=0.25, tau=8.0, tau_mode=F.TAU_REL)
        ws = torch.zeros(F.flowmm_recompress_workspace_bytes(rp), dtype=torch.uint8, device="cuda")
        q, outs = gen(2, Hq, W, D), []
        for x in (dense, want):
            o = [torch.empty((2, H, 40, D), dtype=torch.bfloat16, device="cuda") for _ in "kv"] + [torch.empty((2, H, 40), dtype=torch.uint8, device="cuda")]
            F.flowmm_recompress(rp, q, *x, kept[B], *o, ws)
            outs.append(o)
        assert F.flowmm_last_device_status(ws) == 0 and all(torch.equal(a, b) for a, b in zip(*outs))
        assert 0 < int(outs[0][2].sum()) < outs[0][2].numel()


@pytest.mark.parametrize("D,page,dtype", [(64, 16, F.F32), (128, 128, F.BF16)])
def test_every_row_without_a_place_is_looked_at(D, page, dtype):
    """Many rows of many units: one hole at any place is found, and none where there is none."""
    rng = np.random.default_rng(page)
    U, n = 3, 1100
    pages = P.pages(n, page)
    x = T.dev(rng.standard_normal((U, 1, n, D)).astype(np.float32), dtype)
    p = T.params(U, 1, 1, D, page, U * pages, pages, n, dtype)
    pool = [torch.zeros((U * pages, 1, page, D), dtype=torch.uint8, device="cuda") for _ in "kv"] + [torch.ones((U * pages, 1), device="cuda") for _ in "kv"]
    good = (np.arange(U)[:, None] * pages * page + np.arange(n)).astype(np.int32)
    ws = F.alloc_cache_workspace(p)
    for u in range(U):
        for t in (None, 0, 1, 510, 511, 512, 513, 1022, 1023, 1024, 1025, n - 2, n - 1):
            slots = good.copy()
            if t is not None:
                slots[u, t] = -1
            F.flowmm_cache_store(p, x, x, T.dev(slots), *pool, ws)
            assert F.flowmm_last_device_status(ws) == (0 if t in (None, n - 1) else 10), (u, t)
