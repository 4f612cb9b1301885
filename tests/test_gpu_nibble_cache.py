"""The paged 4-bit cache on the GPU against its 64-bit oracle: bytes and dense rows are equal, attention within the bound that nibble_util derives."""
import numpy as np
import pytest
import torch

from oracle import nibble_cache as N
from oracle import rotary as R
from paper_2511_05534_b200 import binding as F

import nibble_util as T

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -8


def rounded(x, dtype):
    """float64 rows as the call sees them."""
    return torch.from_numpy(np.ascontiguousarray(x)).to(F.torch_dtype(dtype)).double().numpy()


def rows_like_a_cache(rng, shape, dtype):
    x = rng.standard_normal(shape) * np.exp2(rng.integers(-6, 7, shape[:-1] + (1,)))
    x[..., ::37] *= 4
    return rounded(x, dtype)


# ---- store ---------------------------------------------------------------------------------------

def _store(p, x, slots, pool, strided=False):
    ws = F.alloc_nibble_workspace(p)
    rows = []
    for t in x:
        t = T.dev(t, p.dtype)
        if strided:                                            # [units, rows, heads, head_dim] in memory, with room between
            wide = torch.full((t.shape[0], t.shape[2], t.shape[1], t.shape[3] + 8), float("nan"), device="cuda", dtype=t.dtype)
            wide[..., :t.shape[3]] = t.transpose(1, 2)
            t = wide[..., :t.shape[3]].transpose(1, 2)
        rows.append(t)
    dev = [T.dev(b) for b in pool]
    F.flowmm_nibble_store(p, *rows, T.dev(slots), *dev, ws)
    return [b.cpu().numpy() for b in dev], F.flowmm_last_device_status(ws)


def _empty(rng, n_pages, H, page, D):
    return [rng.integers(0, 256, (n_pages, H, page, D // w)).astype(np.uint8) for w in (2, 2, 16, 16)]


def _check_store(p, x, slots, pool, got):
    for i, name in enumerate("kv"):
        codes, scale = N.store(x[i], slots, pool[i], pool[2 + i])
        assert np.array_equal(scale, got[2 + i]), name
        assert np.array_equal(codes, got[i]), name


@pytest.mark.parametrize("dtype", [F.BF16, F.F32])
@pytest.mark.parametrize("U,H,D,page,n_rows,strided", [(1, 1, 128, 16, 1, False), (4, 8, 128, 64, 1, True), (1, 4, 64, 16, 48, False), (3, 5, 128, 32, 77, True),
                                                       (2, 2, 64, 128, 301, False), (7, 3, 64, 64, 9, True), (2, 8, 128, 128, 1000, False)])
def test_store_equals_oracle(dtype, U, H, D, page, n_rows, strided):
    """Rows to places in any order, some to none; all other places keep their bytes."""
    rng = np.random.default_rng(U * 1000 + n_rows + D)
    n_pages = N.pages(U * n_rows, page) + 3
    slots = rng.permutation(n_pages * page)[:U * n_rows].reshape(U, n_rows).astype(np.int32)
    if n_rows > 1:
        slots[rng.random(slots.shape) < 0.1] = -1
    x = [rows_like_a_cache(rng, (U, H, n_rows, D), dtype) for _ in "kv"]
    pool = _empty(rng, n_pages, H, page, D)
    got, status = _store(T.params(U, H, H, D, page, n_pages, 4, n_rows, dtype=dtype), x, slots, pool, strided)
    assert status == 0
    _check_store(None, x, slots, pool, got)


@pytest.mark.parametrize("dtype", [F.BF16, F.F32])
def test_store_of_odd_numbers(dtype):
    """Ties of codes and scales, neighbours of ties, zeros of both signs, the smallest and largest numbers, NaN and infinities."""
    rng = np.random.default_rng(5)
    n, D = 512, 128
    x = np.zeros((1, 1, n, D))
    border = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    for t in range(n):
        s = N.SCALE[rng.integers(N.LEAST, N.MOST + 1, 8)]
        g = rng.choice(border, (8, 16)) * rng.choice([-1, 1], (8, 16))
        g[:, 0] = 6.0 * rng.choice([-1, 1], 8)                                  # so that s is the scale
        near = 1 + rng.integers(-1, 2, (8, 16)) * (2.0 ** -7 if dtype == F.BF16 else 2.0 ** -23)
        near[:, 0] = 1.0
        x[0, 0, t] = (s[:, None] * g * (near if t % 2 else 1.0)).ravel()
    ties = 6 * (N.SCALE[N.LEAST:N.MOST] + N.SCALE[N.LEAST + 1:N.MOST + 1]) / 2     # sizes whose sixth lies between two scales
    for i, size in enumerate(ties[:200]):
        x[0, 0, i, 16] = size * (1 + (i % 3 - 1) * (2.0 ** -7 if dtype == F.BF16 else 2.0 ** -23))
        x[0, 0, i, 17:32] = 0.0
    x[0, 0, 300, :16], x[0, 0, 300, 16:32], x[0, 0, 300, 32:48] = 0.0, -0.0, 1e-30
    x[0, 0, 301, :16], x[0, 0, 301, 16:32] = 3e38, -61440.0
    x[0, 0, 301, 32:48] = np.array([1e-38, -1e-38, 2.0 ** -16, -(2.0 ** -15), 0, -0.0, 1e-44, 2.0 ** -17] * 2)
    x[0, 0, 302, 5], x[0, 0, 303, 21], x[0, 0, 304, 40] = np.nan, np.inf, -np.inf
    x = rounded(x, dtype)
    pool = _empty(rng, 9, 1, 64, D)
    slots = rng.permutation(9 * 64)[:n].reshape(1, n).astype(np.int32)
    got, status = _store(T.params(1, 1, 1, D, 64, 9, 9, n, dtype=dtype), [x, x[:, :, ::-1]], slots, pool)
    assert status == 0
    _check_store(None, [x, x[:, :, ::-1]], slots, pool, got)


@pytest.mark.parametrize("bad", [-2, 64 * 6, 1 << 30, -(1 << 31)])
def test_store_reports_bad_slots_and_stores_the_others(bad):
    rng = np.random.default_rng(3)
    slots = np.arange(40, dtype=np.int32).reshape(2, 20)
    slots[1, 7] = bad
    x = [rows_like_a_cache(rng, (2, 2, 20, 128), F.BF16) for _ in "kv"]
    pool = _empty(rng, 6, 2, 64, 128)
    got, status = _store(T.params(2, 2, 2, 128, 64, 6, 3, 20), x, slots, pool)
    assert status == 10
    slots[1, 7] = -1
    _check_store(None, x, slots, pool, got)


# ---- load ----------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F.BF16, F.F32])
@pytest.mark.parametrize("U,H,D,page,n_rows,most", [(1, 1, 128, 16, 1, 1), (5, 4, 128, 64, 640, 640), (3, 2, 64, 32, 100, 300), (4, 3, 64, 128, 333, 200), (2, 8, 128, 16, 65, 77)])
def test_load_equals_oracle(dtype, U, H, D, page, n_rows, most):
    """Every product of a code and a scale, exactly; rows behind the last one are left."""
    rng = np.random.default_rng(U + n_rows + D)
    rows = rng.integers(0, most + 1, U).astype(np.int32)
    rows[0] = most
    table, n_pages = T.random_table(rng, rows, page)
    pool = T.random_pool(rng, n_pages, H, page, D, rows, table, scales=(0, 227))
    pool[2][table[0, 0], 0, 0, 0] = N.NAN
    p = T.params(U, H, H, D, page, n_pages, table.shape[1], n_rows, dtype=dtype)
    ws = F.alloc_nibble_workspace(p)
    out = [torch.full((U, n_rows, H, D + 8), 7.0, device="cuda", dtype=F.torch_dtype(dtype)) for _ in "kv"]
    F.flowmm_nibble_load(p, *map(T.dev, pool), T.dev(table), T.dev(rows), *(o[..., :D].transpose(1, 2) for o in out), ws)
    assert F.flowmm_last_device_status(ws) == 0
    for i in range(2):
        want = np.full((U, n_rows, H, D + 8), 7.0)
        for u in range(U):
            n = min(rows[u], n_rows)
            want[u, :n, :, :D] = N.load(pool[i], pool[2 + i], table[u], rows[u])[:, :n].swapaxes(0, 1)
        assert np.array_equal(out[i].double().cpu().numpy(), want, equal_nan=True)


@pytest.mark.parametrize("call", ["load", "attention"])
@pytest.mark.parametrize("what", ["page", "negative", "rows", "many"])
def test_bad_pages_and_lengths_are_reported(call, what):
    rng = np.random.default_rng(9)
    rows = np.array([50, 60, 0], np.int32)
    table, n_pages = T.random_table(rng, rows, 16)
    pool = T.random_pool(rng, n_pages, 2, 16, 64, rows, table)
    if what in ("page", "negative"):
        table[1, 2] = n_pages if what == "page" else -1
    else:
        rows[1] = -1 if what == "rows" else table.shape[1] * 16 + 1
    table[2] = 0
    p = T.params(3, 4, 2, 64, 16, n_pages, table.shape[1], 64)
    ws = F.alloc_nibble_workspace(p)
    if call == "load":
        out = [torch.zeros((3, 2, 64, 64), device="cuda", dtype=torch.bfloat16) for _ in "kv"]
        F.flowmm_nibble_load(p, *map(T.dev, pool), T.dev(table), T.dev(rows), *out, ws)
        assert np.array_equal(out[0][0, :, :50].double().cpu().numpy(), N.load(pool[0], pool[2], table[0], 50))
        assert F.flowmm_last_device_status(ws) == 10
    else:
        q = rounded(rng.standard_normal((3, 4, 64)), F.BF16)
        table_ok = np.clip(table, 0, n_pages - 1)
        got, status = T.attend(p, q, pool, table, rows, ws)
        assert status == 10
        want, size, logits = N.attention(q, pool, table_ok, np.array([50, 0, 0]))
        assert (np.abs(got - want) <= T.attention_bound(want, size, logits, 50, 64, F.BF16))[[0, 2]].all()


# ---- attention -----------------------------------------------------------------------------------

def _check(rng, U, H, G, D, page, rows, dtype, q=None, pool=None, table=None, **kw):
    rows = np.asarray(rows, np.int32)
    if table is None:
        table, n_pages = T.random_table(rng, rows, page, wide=kw.pop("wide", None))
        pool = T.random_pool(rng, n_pages, H, page, D, rows, table, **({"scales": kw.pop("scales")} if "scales" in kw else {}))
    p = T.params(U, H * G, H, D, page, pool[0].shape[0], table.shape[1], dtype=dtype, **kw)
    q = rounded(rng.standard_normal((U, H * G, D)) if q is None else q, dtype)
    got, status = T.attend(p, q, pool, table, rows)
    assert status == 0
    want, size, logits = N.attention(q, pool, table, rows, kw.get("softmax_scale", 0.0))
    bound = T.attention_bound(want, size, logits, int(rows.max()), D, dtype)
    worst = np.max(np.abs(got - want) / np.maximum(bound, 1e-300))
    assert worst <= 1, worst
    assert (got[rows == 0] == 0).all()
    return got


@pytest.mark.parametrize("dtype", [F.BF16, F.F32])
@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("n", [1, 2, 7, 15, 16, 17, 31, 63, 64, 65, 127, 128, 129, 218, 383, 640, 1025])
def test_attention_at_every_length(dtype, D, n):
    rng = np.random.default_rng(n + D)
    _check(rng, 2, 2, 3, D, 16 << n % 4, [n, max(0, n - 1)], dtype)


@pytest.mark.parametrize("dtype", [F.BF16, F.F32])
@pytest.mark.parametrize("U,H,G,D,page,most", [(1, 4, 7, 128, 64, 218), (4, 4, 1, 64, 16, 192), (8, 32, 1, 128, 32, 640), (64, 8, 8, 128, 64, 300), (3, 1, 8, 128, 128, 5000),
                                               (33, 2, 5, 128, 16, 500), (70, 8, 4, 64, 64, 200), (320, 8, 2, 128, 64, 40), (1, 1, 6, 64, 128, 9000), (600, 1, 1, 64, 16, 70)])
def test_attention_of_ragged_batches(dtype, U, H, G, D, page, most):
    rng = np.random.default_rng(U + most)
    rows = rng.integers(0, most + 1, U)
    rows[0] = most
    if U > 2:
        rows[1], rows[-1] = 0, 0
    _check(rng, U, H, G, D, page, rows, dtype)


@pytest.mark.parametrize("dtype", [F.BF16, F.F32])
@pytest.mark.parametrize("G", range(1, 9))
def test_attention_of_every_group(dtype, G):
    _check(np.random.default_rng(G), 3, 2, G, 128, 32, [90, 33, 200], dtype)


@pytest.mark.parametrize("dtype", [F.BF16, F.F32])
@pytest.mark.parametrize("spare", [1, 40, 5000])
def test_attention_with_room_in_the_table(dtype, spare):
    rng = np.random.default_rng(spare)
    _check(rng, 3, 2, 4, 128, 16, [218, 0, 77], dtype, wide=14 + spare)


@pytest.mark.parametrize("dtype", [F.BF16, F.F32])
@pytest.mark.parametrize("size,scales", [(2.0 ** 20, (96, 140)), (2.0 ** -30, (96, 140)), (1.0, (8, 40)), (1.0, (200, 227)), (2.0 ** 12, (200, 227)), (0.0, (96, 140))])
def test_attention_of_large_and_small_numbers(dtype, size, scales):
    """Logits of 2^20 and more, where one key takes all; scales at both ends."""
    rng = np.random.default_rng(11)
    _check(rng, 2, 2, 4, 128, 64, [300, 129], dtype, q=size * rng.standard_normal((2, 8, 128)), scales=scales)


@pytest.mark.parametrize("dtype", [F.BF16, F.F32])
def test_attention_of_queries_with_elements_far_apart(dtype):
    rng = np.random.default_rng(12)
    q = rng.standard_normal((2, 8, 128)) * 2.0 ** -rng.integers(0, 12, (2, 8, 128))
    _check(rng, 2, 2, 4, 128, 64, [300, 129], dtype, q=q)


@pytest.mark.parametrize("dtype", [F.BF16, F.F32])
@pytest.mark.parametrize("scale", [1.0, 1e-4, 0.3])
def test_attention_with_a_scale(dtype, scale):
    _check(np.random.default_rng(13), 2, 2, 4, 64, 64, [300, 129], dtype, softmax_scale=scale)


@pytest.mark.parametrize("dtype", [F.BF16, F.F32])
@pytest.mark.parametrize("where", ["key", "value", "query"])
def test_nan_stays_with_its_unit(dtype, where):
    """A NaN key or query makes its heads' outputs NaN, a NaN value its 16 channels; other units and heads have none of it."""
    rng = np.random.default_rng(14)
    rows = np.array([100, 200], np.int32)
    table, n_pages = T.random_table(rng, rows, 32)
    pool = T.random_pool(rng, n_pages, 2, 32, 128, rows, table)
    q = rounded(rng.standard_normal((2, 6, 128)), dtype)
    clean = T.attend(T.params(2, 6, 2, 128, 32, n_pages, table.shape[1], dtype=dtype), q, pool, table, rows)[0]
    want = np.zeros((2, 6, 128), bool)
    if where == "key":
        pool[2][table[1, 3], 1, 7, 2] = N.NAN
        want[1, 3:] = True
    elif where == "value":
        pool[3][table[1, 3], 1, 7, 2] = N.NAN
        want[1, 3:, 32:48] = True
    else:
        q[1, 4, 77] = np.nan
        want[1, 4] = True
    got, status = T.attend(T.params(2, 6, 2, 128, 32, n_pages, table.shape[1], dtype=dtype), q, pool, table, rows)
    assert status == 0 and np.array_equal(np.isnan(got), want)
    assert np.array_equal(got[~want], clean[~want])


@pytest.mark.parametrize("dtype", [F.BF16, F.F32])
def test_several_queries_of_a_sequence(dtype):
    """Units that share a row of the block table, each with the rows up to its own token."""
    rng = np.random.default_rng(15)
    one, n_pages = T.random_table(rng, [203], 16)
    pool = T.random_pool(rng, n_pages, 2, 16, 128, [203], one)
    _check(rng, 4, 2, 3, 128, 16, [200, 201, 202, 203], dtype, pool=pool, table=np.repeat(one, 4, 0))


@pytest.mark.parametrize("U,H,G,D,most,dtype", [(5, 2, 8, 128, 3000, F.BF16), (70, 8, 2, 128, 400, F.BF16), (3, 2, 4, 64, 2500, F.F32)])
def test_attention_repeats_bit_by_bit(U, H, G, D, most, dtype):
    """The same call again, in a graph, with a table that has more room, and on a stream of its own: the same bits."""
    rng = np.random.default_rng(U)
    rows = rng.integers(1, most + 1, U).astype(np.int32)
    table, n_pages = T.random_table(rng, rows, 64)
    pool = [T.dev(x) for x in T.random_pool(rng, n_pages, H, 64, D, rows, table)]
    p = T.params(U, H * G, H, D, 64, n_pages, table.shape[1], dtype=dtype)
    q, t, r, ws = T.dev(rounded(rng.standard_normal((U, H * G, D)), dtype), dtype), T.dev(table), T.dev(rows), F.alloc_nibble_workspace(p)
    outs = [torch.empty_like(q) for _ in range(4)]
    F.flowmm_nibble_attention(p, q, *pool, t, r, outs[0], ws)
    F.flowmm_nibble_attention(p, q, *pool, t, r, outs[1], ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        F.flowmm_nibble_attention(p, q, *pool, t, r, outs[2], ws)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    side, ws2 = torch.cuda.Stream(), F.alloc_nibble_workspace(p)
    with torch.cuda.stream(side):
        F.flowmm_nibble_attention(p, q, *pool, t, r, outs[3], ws2)
    side.synchronize()
    assert F.flowmm_last_device_status(ws) == 0 and F.flowmm_last_device_status(ws2) == 0
    assert all(torch.equal(o, outs[0]) for o in outs[1:])


def test_a_graph_follows_the_lengths():
    """One captured call, replayed with other lengths, queries and pages: the lengths are read on the device."""
    rng = np.random.default_rng(21)
    U, H, G, D, page, wide = 6, 2, 4, 128, 16, 40
    n_pages = U * wide
    table = rng.permutation(n_pages).reshape(U, wide).astype(np.int32)
    p = T.params(U, H * G, H, D, page, n_pages, wide)
    full = np.full(U, wide * page)
    pool = T.random_pool(rng, n_pages, H, page, D, full, table)
    dev = [T.dev(x) for x in pool]
    q, r, t, ws = torch.zeros((U, H * G, D), device="cuda", dtype=torch.bfloat16), torch.ones(U, dtype=torch.int32, device="cuda"), T.dev(table), F.alloc_nibble_workspace(p)
    out = torch.empty_like(q)
    F.flowmm_nibble_attention(p, q, *dev, t, r, out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        F.flowmm_nibble_attention(p, q, *dev, t, r, out, ws)
    for _ in range(4):
        rows = rng.integers(0, wide * page + 1, U).astype(np.int32)
        x = rounded(rng.standard_normal((U, H * G, D)), F.BF16)
        q.copy_(T.dev(x, F.BF16))
        r.copy_(T.dev(rows))
        graph.replay()
        assert F.flowmm_last_device_status(ws) == 0
        want, size, logits = N.attention(x, pool, table, rows)
        assert (np.abs(out.double().cpu().numpy() - want) <= T.attention_bound(want, size, logits, int(rows.max()), D, F.BF16)).all()


# ---- all of them together ------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,D", [(F.BF16, 128), (F.F32, 64)])
def test_decode_steps_from_positions_to_outputs(dtype, D):
    """A compressed cache goes into pages; then steps of rotary, plan, store and attention; in the end the rows are read back."""
    rng = np.random.default_rng(31)
    U, H, G, page, kept, steps = 3, 2, 3, 16, 37, 5
    wide, n_pages = 4, 14
    i32 = lambda x: torch.as_tensor(x, dtype=torch.int32, device="cuda")
    start = np.array([500, 90000, 37], np.int32)                      # positions go on behind the prompt, not behind the kept rows
    cache = [rows_like_a_cache(rng, (U, H, kept, D), dtype) for _ in "kv"]
    admit = T.params(U, H * G, H, D, page, n_pages, wide, kept, dtype=dtype)
    step = T.params(U, H * G, H, D, page, n_pages, wide, 1, dtype=dtype)
    ws = F.alloc_nibble_workspace(admit)
    ws_plan = F.alloc_cache_workspace(admit)
    ring, state, table = i32(rng.permutation(n_pages)), [i32([0, n_pages]), i32([0, 0])], torch.zeros((U, wide), dtype=torch.int32, device="cuda")
    rows = [i32([0] * U), i32([0] * U)]
    slots = torch.empty((U, kept), dtype=torch.int32, device="cuda")
    pool = [T.dev(b) for b in _empty(rng, n_pages, H, page, D)]
    F.flowmm_cache_plan(admit, i32([kept] * U), rows[0], rows[1], ring, state[0], state[1], table, slots, ws_plan)
    F.flowmm_nibble_store(admit, *(T.dev(x, dtype) for x in cache), slots, *pool, ws)
    rp = F.RotaryParams(U, H * G, H, D, 1, dtype=dtype, base=1e6, scaling=F.ROTARY_BY_PARTS, factor=4.0, trained=32768, amplitude=1.1)
    phases = F.alloc_rotary_table(rp)
    freq = R.frequencies(D, 1e6, R.BY_PARTS, factor=4.0, trained=32768)
    slots = torch.empty((U, 1), dtype=torch.int32, device="cuda")
    for s in range(steps):
        q, k, v = (rounded(rng.standard_normal((U, n, 1, D)), dtype) for n in (H * G, H, H))
        positions = (start + s).reshape(U, 1, 1)
        dq, dk, dv = (T.dev(x, dtype) for x in (q, k, v))
        F.flowmm_rotary(rp, dq, dk, i32(positions), phases, dq, dk)
        for x, y in ((q, dq), (k, dk)):
            want = R.rotate(x, positions, freq, amplitude=np.float32(1.1).item())
            assert np.allclose(y.double().cpu().numpy(), want, atol=1e-5, rtol=HALF if dtype == F.BF16 else 1e-5)
        rows, state = rows[::-1], state[::-1]
        F.flowmm_cache_plan(step, i32([1] * U), rows[0], rows[1], ring, state[0], state[1], table, slots, ws_plan)
        F.flowmm_nibble_store(step, dk, dv, slots, *pool, ws)
        out = torch.empty((U, H * G, D), device="cuda", dtype=dq.dtype)
        F.flowmm_nibble_attention(step, dq[:, :, 0].contiguous(), *pool, table, rows[1], out, ws)
        assert F.flowmm_last_device_status(ws) == 0 and F.flowmm_last_device_status(ws_plan) == 0
        cache = [np.concatenate([c, n.double().cpu().numpy()], 2) for c, n in zip(cache, (dk, dv))]
        dense = [N.E2M1[c] * np.repeat(N.SCALE[b], 16, -1) for c, b in map(N.quantise, cache)]
        host = [b.cpu().numpy() for b in pool]
        n = np.full(U, kept + s + 1)
        assert np.array_equal(rows[1].cpu().numpy(), n)
        for u in range(U):
            assert all(np.array_equal(N.load(host[i], host[2 + i], table[u].cpu().numpy(), n[u]), dense[i][u]) for i in range(2))
        want, size, logits = N.attention(dq[:, :, 0].double().cpu().numpy(), host, table.cpu().numpy(), n)
        assert (np.abs(out.double().cpu().numpy() - want) <= T.attention_bound(want, size, logits, int(n[0]), D, dtype)).all()
    back = T.params(U, H * G, H, D, page, n_pages, wide, kept + steps, dtype=dtype)
    read = [torch.zeros((U, H, kept + steps, D), device="cuda", dtype=dq.dtype) for _ in "kv"]
    F.flowmm_nibble_load(back, *pool, table, rows[1], *read, ws)
    assert all(np.array_equal(r.double().cpu().numpy(), d) for r, d in zip(read, dense))


@pytest.mark.parametrize("U,H,B", [(2, 2, 100)])
def test_rows_read_back_can_be_compressed_again(U, H, B):
    """What flowmm_nibble_load gives is what flowmm_recompress takes."""
    rng = np.random.default_rng(41)
    D, page, G, keep = 128, 32, 2, 40
    rows = np.full(U, B, np.int32)
    table, n_pages = T.random_table(rng, rows, page)
    pool = [T.dev(x) for x in T.random_pool(rng, n_pages, H, page, D, rows, table)]
    p = T.params(U, H * G, H, D, page, n_pages, table.shape[1], B)
    k, v = (torch.empty((U, H, B, D), device="cuda", dtype=torch.bfloat16) for _ in "kv")
    ws = F.alloc_nibble_workspace(p)
    F.flowmm_nibble_load(p, *pool, T.dev(table), T.dev(rows), k, v, ws)
    fp = F.Params(U, H * G, H, D, B, 8, keep)
    wsr = torch.zeros(F.flowmm_recompress_workspace_bytes(fp), dtype=torch.uint8, device="cuda")
    ko, vo = (torch.empty((U, H, keep, D), device="cuda", dtype=torch.bfloat16) for _ in "kv")
    mo = torch.empty((U, H, keep), dtype=torch.uint8, device="cuda")
    q = T.dev(rng.standard_normal((U, H * G, 8, D)), F.BF16)
    F.flowmm_recompress(fp, q, k, v, torch.zeros((U, H, B), dtype=torch.uint8, device="cuda"), ko, vo, mo, wsr)
    assert F.flowmm_last_device_status(wsr) == 0 and F.flowmm_last_device_status(ws) == 0
    assert torch.isfinite(ko).all() and torch.isfinite(vo).all()


@pytest.mark.parametrize("dtype", [F.BF16, F.F32])
@pytest.mark.parametrize("U,H,most", [(64, 8, 1690), (64, 8, 2048), (37, 8, 64), (64, 5, 700), (40, 9, 1500), (38, 8, 1), (60, 8, 2049), (65, 8, 300),
                                        (128, 4, 900), (160, 3, 500), (161, 3, 100), (148, 4, 64)])
def test_attention_of_two_whole_heads_a_block(dtype, U, H, most):
    """More heads than blocks, twice as many at most, and on both sides of that: lengths that differ, that are all the same, and none."""
    rng = np.random.default_rng(U + most)
    rows = rng.integers(0, most + 1, U)
    rows[rng.integers(0, U, U // 3)] = most
    _check(rng, U, H, 2, 64, 64, rows, dtype, wide=(most + 63) // 64)


@pytest.mark.parametrize("dtype", [F.BF16, F.F32])
@pytest.mark.parametrize("U,H,most", [(320, 8, 100), (200, 4, 512), (200, 4, 513), (700, 1, 64), (75, 8, 512), (1000, 2, 1), (90, 16, 130)])
def test_attention_of_many_short_heads(dtype, U, H, most):
    """More heads than two for a block: whole ones of a line that is cut between heads, of up to eight tiles, and cut ones beyond."""
    rng = np.random.default_rng(U + most)
    rows = rng.integers(0, most + 1, U)
    rows[rng.integers(0, U, U // 3)] = most
    rows[rng.integers(0, U, U // 9)] = 0
    _check(rng, U, H, 2, 64, 16, rows, dtype, wide=(most + 15) // 16)


@pytest.mark.parametrize("dtype", [F.BF16, F.F32])
@pytest.mark.parametrize("U,H,wide", [(3, 2, 4), (3, 2, 100), (64, 8, 20), (400, 2, 3), (400, 2, 40)])
def test_attention_of_units_without_rows(dtype, U, H, wide):
    """No unit has any, and one has."""
    rng = np.random.default_rng(U + wide)
    for some in (0, 1):
        rows = np.zeros(U, np.int32)
        rows[U - 1] = some * wide * 64
        got = _check(rng, U, H, 3, 128, 64, rows, dtype, wide=wide)
        assert (got[:U - 1] == 0).all() and (got[U - 1] != 0).any() == bool(some)


@pytest.mark.parametrize("dtype", [F.BF16, F.F32])
def test_attention_over_the_smallest_scales(dtype):
    """Scales that no store writes: the steps below fp16's least normal number, and zero."""
    rng = np.random.default_rng(51)
    _check(rng, 2, 2, 4, 128, 64, [300, 129], dtype, scales=(0, 12), q=2.0 ** 14 * rng.standard_normal((2, 8, 128)))


@pytest.mark.parametrize("dtype", [F.BF16, F.F32])
def test_pools_beyond_32_bits(dtype):
    """Pages whose bytes lie more than 2^32 behind the pool's first ones: stored, read back and attended to."""
    rng = np.random.default_rng(61)
    U, H, D, page, n, n_pages = 2, 8, 128, 128, 300, 70000
    table = (n_pages - 1 - rng.permutation(6)).reshape(U, 3).astype(np.int32)
    table[0, 0] = 1
    slots = np.stack([table[u, np.arange(n) // page] * page + np.arange(n) % page for u in range(U)]).astype(np.int32)
    x = [rows_like_a_cache(rng, (U, H, n, D), dtype) for _ in "kv"]
    p = T.params(U, H, H, D, page, n_pages, 3, n, dtype=dtype)
    pool = [torch.empty((n_pages, H, page, D // w), dtype=torch.uint8, device="cuda") for w in (2, 2, 16, 16)]
    assert pool[0].numel() > 1 << 32
    ws, t, r = F.alloc_nibble_workspace(p), T.dev(table), T.dev(np.full(U, n, np.int32))
    F.flowmm_nibble_store(p, *(T.dev(v, dtype) for v in x), T.dev(slots), *pool, ws)
    back = [torch.empty((U, H, n, D), device="cuda", dtype=F.torch_dtype(dtype)) for _ in "kv"]
    F.flowmm_nibble_load(p, *pool, t, r, *back, ws)
    q = rounded(rng.standard_normal((U, H, D)), dtype)
    out = torch.empty((U, H, D), device="cuda", dtype=F.torch_dtype(dtype))
    F.flowmm_nibble_attention(p, T.dev(q, dtype), *pool, t, r, out, ws)
    assert F.flowmm_last_device_status(ws) == 0
    low = [b[torch.from_numpy(table.ravel()).long().cuda()].cpu().numpy() for b in pool]
    near = np.arange(6, dtype=np.int32).reshape(U, 3)
    for i in range(2):
        codes, scale = N.quantise(x[i])
        assert np.array_equal(back[i].double().cpu().numpy(), N.E2M1[codes] * np.repeat(N.SCALE[scale], 16, -1))
    want, size, logits = N.attention(q, low, near, np.full(U, n))
    assert (np.abs(out.double().cpu().numpy() - want) <= T.attention_bound(want, size, logits, n, D, dtype)).all()


def test_two_calls_at_once():
    """Two streams, a workspace each, the same pages: each gives what it gives alone; a call in between on a third changes nothing."""
    rng = np.random.default_rng(71)
    U, H, G, D, page = 6, 4, 8, 128, 32
    rows = rng.integers(1, 4000, U).astype(np.int32)
    table, n_pages = T.random_table(rng, rows, page)
    pool = [T.dev(x) for x in T.random_pool(rng, n_pages, H, page, D, rows, table)]
    p = T.params(U, H * G, H, D, page, n_pages, table.shape[1])
    t, r = T.dev(table), T.dev(rows)
    q = [T.dev(rng.standard_normal((U, H * G, D)), F.BF16) for _ in range(3)]
    ws = [F.alloc_nibble_workspace(p) for _ in q]
    alone = [torch.empty_like(x) for x in q]
    for x, o, w in zip(q, alone, ws):
        F.flowmm_nibble_attention(p, x, *pool, t, r, o, w)
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in q], [torch.empty_like(x) for x in q]
    for _ in range(20):
        for x, o, w, s in zip(q, outs, ws, streams):
            with torch.cuda.stream(s):
                F.flowmm_nibble_attention(p, x, *pool, t, r, o, w)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(alone, outs))
    assert [F.flowmm_last_device_status(w) for w in ws] == [0, 0, 0]


def test_two_graphs_share_a_workspace():
    """Calls of different units, lengths and ways of sharing the work out, replayed in turn on one workspace."""
    rng = np.random.default_rng(81)
    shapes = [(2, 8, 8, 6000), (64, 8, 4, 1500), (3, 4, 7, 200), (200, 4, 2, 300), (90, 8, 2, 2500)]
    calls = []
    for U, H, G, most in shapes:
        rows = rng.integers(0, most + 1, U).astype(np.int32)
        table, n_pages = T.random_table(rng, rows, 64, wide=(most + 63) // 64)
        pool = [T.dev(x) for x in T.random_pool(rng, n_pages, H, 64, 64, rows, table)]
        p = T.params(U, H * G, H, 64, 64, n_pages, table.shape[1])
        q = T.dev(rng.standard_normal((U, H * G, 64)), F.BF16)
        calls.append((p, q, pool, T.dev(table), T.dev(rows), torch.empty_like(q)))
    ws = max((F.alloc_nibble_workspace(c[0]) for c in calls), key=torch.Tensor.numel)
    graphs, want = [], []
    for p, q, pool, t, r, out in calls:
        F.flowmm_nibble_attention(p, q, *pool, t, r, out, F.alloc_nibble_workspace(p))
        torch.cuda.synchronize()
        want.append(out.clone())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            F.flowmm_nibble_attention(p, q, *pool, t, r, out, ws)
        graphs.append(graph)
    for order in (range(5), (4, 0, 3, 0, 1, 2), (2, 1, 0, 4, 3)):
        for c in calls:
            c[5].fill_(7.0)
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        assert F.flowmm_last_device_status(ws) == 0
        assert all(torch.equal(calls[i][5], want[i]) for i in order)
