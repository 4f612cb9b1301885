"""The paged cache without a GPU: its oracle against what can be worked out by hand, and the calls that are refused."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

from oracle import paged_cache as P
from paper_2511_05534_b200 import binding as F
from paper_2511_05534_b200 import build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return F.load()


def test_e4m3_values_and_rounding():
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(codes, P.E4M3, equal_nan=True)
    x = np.concatenate([np.linspace(-448, 448, 20011), np.ldexp(np.random.default_rng(1).standard_normal(5000), np.random.default_rng(2).integers(-14, 4, 5000)),
                        (P.E4M3[:126] + P.E4M3[1:127]) / 2])               # (the midpoints: ties)
    x = x.astype(np.float32).astype(np.float64)
    assert np.array_equal(P.to_e4m3(x), torch.from_numpy(x).float().to(torch.float8_e4m3fn).double().numpy())
    assert np.isnan(P.to_e4m3(np.array([np.inf, -np.inf, np.nan]))).all()


def test_scale_is_the_smallest_power_of_two():
    for size in (1e-35, 2.0 ** -88 * 1.75, 448.0, 448.0001, 1.0, 3.4e38, 1.75, 1.7500001, 0.1):
        s = P.scale_for(size)
        assert 448 * s >= size and (s == 2.0 ** P.LOWEST or 448 * s / 2 < size), size
    assert P.scale_for(0.0) == 2.0 ** P.LOWEST


def test_plan_by_hand():
    ring, state = np.array([7, 0, 0, 5, 6], np.int32), np.array([3, 3], np.int32)       # free: 5, 6, 7
    table = np.array([[1, 2, 9], [3, 4, 9], [9, 9, 9]], np.int32)
    rows, grow = np.array([20, 17, 0], np.int32), np.array([13, -17, 16], np.int32)
    out, left, t, r, slots, refused = P.plan(grow, rows, ring, state, table, 16, 16)
    assert out.tolist() == [33, 0, 16] and not refused
    assert t.tolist() == [[1, 2, 5], [3, 4, 9], [6, 9, 9]]
    assert left.tolist() == [0, 3] and [int(r[i % 5]) for i in (0, 1, 2)] == [7, 3, 4]
    assert slots[0].tolist() == [2 * 16 + 4 + i for i in range(12)] + [5 * 16] + [-1] * 3
    assert (slots[1] == -1).all() and slots[2].tolist() == [6 * 16 + i for i in range(16)]
    refused = P.plan(np.array([28, 1, 1], np.int32), rows, ring, state, table, 16, 16)[5]      # more slots than there are
    assert refused == [0]


def _call(lib, name, p, args, ws=1 << 20, ws_bytes=1 << 40):
    return getattr(lib, name)(ctypes.byref(p), *args, ws, ws_bytes, None)


GOOD = dict(n_units=2, n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=64, n_pages=10, max_pages=4, n_rows=8)
POINTERS = {"flowmm_cache_plan": 8, "flowmm_cache_store": 7, "flowmm_cache_load": 8, "flowmm_cache_attention": 8}
OPTIONAL = {("flowmm_cache_plan", 7)}


def _args(name):
    return [(i + 1) << 20 for i in range(POINTERS[name])]


@pytest.mark.parametrize("name", sorted(POINTERS))
def test_refusals(lib, name):
    """Every call here is refused by a check on the host, before the library looks for a device."""
    for change, code in [(dict(n_units=0), 2), (dict(n_q_heads=7), 2), (dict(n_q_heads=18), 2), (dict(n_kv_heads=0), 2), (dict(head_dim=96), 2),
                         (dict(page_size=48), 2), (dict(page_size=0), 2), (dict(n_pages=0), 2), (dict(max_pages=0), 2), (dict(n_rows=-1), 2),
                         (dict(n_pages=1 << 26), 2), (dict(max_pages=1 << 25), 2), (dict(max_pages=(1 << 24) + 1), 2), (dict(n_units=1, n_rows=(1 << 30) + 1), 2), (dict(n_units=1 << 12, n_rows=1 << 19), 2),
                         (dict(n_units=1 << 22), 2), (dict(dtype=2), 4), (dict(softmax_scale=-1.0), 2), (dict(softmax_scale=float("nan")), 2), (dict(path=3), 2)]:
        p = F.CacheParams(**{**GOOD, **change}).c()
        assert _call(lib, name, p, _args(name)) == code, change
        n = ctypes.c_size_t(0)
        assert lib.flowmm_cache_workspace_bytes(ctypes.byref(p), ctypes.byref(n)) == code, change
    p = F.CacheParams(**GOOD).c()
    for i in range(POINTERS[name]):
        args = _args(name)
        args[i] = None
        if (name, i) not in OPTIONAL:
            assert _call(lib, name, p, args) == 1, i
    need = F.flowmm_cache_workspace_bytes(F.CacheParams(**GOOD))
    assert _call(lib, name, p, _args(name), ws=None) == 1
    assert _call(lib, name, p, _args(name), ws=(1 << 20) + 128) == 6
    assert _call(lib, name, p, _args(name), ws_bytes=need - 1) == 5
    assert getattr(lib, name)(None, *_args(name), 1 << 20, 1 << 40, None) == 1


def test_refusals_of_alignment_and_aliases(lib):
    p = F.CacheParams(**GOOD)
    wide = {"flowmm_cache_plan": (), "flowmm_cache_store": (0, 1, 3, 4), "flowmm_cache_load": (0, 1, 6, 7), "flowmm_cache_attention": (0, 1, 2)}
    for name, places in wide.items():
        for i in range(POINTERS[name]):
            args = _args(name)
            args[i] += 8 if i in places else 2
            assert _call(lib, name, p.c(), args) == 6, (name, i)
    for name in ("flowmm_cache_store", "flowmm_cache_load"):
        for field in ("k_stride", "v_stride"):
            for i, bad in ((0, 1004), (1, -128), (2, 64)):
                c = p.c()
                getattr(c, field)[i] = bad
                assert _call(lib, name, c, _args(name)) == 6, (name, field, i)
        assert _call(lib, name, F.CacheParams(**{**GOOD, "n_rows": 0}).c(), _args(name)) == 2
    for same in ((1, 2), (0, 2), (4, 5)):               # rows_out on rows and on grow, free_state_out on free_state
        args = _args("flowmm_cache_plan")
        args[same[1]] = args[same[0]]
        assert _call(lib, "flowmm_cache_plan", p.c(), args) == 2
    assert _call(lib, "flowmm_cache_plan", F.CacheParams(**{**GOOD, "n_rows": 0}).c(), _args("flowmm_cache_plan")) == 2
    assert lib.flowmm_cache_workspace_bytes(ctypes.byref(p.c()), None) == 1


def test_struct_matches_header():
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "flowmm.h")).read()
    end = header.index("} flowmm_cache_params;")
    body = header[header.rindex("typedef struct {", 0, end):end]
    names = [n.strip().split("[")[0] for group in re.findall(r"(?:int32_t|float|int64_t)\s+([^;]+);", body) for n in group.split(",")]
    assert names == [f[0] for f in F._CCacheParams._fields_]
    assert F.status_string(11) != "unknown status" and F.status_string(12) == "unknown status"


def test_binding_looks_at_shapes_and_devices():
    """What the C side cannot see is refused by the binding: host tensors among it."""
    p = F.CacheParams(**GOOD)
    rows = torch.zeros(2, dtype=torch.int32)
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    with pytest.raises(ValueError, match="CUDA"):
        F.flowmm_cache_plan(p, rows, rows, rows.clone(), torch.zeros(10, dtype=torch.int32), rows, rows.clone(), torch.zeros((2, 4), dtype=torch.int32),
                            torch.zeros((2, 8), dtype=torch.int32), ws)


@pytest.mark.parametrize("D,dtype", [(128, F.BF16), (64, F.F32)])
def test_workspace_never_shrinks(lib, D, dtype):
    """A workspace kept for the most units, the widest table and the most rows serves smaller calls."""
    size = lambda U, wide, page, G: F.flowmm_cache_workspace_bytes(F.CacheParams(U, 2 * G, 2, D, page, 100, wide, 1, dtype=dtype))
    for G in (1, 4, 7, 8):
        for U in (1, 3, 40, 300):
            sizes = [size(U, wide, 64, G) for wide in range(1, 700)]
            assert sizes == sorted(sizes)
        for wide in (1, 10, 500):
            sizes = [size(U, wide, 16, G) for U in range(1, 700)]
            assert sizes == sorted(sizes)
