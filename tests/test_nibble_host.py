"""The paged 4-bit cache and rotary positions without a GPU: their oracles against what can be worked out by hand, and the calls that are refused."""
import ctypes
import math
import os
import re

import numpy as np
import pytest
import torch

from oracle import nibble_cache as N
from oracle import rotary as R
from paper_2511_05534_b200 import binding as F
from paper_2511_05534_b200 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    build.build()
    return F.load()


def test_codes_and_scales():
    assert N.E2M1[:8].tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6] and np.array_equal(N.E2M1[8:], -N.E2M1[:8])
    half = torch.from_numpy((np.arange(256) << 7).astype(np.int16)).view(torch.float16).double().numpy()
    assert np.array_equal(N.SCALE, half, equal_nan=True)
    assert N.SCALE[N.LEAST] == 2.0 ** -14 and N.SCALE[N.MOST] == 10240 and np.isnan(N.SCALE[N.NAN])
    products = np.abs(N.E2M1[:, None] * N.SCALE[:N.MOST + 1])
    assert np.array_equal(products.astype(np.float16).astype(np.float64), products)       # every one is an fp16 number


def test_quantise_by_hand():
    x = np.zeros((1, 64))
    x[0, :16] = [6, 0.25, 0.26, 0.75, 0.74, 1.25, 1.26, 1.75, -2.5, -2.6, 3.5, 3.4, 5, 5.1, -0.0, -6]     # the scale is 1
    x[0, 16:20] = [6 * 1.0625, 1, 0, 0]                        # 1.0625: a tie of scales, to the even one, 1; 6.375 becomes 6
    x[0, 32] = 1e-9
    x[0, 48] = 1e9
    codes, scale = N.quantise(x)
    assert codes[0, :16].tolist() == [7, 0, 1, 2, 1, 2, 3, 4, 12, 13, 6, 5, 6, 7, 8, 15]
    assert N.SCALE[scale[0]].tolist() == [1, 1, 2.0 ** -14, 10240] and codes[0, [16, 17, 32, 48]].tolist() == [7, 2, 0, 7]
    x[0, 3], x[0, 40] = np.nan, -np.inf
    codes, scale = N.quantise(x)
    assert scale[0, 0] == scale[0, 2] == N.NAN and (codes[0, :16] == 0).all() and scale[0, 1] == 120
    assert N.pack(np.array([[1, 15, 8, 0]])).tolist() == [[0xF1, 0x08]]
    assert np.array_equal(N.unpack(N.pack(codes)), codes)


def test_rotary_by_hand():
    f = R.frequencies(4, 100.0)
    assert np.allclose(f, [1.0, 0.1])
    x = np.array([1.0, 0.0, 0.0, 2.0, 9.0]).reshape(1, 1, 1, 5)
    y = R.rotate(x, np.full((1, 1, 1), 3), f)
    assert np.allclose(y.ravel(), [math.cos(3), -2 * math.sin(0.3), math.sin(3), 2 * math.cos(0.3), 9])
    y = R.rotate(x, np.full((1, 1, 1), 3), f, R.PAIRS, amplitude=2.0, adjoint=True)
    assert np.allclose(y.ravel(), [2 * math.cos(3), -2 * math.sin(3), 4 * math.sin(0.3), 4 * math.cos(0.3), 9])
    y = R.rotate(x, np.array([[[3], [0], [10]]]), f, sections=[1, 0, 1])
    assert np.allclose(y.ravel(), [math.cos(3), -2 * math.sin(1), math.sin(3), 2 * math.cos(1), 9])
    assert np.allclose(R.frequencies(4, 100.0, R.LINEAR, factor=4.0), [0.25, 0.025])
    f = R.frequencies(64, 10000.0, R.BY_PARTS, factor=4.0, low=1.0, high=32.0, trained=1000)
    assert f[0] == 1.0 and np.isclose(f[-1], 10000.0 ** (-62 / 64) / 4) and (np.diff(f) < 0).all()


GOOD = dict(n_units=2, n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=64, n_pages=10, max_pages=4, n_rows=8)
POINTERS = {"flowmm_nibble_store": 7, "flowmm_nibble_load": 8, "flowmm_nibble_attention": 8}
WIDE = {"flowmm_nibble_store": (0, 1, 3, 4, 5, 6), "flowmm_nibble_load": (0, 1, 2, 3, 6, 7), "flowmm_nibble_attention": (0, 1, 2, 3, 4, 7)}


def _args(n):
    return [(i + 1) << 20 for i in range(n)]


@pytest.mark.parametrize("name", sorted(POINTERS))
def test_refusals_of_the_cache(lib, name):
    """Every call here is refused by a check on the host, before the library looks for a device."""
    call = lambda p, args, ws=1 << 20, ws_bytes=1 << 40: getattr(lib, name)(ctypes.byref(p), *args, ws, ws_bytes, None)
    n = POINTERS[name]
    for change, code in [(dict(n_units=0), 2), (dict(n_q_heads=7), 2), (dict(n_q_heads=18), 2), (dict(n_kv_heads=0), 2), (dict(head_dim=96), 2), (dict(page_size=48), 2),
                         (dict(n_pages=0), 2), (dict(max_pages=0), 2), (dict(n_rows=-1), 2), (dict(n_pages=1 << 26), 2), (dict(max_pages=1 << 25), 2),
                         (dict(n_units=1 << 12, n_rows=1 << 19), 2), (dict(n_units=1 << 22), 2), (dict(dtype=2), 4), (dict(softmax_scale=-1.0), 2),
                         (dict(softmax_scale=float("nan")), 2), (dict(path=3), 2)]:
        p = F.CacheParams(**{**GOOD, **change}).c()
        assert call(p, _args(n)) == code, change
        size = ctypes.c_size_t(0)
        assert lib.flowmm_nibble_workspace_bytes(ctypes.byref(p), ctypes.byref(size)) == code, change
    p = F.CacheParams(**GOOD).c()
    for i in range(n):
        args = _args(n)
        args[i] = None
        assert call(p, args) == 1, i
        args[i] = ((i + 1) << 20) + (8 if i in WIDE[name] else 2)
        assert call(p, args) == 6, i
    need = F.flowmm_nibble_workspace_bytes(F.CacheParams(**GOOD))
    assert call(p, _args(n), ws=None) == 1 and call(p, _args(n), ws=(1 << 20) + 128) == 6 and call(p, _args(n), ws_bytes=need - 1) == 5
    assert getattr(lib, name)(None, *_args(n), 1 << 20, 1 << 40, None) == 1
    assert lib.flowmm_nibble_workspace_bytes(ctypes.byref(p), None) == 1
    if name != "flowmm_nibble_attention":
        for field in ("k_stride", "v_stride"):
            for i, bad in ((0, 1004), (1, -128), (2, 64)):
                c = F.CacheParams(**GOOD).c()
                getattr(c, field)[i] = bad
                assert call(c, _args(n)) == 6, (field, i)
        assert call(F.CacheParams(**{**GOOD, "n_rows": 0}).c(), _args(n)) == 2
        many = dict(n_units=4, n_kv_heads=8, n_rows=1 << 28) if name == "flowmm_nibble_store" else dict(n_units=1 << 16, n_kv_heads=64, n_q_heads=64, n_rows=(1 << 15) - 1)
        assert call(F.CacheParams(**{**GOOD, **many}).c(), _args(n)) == 2
    else:
        assert call(F.CacheParams(**{**GOOD, "n_units": 1 << 20, "max_pages": 1 << 12}).c(), _args(n)) == 2


ROTARY = dict(n_units=2, n_q_heads=4, n_kv_heads=2, head_dim=128, n_rows=8)


def test_refusals_of_rotary(lib):
    call = lambda c, args: lib.flowmm_rotary(ctypes.byref(c), *args, None)
    for change, code in [(dict(n_units=0), 2), (dict(n_q_heads=0), 2), (dict(n_kv_heads=0), 2), (dict(n_rows=0), 2), (dict(head_dim=96), 2), (dict(rotary_dim=144), 2),
                         (dict(rotary_dim=24), 2), (dict(rotary_dim=-16), 2), (dict(layout=2), 2), (dict(sections=(16, 24, 23)), 2), (dict(sections=(-1, 64, 1)), 2),
                         (dict(scaling=3), 2), (dict(base=0.5), 2), (dict(base=float("nan")), 2), (dict(base=float("inf")), 2), (dict(scaling=1, factor=0.0), 2),
                         (dict(scaling=2, low=4.0, high=4.0), 2), (dict(scaling=2, trained=-1), 2), (dict(amplitude=float("nan")), 2), (dict(dtype=2), 4),
                         (dict(n_units=1 << 16, n_rows=1 << 15), 2)]:
        c = F.RotaryParams(**{**ROTARY, **change}).c()
        assert call(c, _args(6)) == code, change
        assert lib.flowmm_rotary_table(ctypes.byref(c), 1 << 20, None) == code, change
    good = F.RotaryParams(**ROTARY).c()
    c = F.RotaryParams(**ROTARY).c()
    c.n_axes = 2
    assert call(c, _args(6)) == 2
    c = F.RotaryParams(**ROTARY).c()
    c.adjoint = 2
    assert call(c, _args(6)) == 2
    for missing, code in [((0,), 1), ((1,), 1), ((2,), 1), ((3,), 1), ((4,), 1), ((5,), 1), ((0, 4, 1, 5), 1)]:
        args = _args(6)
        for i in missing:
            args[i] = None
        assert call(good, args) == code, missing
    for i, off in ((0, 8), (1, 8), (2, 2), (3, 4), (4, 8), (5, 8)):
        args = _args(6)
        args[i] += off
        assert call(good, args) == 6, i
    for field in ("q_stride", "k_stride", "q_out_stride", "k_out_stride"):
        for i, bad in ((0, 1004), (1, -128), (2, 64)):
            c = F.RotaryParams(**ROTARY).c()
            getattr(c, field)[i] = bad
            assert call(c, _args(6)) == 6, (field, i)
    args = _args(6)
    args[4] = args[0]
    c = F.RotaryParams(**ROTARY).c()
    c.q_out_stride[1] += 128
    assert call(c, args) == 2                                   # in place with other strides
    assert lib.flowmm_rotary(None, *_args(6), None) == 1 and lib.flowmm_rotary_table(None, 1 << 20, None) == 1
    assert lib.flowmm_rotary_table(ctypes.byref(good), None, None) == 1 and lib.flowmm_rotary_table(ctypes.byref(good), (1 << 20) + 4, None) == 6


def test_binding_looks_at_tensors():
    p = F.CacheParams(**GOOD)
    t = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        F.flowmm_nibble_store(p, t, t, t, t, t, t, t, t)
    r = F.RotaryParams(**ROTARY)
    q, k = torch.zeros(2, 4, 8, 128, dtype=torch.bfloat16), torch.zeros(2, 2, 8, 128, dtype=torch.bfloat16)
    pos, table = torch.zeros(2, 8, dtype=torch.int32), torch.zeros(64, dtype=torch.int64)
    for bad in ((k, k, pos, table, k, k), (q, k.float(), pos, table, q, k), (q, k, pos[:1], table, q, k), (q, k, pos.long(), table, q, k), (q, k, pos, table[:32], q, k),
                (q, k, pos, table.int(), q, k), (q, k, pos, table, q, k)):
        with pytest.raises(ValueError):
            F.flowmm_rotary(r, *bad)
    with pytest.raises(ValueError):
        F.RotaryParams(**ROTARY, sections=(1, 63)).c()


def test_struct_matches_header():
    header = open(os.path.join(ROOT, "include", "flowmm.h")).read()
    end = header.index("} flowmm_rotary_params;")
    body = re.sub(r"/\*.*?\*/", "", header[header.rindex("typedef struct {", 0, end):end], flags=re.S)
    names = [n.strip().split("[")[0] for group in re.findall(r"(?:int32_t|float|double|int64_t)\s+([^;]+);", body) for n in group.split(",")]
    assert names == [f[0] for f in F._CRotaryParams._fields_]
    assert ctypes.sizeof(F._CRotaryParams) == 16 * 4 + 4 * 8 + 12 * 8
    for name, value in (("HALVES", 0), ("PAIRS", 1), ("PLAIN", 0), ("LINEAR", 1), ("BY_PARTS", 2)):
        assert "FLOWMM_ROTARY_%s = %d" % (name, value) in header and getattr(F, "ROTARY_" + name) == value


@pytest.mark.parametrize("D,dtype", [(128, F.BF16), (64, F.F32)])
def test_workspace_never_shrinks(lib, D, dtype):
    """A workspace kept for the most units, the widest table and the most rows serves smaller calls."""
    size = lambda U, wide, page, G: F.flowmm_nibble_workspace_bytes(F.CacheParams(U, 2 * G, 2, D, page, 100, wide, 1, dtype=dtype))
    for G in (1, 4, 7, 8):
        for U in (1, 3, 40, 300):
            sizes = [size(U, wide, 64, G) for wide in range(1, 700)]
            assert sizes == sorted(sizes)
        for wide in (1, 10, 95, 97, 110, 128, 129, 500):
            sizes = [size(U, wide, 16, G) for U in range(1, 700)]
            assert sizes == sorted(sizes)


def test_rotary_params_can_be_copied_and_pickled():
    """Also with the handle of a call in them, which is an address of this process and gone when a field changes."""
    import copy
    import pickle
    p = F.RotaryParams(**ROTARY, sections=[16, 24, 24], scaling=F.ROTARY_BY_PARTS, factor=4.0, trained=100, adjoint=True, amplitude=1.5)
    p.calls["flowmm_rotary"] = object()
    for q in (copy.copy(p), copy.deepcopy(p), pickle.loads(pickle.dumps(p))):
        assert q == p and q.calls == {} and q.sections == (16, 24, 24) and bytes(q.c()) == bytes(p.c())
    p.base = 5.0
    assert p.calls == {} and p.c().base == 5.0
