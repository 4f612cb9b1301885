"""Rotary positions of many rows: on both sides of the number from which a block takes more rows (4 KB of a head on end instead of four)."""
import numpy as np
import pytest
import torch

from oracle import rotary as R
from paper_2511_05534_b200 import binding as F

from test_gpu_rotary import case, check

pytestmark = pytest.mark.gpu
MANY = {(F.BF16, 128): 9472, (F.F32, 128): 4736, (F.BF16, 64): 18944, (F.F32, 64): 9472}      # 4 blocks for each of 148 SMs


@pytest.mark.parametrize("dtype", [F.BF16, F.F32])
@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("layout", [R.HALVES, R.PAIRS])
@pytest.mark.parametrize("units,more", [(1, -1), (1, 0), (1, 13), (7, 5), (331, 1)])
def test_equals_oracle(dtype, D, layout, units, more):
    """Rows that fill the last block or not, blocks that span two units and three, the whole head and part of it, an odd number of heads."""
    rng = np.random.default_rng(units + more + D)
    T = MANY[dtype, D] // units + more
    rot, Hq, H = (D, 3, 2) if units == 1 else (D // 2, 1, 2)
    x, pos = case(rng, units, Hq, H, D, T, dtype)
    p = F.RotaryParams(units, Hq, H, D, T, dtype=dtype, rotary_dim=rot, layout=layout)
    y = [torch.full_like(t, float("nan")) for t in x]
    F.flowmm_rotary(p, *x, torch.from_numpy(pos).cuda(), F.alloc_rotary_table(p), *y)
    check(x, y, pos, R.frequencies(rot, 10000.0), dtype, layout, None, 1.0, False)


@pytest.mark.parametrize("dtype", [F.BF16, F.F32])
@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("layout", [R.HALVES, R.PAIRS])
def test_three_positions_in_place_and_strides(dtype, D, layout):
    """In place, in rows that are heads' neighbours in memory, with room between them; what lies there is left."""
    rng = np.random.default_rng(D)
    units, Hq, H, rot = 5, 3, 1, D // 2 + 16
    T, sections = MANY[dtype, D] // units + 3, (rot // 4, 0, rot // 4)
    x, pos = case(rng, units, Hq, H, D, T, dtype, axes=3)
    wide = torch.full((units, T, Hq + H, D + 8), 7.0, device="cuda", dtype=x[0].dtype)
    views = [wide[:, :, :Hq, :D].transpose(1, 2), wide[:, :, Hq:, :D].transpose(1, 2)]
    for v, t in zip(views, x):
        v.copy_(t)
    p = F.RotaryParams(units, Hq, H, D, T, dtype=dtype, rotary_dim=rot, layout=layout, sections=sections, adjoint=True, amplitude=1.25)
    F.flowmm_rotary(p, *views, torch.from_numpy(pos).cuda(), F.alloc_rotary_table(p), *views)
    check(x, views, pos, R.frequencies(rot, 10000.0), dtype, layout, sections, 1.25, True)
    assert (wide[..., D:] == 7.0).all()


def test_calls_of_many_rows_and_of_few_give_the_same_bits():
    """A row's angle and products do not depend on the number of rows that are turned with it."""
    rng = np.random.default_rng(5)
    x, pos = case(rng, 1, 2, 1, 128, 9999, F.BF16)
    p = F.RotaryParams(1, 2, 1, 128, 9999)
    t, at = F.alloc_rotary_table(p), torch.from_numpy(pos).cuda()
    y = [torch.empty_like(a) for a in x]
    F.flowmm_rotary(p, *x, at, t, *y)
    p.n_rows = 999
    few = [torch.empty_like(a[:, :, 9000:]) for a in x]
    F.flowmm_rotary(p, *(a[:, :, 9000:] for a in x), at[..., 9000:].contiguous(), t, *few)
    assert all(torch.equal(a[:, :, 9000:], b) for a, b in zip(y, few))
