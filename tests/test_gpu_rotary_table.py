"""The table of phases and the angles of far positions, against arithmetic in 60 digits."""
from decimal import Decimal, getcontext

import numpy as np
import pytest
import torch

from paper_2511_05534_b200 import binding as F

pytestmark = pytest.mark.gpu
getcontext().prec = 60
TURN = 2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")
FORMS = [dict(base=10000.0), dict(base=500000.0), dict(base=1e6), dict(base=1.0), dict(base=1e300), dict(base=10000.0, scaling=F.ROTARY_LINEAR, factor=3.7),
         dict(base=1e6, scaling=F.ROTARY_BY_PARTS, factor=4.0, low=1.0, high=32.0, trained=32768),
         dict(base=500000.0, scaling=F.ROTARY_BY_PARTS, factor=8.0, low=1.0, high=4.0, trained=8192)]


def turns(R, base, scaling=F.ROTARY_PLAIN, factor=1.0, low=1.0, high=32.0, trained=0):
    """What a position adds to each pair's phase, in turns."""
    out = []
    for i in range(R // 2):
        f = Decimal(base) ** (Decimal(-2 * i) / R)
        if scaling == F.ROTARY_LINEAR:
            f /= Decimal(factor)
        if scaling == F.ROTARY_BY_PARTS:
            g = min(Decimal(1), max(Decimal(0), (trained * f / TURN - Decimal(low)) / (Decimal(high) - Decimal(low))))
            f = g * f + (1 - g) * f / Decimal(factor)
        out.append(f / TURN)
    return out


def table_of(D, rot, form):
    return F.alloc_rotary_table(F.RotaryParams(1, 1, 1, D, 1, rotary_dim=rot, **form)).cpu().numpy().view(np.uint64)


def away(x):
    """How far a number of turns is from a whole one."""
    x = abs(x) % 1
    return min(x, 1 - x)


@pytest.mark.parametrize("D,rot", [(128, 128), (128, 112), (64, 64), (64, 16)])
@pytest.mark.parametrize("form", FORMS)
def test_table(D, rot, form):
    """Numbers up to 0.16 with 64 significant bits: the power and the division within a unit of 2^-66, the parts' products as many, then the nearest
    multiple of 2^-64: within two of them."""
    want = turns(rot, **form)
    got = table_of(D, rot, form)
    assert got.shape == (rot // 2,)
    for i, t in enumerate(want):
        assert away(Decimal(int(got[i])) / 2 ** 64 - t) <= Decimal(2) ** -63, i


@pytest.mark.parametrize("factor", [0.5, 2.0 ** -20, 1e-30, 1e-300, 5e-324])
def test_table_of_a_factor_below_one(factor):
    """64 significant bits of a number that is 1 / factor times as large; beyond 2^64 turns nothing is left of the fraction, and the call still ends well."""
    form = dict(base=10000.0, scaling=F.ROTARY_LINEAR, factor=factor)
    got = table_of(128, 128, form)
    for i, t in enumerate(turns(128, **form)):
        allowed = max(Decimal(2) ** -63, t * Decimal(2) ** -62)
        assert allowed >= 0.5 or away(Decimal(int(got[i])) / 2 ** 64 - t) <= allowed, i


@pytest.mark.parametrize("form", FORMS)
def test_far_positions(form):
    """Any position's angle within 2^-31 turns, then sine and cosine within 2^-23 (of one: 2^-24 rounding, the angle's own 2^-25)."""
    rng = np.random.default_rng(3)
    pos = rng.integers(-(1 << 31), 1 << 31, 256).astype(np.int32)
    pos[:8] = [0, 1, -1, 2147483647, -2147483648, 1 << 24, 1 << 28, -(1 << 20)]
    x = torch.zeros((1, 1, 256, 128), device="cuda")
    x[..., :64] = 1.0
    p = F.RotaryParams(1, 1, 1, 128, 256, dtype=F.F32, **form)
    y = torch.empty_like(x)
    F.flowmm_rotary(p, x, None, torch.from_numpy(pos).cuda().view(1, 256), F.alloc_rotary_table(p), y, None)
    y = y.double().cpu().numpy()[0, 0]
    each = turns(128, **form)
    phase = np.array([[float((int(at) * t + Decimal("0.5")) % 1) for t in each] for at in pos])
    angle = 2 * np.pi * (phase - 0.5)
    allowed = 2 * np.pi * 2.0 ** -31 + 2.0 ** -23
    assert np.abs(y[:, :64] - np.cos(angle)).max() <= allowed
    assert np.abs(y[:, 64:] - np.sin(angle)).max() <= allowed


def test_a_table_of_one_s_own():
    """Frequencies of any other kind: what a caller writes into the table, as 64-bit fractions of a turn, is what is turned by."""
    rng = np.random.default_rng(4)
    own = [Decimal(int(x)) / 10 ** 12 for x in rng.integers(1, 10 ** 12, 64)]
    bits = np.array([int((t % 1) * 2 ** 64) for t in own], np.uint64)
    x = torch.zeros((1, 1, 100, 128), device="cuda")
    x[..., 0::2] = 1.0
    pos = torch.arange(1000, 1100, dtype=torch.int32, device="cuda").view(1, 100)
    y = torch.empty_like(x)
    p = F.RotaryParams(1, 1, 1, 128, 100, dtype=F.F32, layout=F.ROTARY_PAIRS)
    F.flowmm_rotary(p, x, None, pos, torch.from_numpy(bits.view(np.int64)).cuda(), y, None)
    angle = 2 * np.pi * np.array([[float(at * t % 1) for t in own] for at in range(1000, 1100)])
    y = y.double().cpu().numpy()[0, 0]
    allowed = 2 * np.pi * 2.0 ** -31 + 2.0 ** -23
    assert np.abs(y[:, 0::2] - np.cos(angle)).max() <= allowed and np.abs(y[:, 1::2] - np.sin(angle)).max() <= allowed
