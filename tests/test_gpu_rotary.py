"""Rotary positions on the GPU against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from oracle import rotary as R
from paper_2511_05534_b200 import binding as F

pytestmark = pytest.mark.gpu


def dev(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda().to(F.torch_dtype(dtype))


def bound(x, want, dtype, R_, amplitude, layout, slack=0.0):
    """cos and sin within 2^-23 (one unit in the last place, and the angle's own 2^-25), the amplitude, two products and their sum within 2^-24 each: 2^-21
    of |a| + |b|; a bf16 output half a step, 2^-8; slack: what the angle may be off by."""
    y = np.abs(x)
    pair = np.zeros_like(y)
    a, b = (slice(0, R_ // 2), slice(R_ // 2, R_)) if layout == R.HALVES else (slice(0, R_, 2), slice(1, R_, 2))
    pair[..., a] = pair[..., b] = y[..., a] + y[..., b]
    out = pair * amplitude * (2.0 ** -21 + slack) + 1e-37
    out[..., R_:] = 0.0
    if dtype == F.BF16:
        out[..., :R_] += 2.0 ** -8 * (np.abs(want[..., :R_]) + out[..., :R_])
    return out


def case(rng, U, Hq, H, D, T, dtype, axes=1, far=100000):
    x = [dev(rng.standard_normal((U, h, T, D)), dtype) for h in (Hq, H)]
    pos = rng.integers(-far if far < 1000 else 0, far, (U, axes, T)).astype(np.int32)
    return x, pos


def check(x, y, pos, freq, dtype, layout, sections, amplitude, adjoint, slack=0.0):
    for a, b in zip(x, y):
        a = a.double().cpu().numpy()
        want = R.rotate(a, pos, freq, layout, sections, amplitude, adjoint)
        err = np.abs(b.double().cpu().numpy() - want)
        assert (err <= bound(a, want, dtype, 2 * len(freq), amplitude, layout, slack)).all(), err.max()


@pytest.mark.parametrize("dtype", [F.BF16, F.F32])
@pytest.mark.parametrize("layout", [R.HALVES, R.PAIRS])
@pytest.mark.parametrize("U,Hq,H,D,T,rot", [(1, 1, 1, 64, 1, 64), (4, 64, 8, 128, 1, 128), (2, 4, 4, 64, 577, 32), (3, 7, 1, 128, 33, 64), (1, 28, 4, 128, 2000, 128), (5, 5, 5, 64, 3, 16),
                                            (2, 3, 2, 128, 100, 112)])
def test_equals_oracle(dtype, layout, U, Hq, H, D, T, rot):
    rng = np.random.default_rng(T + D)
    x, pos = case(rng, U, Hq, H, D, T, dtype)
    p = F.RotaryParams(U, Hq, H, D, T, dtype=dtype, rotary_dim=rot, layout=layout)
    y = [torch.full_like(t, float("nan")) for t in x]
    keep = [t.clone() for t in x]
    F.flowmm_rotary(p, *x, torch.from_numpy(pos).cuda(), F.alloc_rotary_table(p), *y)
    assert all(torch.equal(a, b) for a, b in zip(x, keep))
    check(x, y, pos, R.frequencies(rot, 10000.0), dtype, layout, None, 1.0, False)


@pytest.mark.parametrize("scaling", [R.PLAIN, R.LINEAR, R.BY_PARTS])
@pytest.mark.parametrize("sections", [None, (16, 24, 24), (0, 64, 0), (1, 2, 61)])
@pytest.mark.parametrize("adjoint", [False, True])
@pytest.mark.parametrize("layout", [R.HALVES, R.PAIRS])
def test_scaled_frequencies_and_three_positions(scaling, sections, adjoint, layout):
    rng = np.random.default_rng(7)
    kw = dict(scaling=scaling, base=500000.0, factor=8.0, low=1.0, high=4.0, trained=8192)
    x, pos = case(rng, 2, 4, 2, 128, 50, F.F32, axes=3 if sections else 1, far=1 << 20)
    p = F.RotaryParams(2, 4, 2, 128, 50, dtype=F.F32, layout=layout, adjoint=adjoint, sections=sections, amplitude=1.25, **kw)
    y = [torch.empty_like(t) for t in x]
    F.flowmm_rotary(p, *x, torch.from_numpy(pos).cuda(), F.alloc_rotary_table(p), *y)
    freq = R.frequencies(128, **{k: v for k, v in kw.items() if k != "base"}, base=kw["base"])
    check(x, y, pos, freq, F.F32, layout, sections, 1.25, adjoint)


def test_far_and_negative_positions():
    """Frequencies carry 2^-51 of themselves (a power in 64 bits, here and there), so an angle of position * frequency that part of it."""
    rng = np.random.default_rng(8)
    x, _ = case(rng, 1, 2, 2, 128, 64, F.F32)
    pos = rng.integers(-(1 << 31), 1 << 31, (1, 1, 64)).astype(np.int32)
    pos[0, 0, :6] = [0, -1, 1, 2147483647, -2147483648, 1 << 24]
    p = F.RotaryParams(1, 2, 2, 128, 64, dtype=F.F32)
    y = [torch.empty_like(t) for t in x]
    F.flowmm_rotary(p, *x, torch.from_numpy(pos).cuda(), F.alloc_rotary_table(p), *y)
    check(x, y, pos, R.frequencies(128, 10000.0), F.F32, R.HALVES, None, 1.0, False, slack=2.0 ** 31 * 2.0 ** -51 + 2.0 ** -28)


@pytest.mark.parametrize("dtype", [F.BF16, F.F32])
@pytest.mark.parametrize("layout", [R.HALVES, R.PAIRS])
@pytest.mark.parametrize("rot", [64, 32])
def test_in_place_one_tensor_and_strides(dtype, layout, rot):
    """An output that is its input, queries or keys alone, and tensors [units, rows, heads, head_dim]: the same bits as the plain call."""
    rng = np.random.default_rng(9)
    x, pos = case(rng, 2, 6, 2, 64, 37, dtype)
    p = F.RotaryParams(2, 6, 2, 64, 37, dtype=dtype, rotary_dim=rot, layout=layout, base=1e6)
    t, pos = F.alloc_rotary_table(p), torch.from_numpy(pos).cuda()
    y = [torch.empty_like(a) for a in x]
    F.flowmm_rotary(p, *x, pos, t, *y)
    z = [a.clone() for a in x]
    F.flowmm_rotary(p, *z, pos, t, *z)
    assert all(torch.equal(a, b) for a, b in zip(y, z))
    z = [torch.empty_like(a) for a in x]
    F.flowmm_rotary(p, x[0], None, pos, t, z[0], None)
    F.flowmm_rotary(p, None, x[1], pos, t, None, z[1])
    assert all(torch.equal(a, b) for a, b in zip(y, z))
    fused = torch.cat([a.transpose(1, 2) for a in x], 2).contiguous()              # as a projection leaves them
    out = torch.zeros_like(fused)
    F.flowmm_rotary(p, *(fused[:, :, s].transpose(1, 2) for s in (slice(0, 6), slice(6, 8))), pos, t,
                    *(out[:, :, s].transpose(1, 2) for s in (slice(0, 6), slice(6, 8))))
    assert torch.equal(out, torch.cat([a.transpose(1, 2) for a in y], 2))


@pytest.mark.parametrize("layout", [R.HALVES, R.PAIRS])
@pytest.mark.parametrize("amplitude", [1.0, 1.2])
def test_adjoint_is_the_gradient(layout, amplitude):
    """Against the transposed matrix of the forward call, found column by column (a linear map's differences), and the inverse for amplitude 1."""
    U, D, T, rot = 1, 64, 5, 32
    pos = torch.tensor([[3, 1000, 77777, 0, 12]], dtype=torch.int32, device="cuda")
    p = F.RotaryParams(U, D, 1, D, T, dtype=F.F32, rotary_dim=rot, layout=layout, amplitude=amplitude)
    t = F.alloc_rotary_table(p)
    eye = torch.eye(D, device="cuda").view(1, D, 1, D).expand(U, D, T, D).contiguous()
    m = torch.empty_like(eye)                                                     # m[:, i]: what the i-th unit vector becomes
    F.flowmm_rotary(p, eye, None, pos, t, m, None)
    p.adjoint = True
    back = torch.empty_like(eye)
    F.flowmm_rotary(p, eye, None, pos, t, back, None)
    assert torch.equal(back, m.permute(0, 3, 2, 1))
    if amplitude == 1.0:
        x = torch.randn((U, D, T, D), device="cuda")
        there, again = torch.empty_like(x), torch.empty_like(x)
        p.adjoint = False
        F.flowmm_rotary(p, x, None, pos, t, there, None)
        p.adjoint = True
        F.flowmm_rotary(p, there, None, pos, t, again, None)
        # (each way within 2^-21 of |a| + |b|, at most 2 (|a| + |b|) after the first)
        assert (again - x).abs().max() <= 3 * 2.0 ** -21 * 2 * x.abs().max()


def test_captured_in_a_graph_on_another_stream():
    rng = np.random.default_rng(10)
    x, pos = case(rng, 3, 4, 2, 128, 1, F.BF16)
    p = F.RotaryParams(3, 4, 2, 128, 1)
    t, pos_d = F.alloc_rotary_table(p), torch.from_numpy(pos).cuda()
    y = [torch.empty_like(a) for a in x]
    F.flowmm_rotary(p, *x, pos_d, t, *y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        F.flowmm_rotary(p, *x, pos_d, t, *y)
    for step in range(3):
        pos_d += 1
        graph.replay()
        check(x, y, pos + step + 1, R.frequencies(128, 10000.0), F.BF16, R.HALVES, None, 1.0, False)
