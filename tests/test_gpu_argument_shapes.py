"""Which shapes the calls through the marshalling module take: one only for each argument, but for positions with one a row."""
import pytest
import torch

from paper_2511_05534_b200 import binding as F

pytestmark = pytest.mark.gpu


def _zeros(*shape, dtype=torch.uint8):
    return torch.zeros(shape, dtype=dtype, device="cuda")


@pytest.mark.parametrize("which", ["q", "out"])
@pytest.mark.parametrize("cache", ["8 bits", "4 bits"])
def test_queries_of_one_head_keep_their_dimension(cache, which):
    p = F.CacheParams(2, 1, 1, 64, 16, 4, 2)
    table, rows = _zeros(2, 2, dtype=torch.int32), _zeros(2, dtype=torch.int32)
    q = _zeros(2, 1, 64, dtype=torch.bfloat16)
    if cache == "8 bits":
        call, ws, out = F.flowmm_cache_attention, F.alloc_cache_workspace(p), _zeros(2, 1, 64, dtype=torch.float32)
        pool = [_zeros(4, 1, 16, 64), _zeros(4, 1, 16, 64), _zeros(4, 1, dtype=torch.float32), _zeros(4, 1, dtype=torch.float32)]
    else:
        call, ws, out = F.flowmm_nibble_attention, F.alloc_nibble_workspace(p), torch.empty_like(q)
        pool = [_zeros(4, 1, 16, 32), _zeros(4, 1, 16, 32), _zeros(4, 1, 16, 4), _zeros(4, 1, 16, 4)]
    call(p, q, *pool, table, rows, out, ws)
    assert F.flowmm_last_device_status(ws) == 0
    with pytest.raises(ValueError, match="%s must be a .* of shape \\[2, 1, 64\\]" % which):
        call(p, q.view(2, 64) if which == "q" else q, *pool, table, rows, out.view(2, 64) if which == "out" else out, ws)


def test_positions_with_and_without_their_axis():
    p = F.RotaryParams(2, 1, 1, 64, 5)
    q, k = (torch.randn((2, 1, 5, 64), device="cuda").to(torch.bfloat16) for _ in "qk")
    table, pos = F.alloc_rotary_table(p), torch.arange(10, dtype=torch.int32, device="cuda").view(2, 5)
    outs = []
    for at in (pos, pos.view(2, 1, 5)):
        outs.append([torch.empty_like(q), torch.empty_like(k)])
        F.flowmm_rotary(p, q, k, at, table, *outs[-1])
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    for bad in (pos.view(10), pos.view(1, 2, 5), pos[:, :4].contiguous(), pos.view(2, 1, 1, 5), pos.view(5, 2)):
        with pytest.raises(ValueError, match="positions"):
            F.flowmm_rotary(p, q, k, bad, table, *outs[0])
    p = F.RotaryParams(2, 1, 1, 64, 5, sections=(8, 8, 16))
    with pytest.raises(ValueError, match="positions"):
        F.flowmm_rotary(p, q, k, pos, table, *outs[0])


def test_rotary_of_one_row_and_unit():
    """All sizes one: nothing else of as many elements passes for another shape."""
    p = F.RotaryParams(1, 1, 1, 64, 1)
    q = torch.randn((1, 1, 1, 64), device="cuda").to(torch.bfloat16)
    pos, table = _zeros(1, 1, dtype=torch.int32), F.alloc_rotary_table(p)
    F.flowmm_rotary(p, q, None, pos, table, q, None)
    for bad in (dict(q=q.view(1, 1, 64)), dict(table=table.view(1, 32)), dict(pos=pos.view(1))):
        with pytest.raises(ValueError):
            F.flowmm_rotary(p, bad.get("q", q), None, bad.get("pos", pos), bad.get("table", table), q, None)
