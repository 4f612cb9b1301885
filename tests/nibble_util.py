"""Paged 4-bit caches for the tests: pools with bytes of any kind in them, and the calls of the binding."""
import numpy as np
import torch

from oracle import nibble_cache as N
from paper_2511_05534_b200 import binding as F

from paged_util import dev, params, random_table        # noqa: F401 (the same for both caches)


def random_pool(rng, n_pages, H, page, D, rows, table, scales=(96, 140)):
    """[k, v, k scale, v scale] as bytes: scales from 2^-3 to 2^2 in rows that units hold, any byte elsewhere, NaN and infinity among them."""
    pool = [rng.integers(0, 256, (n_pages, H, page, D // w)).astype(np.uint8) for w in (2, 2, 16, 16)]
    for s in pool[2:]:
        for u, n in enumerate(rows):
            for j in range(N.pages(int(n), page)):
                there = s[table[u, j], :, :min(page, int(n) - j * page)]
                there[...] = rng.integers(*scales, there.shape)
    return pool


def attend(p, q, pool, table, rows, ws=None):
    """flowmm_nibble_attention on numpy arrays; (out float64, device status)."""
    ws = F.alloc_nibble_workspace(p) if ws is None else ws
    out = torch.full((p.n_units, p.n_q_heads, p.head_dim), float("nan"), device="cuda", dtype=F.torch_dtype(p.dtype))
    F.flowmm_nibble_attention(p, dev(q, p.dtype), *map(dev, pool), dev(table), dev(np.asarray(rows, np.int32)), out, ws)
    status = F.flowmm_last_device_status(ws)
    return out.double().cpu().numpy(), status


def attention_bound(out, size, logits, n, D, dtype):
    """How far an implementation may be from the 64-bit one, per output.
    Logits: D products and their sum in fp32, the scale, each within 2^-23 (a tensor core that truncates); an fp32 query as two fp16 numbers,
    2^-21 of its largest element (a bf16 one is an fp16 number exactly).  Weights: exp2 within 2^-21; in fp16, whose least normal number is 2^-14 and whose
    step below that is 2^-24, the largest weight is 2^10 at least for bf16 (2^14 for fp32).  bf16: one number, 2^-11 of itself down to 2^-14, 2^-24 of the
    largest.  fp32: two numbers, the second within 2^-11 of itself, 2^-22 of the weight, or half a step, 2^-25, which is 2^-21 of a weight of 2^-4, 2^-18 of the
    largest.  `size` counts weights as 2^-18 of the largest at least (oracle.nibble_cache.attention).
    Sums of n weights and products, each within 2^-23.  Numerator and denominator both carry the weights' error.  A bf16 output: half a step, 2^-8."""
    split = 2.0 ** -11 if dtype == F.BF16 else 2.0 ** -21
    rel = (D + 16) * 2.0 ** -23 * logits + 2.0 ** -21 * logits + split + 2.0 ** -21 + (n + 16) * 2.0 ** -23
    bound = 2 * rel[..., None] * size + 1e-30
    return bound if dtype == F.F32 else bound + 2.0 ** -8 * (np.abs(out) + bound)
