"""Rotary positions and the paged 4-bit cache's operators, as timed cases, with their plain forms.

  rotary     flowmm_rotary: queries and keys turned by their tokens' positions, halves or neighbouring pairs, a part of the head,
             one position a row or three (time, height, width of image tokens), frequencies scaled for long contexts
  store      flowmm_nibble_store: rows of K and V into pages, e2m1 codes, two a byte, with a scale for every 16 channels of a row
  load       flowmm_nibble_load: pages back into dense rows, as flowmm_recompress takes them
  attention  flowmm_nibble_attention: one new query per query head over the pages of every unit, lengths of their own

A unit is one (layer, sequence) pair, as in the rest of the library.  Head layouts, lengths and budgets are those of
`configs.WORKLOADS`.  Rows that no sequence holds (behind a unit's last row, pages nobody owns) hold arbitrary bytes, scales of
NaN among them, as memory that earlier requests have left does.  Codes and scales come back as the bytes that they are held in."""
import math
import random

import torch

own = False

DEV = "cuda"
GROUP = 16                                              # channels that share a scale
LEAST, MOST = 2.0 ** -14, 10240.0                       # the scales that a store writes
HALVES, PAIRS = 0, 1                                    # channels i and i + R / 2 are a pair, or 2 i and 2 i + 1
PLAIN, LINEAR, BY_PARTS = 0, 1, 2                       # how frequencies are scaled


def listed():
    return [
        # every decode step: one layer's new queries and keys of four sequences, context stretched fourfold
        dict(name="rotary_step", op="rotary", units=4, q_heads=64, heads=8, dim=128, rows=1, part=128, layout=HALVES, adjoint=False,
             axes=1, scaling=BY_PARTS, base=1000000.0, far=131072, dtype="bf16"),
        # the gradient of a small fp32 layer whose heads are turned in part, neighbouring channels as pairs
        dict(name="rotary_part", op="rotary", units=2, q_heads=4, heads=4, dim=64, rows=577, part=32, layout=PAIRS, adjoint=True,
             axes=1, scaling=LINEAR, base=10000.0, far=8192, dtype="f32"),
        # prefill of one long image prompt, a layer: three positions a token
        dict(name="rotary_prompt", op="rotary", units=1, q_heads=64, heads=8, dim=128, rows=33792, part=128, layout=HALVES, adjoint=False,
             axes=3, scaling=PLAIN, base=1000000.0, far=40000, dtype="bf16"),
        # the row that a decode step adds, one layer of four sequences
        dict(name="store_append", op="store", units=4, heads=8, dim=128, page=64, new=1, held=1690, dtype="bf16"),
        # a small fp32 layer with heads of 64, just compressed
        dict(name="store_fp32_small", op="store", units=1, heads=4, dim=64, page=16, new=48, held=0, dtype="f32"),
        # compressed caches of 20 layers of four long sequences
        dict(name="store_stack", op="store", units=80, heads=8, dim=128, page=64, new=1690, held=0, dtype="bf16"),
        # a stack's caches that have grown to different lengths, read back before they are compressed again
        dict(name="load_stack_small", op="load", units=28, heads=4, dim=128, page=64, most=640, dtype="bf16"),
        # the same of 20 layers of four long sequences
        dict(name="load_stack", op="load", units=80, heads=8, dim=128, page=64, most=1690, dtype="bf16"),
        # a decode step of one layer over its compressed cache, a single sequence
        dict(name="attention_one", op="attention", units=1, heads=4, group=7, dim=128, page=64, most=218, dtype="bf16"),
        # small fp32 heads of 64
        dict(name="attention_fp32_small", op="attention", units=4, heads=4, group=1, dim=64, page=16, most=192, dtype="f32"),
        # a batch of compressed long sequences of different lengths
        dict(name="attention_batch", op="attention", units=64, heads=8, group=8, dim=128, page=64, most=1690, dtype="bf16"),
        # full long caches, 16 sequences of different lengths: the large end
        dict(name="attention_long", op="attention", units=16, heads=8, group=8, dim=128, page=128, most=33792, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# Rows times heads of a drawn case: below the largest listed one's.
MOST_ROTARY, MOST_STORE, MOST_ATTENTION = 72 * 33000, 80 * 8 * 1690, 16 * 8 * 16000
LAYOUTS = [(4, 1, 64, "f32"), (32, 1, 128, "bf16"), (4, 7, 128, "bf16"), (8, 8, 128, "bf16"), (8, 8, 128, "bf16"), (2, 5, 128, "bf16"),
           (8, 4, 64, "bf16"), (4, 2, 128, "f32")]      # KV heads, query heads of each, channels, type


def draw(rng):
    op = rng.choice(["rotary", "rotary", "store", "store", "load", "attention", "attention", "attention"])
    heads, group, dim, dtype = rng.choice(LAYOUTS)
    if op == "rotary":
        rows = rng.choice([1, 1, rng.randint(2, 9), _log_int(rng, 10, 33792)])
        all_heads = heads * (group + 1)
        units = max(1, min(_log_int(rng, 1, 320), MOST_ROTARY // (all_heads * rows * (2 if dtype == "f32" else 1))))
        part = rng.choice([dim, dim, dim // 2, dim // 4])
        return dict(op=op, units=units, q_heads=heads * group, heads=heads, dim=dim, rows=rows, part=part, layout=rng.choice([HALVES, PAIRS]),
                    adjoint=rng.random() < 0.3, axes=rng.choice([1, 1, 3]), scaling=rng.choice([PLAIN, LINEAR, BY_PARTS]),
                    base=rng.choice([10000.0, 500000.0, 1000000.0]), far=_log_int(rng, rows, 1 << 20), dtype=dtype)
    page = rng.choice([16, 32, 64, 64, 128])
    if op == "attention":
        most = _log_int(rng, 1, 33792) if dim == 128 else _log_int(rng, 1, 2200)
        units = _log_int(rng, 1, 320)
        return dict(op=op, units=max(1, min(units, MOST_ATTENTION // (heads * most))), heads=heads, group=group, dim=dim, page=page, most=most, dtype=dtype)
    most = _log_int(rng, 1, 8000) if dim == 128 else _log_int(rng, 1, 1000)
    units = max(1, min(_log_int(rng, 1, 320), MOST_STORE // (heads * most * (2 if dtype == "f32" else 1))))
    if op == "load":
        return dict(op=op, units=units, heads=heads, dim=dim, page=page, most=most, dtype=dtype)
    held = rng.choice([0, 0, rng.randint(1, 300)])
    new = rng.choice([1, 1, rng.randint(2, 9), most])
    units = _log_int(rng, 1, 320) if new < 10 else units
    return dict(op=op, units=units, heads=heads, dim=dim, page=page, new=new, held=held, dtype=dtype)


def _pages(n, page):
    return (n + page - 1) // page


def _lengths(case, seed):
    """Rows of every unit: the longest as the case says, the others anything from an eighth of it."""
    rng = random.Random("%d rows" % seed)
    most = case["most"]
    rows = [rng.randint(max(1, most // 8), most) for _ in range(case["units"])]
    rows[rng.randrange(len(rows))] = most
    return rows


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _gauss(gen, shape, keys):
    """What keys and values look like: keys with a few strong channels, values off centre."""
    x = torch.randn(shape, generator=gen, device=DEV)
    if keys:
        x[..., ::37] *= 4.0
        return x
    return x.mul_(1.5).add_(0.5)


def _pool(gen, n_pages, heads, page, dim, rows, table, keys):
    """Pages that hold rows, and bytes of any kind behind them."""
    codes = torch.randint(0, 256, (n_pages, heads, page, dim // 2), generator=gen, device=DEV, dtype=torch.uint8)
    scales = torch.randint(0, 256, (n_pages, heads, page, dim // GROUP), generator=gen, device=DEV, dtype=torch.uint8)
    step = max(1, (1 << 26) // (heads * page * dim))
    left = torch.zeros(n_pages, dtype=torch.int64, device=DEV)
    at = torch.arange(table.shape[1], device=DEV)
    held = (rows.long().unsqueeze(1) - at * page).clamp(0, page)
    left[table.long()[held > 0]] = held[held > 0]
    for i in range(0, n_pages, step):
        n = left[i:i + step]
        there = (torch.arange(page, device=DEV) < n.unsqueeze(1))[:, None, :, None]
        c, s = _quantised(_gauss(gen, (n.numel(), heads, page, dim), keys))
        codes[i:i + step] = torch.where(there, c, codes[i:i + step])
        scales[i:i + step] = torch.where(there, s, scales[i:i + step])
    return codes, scales


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    rng = random.Random(seed)
    op = case["op"]
    s = dict(op=op, case=case)
    F = None
    if own:
        from paper_2511_05534_b200 import binding as F
        s["F"] = F
    tdt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    dtype = F and (F.BF16 if tdt == torch.bfloat16 else F.F32)
    if op == "rotary":
        _prepare_rotary(s, case, gen, rng, F, tdt, dtype)
        return s
    page, U, H, D = case["page"], case["units"], case["heads"], case["dim"]
    if op == "store":
        held = [case["held"] if case["new"] > 9 else rng.randint(0, max(0, 2 * case["held"])) for _ in range(U)]
        rows = [r + case["new"] for r in held]
    else:
        held = rows = _lengths(case, seed)
    wide = max(_pages(r, page) for r in rows)
    n_pages = (U * _pages(2 * case["held"] + case["new"], page) if op == "store" else sum(_pages(r, page) for r in rows)) + 7
    order = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    count = torch.tensor([_pages(r, page) for r in rows], device=DEV)
    at = torch.arange(wide, device=DEV)
    first = count.cumsum(0) - count
    table = torch.where(at < count.unsqueeze(1), order[(first.unsqueeze(1) + at).clamp(max=n_pages - 1)], torch.zeros((), dtype=torch.int32, device=DEV))
    s["table"] = table.contiguous()
    s["rows"] = _ints(rows)
    for name in "kv":
        s[name + "_pages"], s[name + "_scale"] = _pool(gen, n_pages, H, page, D, _ints(held), table, name == "k")
    n_rows = 0
    if op == "store":
        n_rows = case["new"]
        s["k"], s["v"] = (_gauss(gen, (U, H, n_rows, D), name == "k").to(tdt) for name in "kv")
        pos = _ints(held).long().unsqueeze(1) + torch.arange(n_rows, device=DEV)
        s["slots"] = (table.long().gather(1, pos // page) * page + pos % page).to(torch.int32)
    elif op == "load":
        n_rows = max(rows)
        s["k"], s["v"] = (torch.zeros((U, H, n_rows, D), dtype=tdt, device=DEV) for _ in "kv")
    else:
        s["q"] = torch.randn((U, H * case["group"], D), generator=gen, device=DEV).to(tdt)
        s["out"] = torch.empty_like(s["q"])
    if own:
        s["p"] = F.CacheParams(U, H * case.get("group", 1), H, D, page, n_pages, wide, n_rows, dtype=dtype)
        s["ws"] = F.alloc_nibble_workspace(s["p"])
    return s


def _sections(case):
    """How many of the pairs go by each of three positions: a quarter by the first, the others in equal parts."""
    n = case["part"] // 2
    first = n // 4
    second = (n - first) // 2
    return [first, second, n - first - second] if case["axes"] == 3 else [n]


# the numbers of a model whose context was stretched
FACTOR, LOW, HIGH, TRAINED, AMPLITUDE = 4.0, 1.0, 32.0, 32768, 1.1386


def _prepare_rotary(s, case, gen, rng, F, tdt, dtype):
    U, Hq, H, D, T = (case[x] for x in ("units", "q_heads", "heads", "dim", "rows"))
    s["q"] = torch.randn((U, Hq, T, D), generator=gen, device=DEV).to(tdt)
    s["k"] = _gauss(gen, (U, H, T, D), True).to(tdt)
    s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
    start = torch.tensor([[[rng.randint(0, case["far"] - T)] for _ in range(case["axes"])] for _ in range(U)], device=DEV)
    s["positions"] = (start + torch.arange(T, device=DEV) // torch.tensor([1, 32, 7][:case["axes"]], device=DEV).unsqueeze(1)).to(torch.int32)
    if own:
        section = _sections(case)
        s["p"] = F.RotaryParams(U, Hq, H, D, T, dtype=dtype, rotary_dim=case["part"], layout=F.ROTARY_PAIRS if case["layout"] == PAIRS else F.ROTARY_HALVES,
                                adjoint=case["adjoint"], sections=section if case["axes"] == 3 else None,
                                scaling=[F.ROTARY_PLAIN, F.ROTARY_LINEAR, F.ROTARY_BY_PARTS][case["scaling"]], base=case["base"], factor=FACTOR,
                                low=LOW, high=HIGH, trained=TRAINED, amplitude=AMPLITUDE if case["scaling"] == BY_PARTS else 1.0)
        s["phases"] = F.alloc_rotary_table(s["p"])


def run(state):
    return {"rotary": _run_rotary, "store": _run_store, "load": _run_load, "attention": _run_attention}[state["op"]](state)


def _run_rotary(s):
    """Returns the turned queries and keys."""
    if own:
        s["F"].flowmm_rotary(s["p"], s["q"], s["k"], s["positions"], s["phases"], s["q_out"], s["k_out"])
        return s["q_out"], s["k_out"]
    case = s["case"]
    R = case["part"]
    i = torch.arange(R // 2, device=DEV, dtype=torch.float64)
    freq = case["base"] ** (-2 * i / R)
    if case["scaling"] == LINEAR:
        freq = freq / FACTOR
    elif case["scaling"] == BY_PARTS:
        kept = ((TRAINED * freq / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0, 1)
        freq = freq * (kept + (1 - kept) / FACTOR)
    axis = torch.cat([torch.full((n,), a, device=DEV) for a, n in enumerate(_sections(case))])
    angle = s["positions"].double()[:, axis] * freq[:, None]                    # [U, R / 2, T]
    m = AMPLITUDE if case["scaling"] == BY_PARTS else 1.0
    c, d = (m * torch.cos(angle)).float().transpose(1, 2), (m * torch.sin(angle)).float().transpose(1, 2)
    if case["adjoint"]:
        d = -d
    return tuple(_turned(s[name], c[:, None], d[:, None], R, case["layout"]) for name in "qk")


def _turned(x, c, d, R, layout):
    turn, rest = x[..., :R].float(), x[..., R:]
    if layout == HALVES:
        a, b = turn[..., :R // 2], turn[..., R // 2:]
        y = torch.cat([a * c - b * d, b * c + a * d], -1)
    else:
        a, b = turn[..., ::2], turn[..., 1::2]
        y = torch.stack([a * c - b * d, b * c + a * d], -1).flatten(-2)
    return torch.cat([y.to(x.dtype), rest], -1)


def _four_bits(x):
    """float64 rounded to four significant bits, ties to even."""
    m, e = torch.frexp(x)
    return torch.ldexp(torch.round(m * 16) / 16, e)


def _quantised(x):
    """(bytes of two codes, bytes of scales) of rows [..., D].  Quotients in 64 bits: some lie next to a border between codes."""
    g = x.unflatten(-1, (-1, GROUP)).double()
    size = g.abs().amax(-1)
    s = _four_bits(size / 6).clamp(LEAST, MOST)
    bad = ~torch.isfinite(g).all(-1)
    scale = torch.where(bad, 255, (s.float().view(torch.int32) >> 20) - 896).to(torch.uint8)     # the exponent with a bias of 15, three bits of mantissa
    y = (g / s.unsqueeze(-1)).abs()
    code = sum((y > border).to(torch.uint8) if tie_down else (y >= border).to(torch.uint8)
               for border, tie_down in ((0.25, True), (0.75, False), (1.25, True), (1.75, False), (2.5, True), (3.5, False), (5.0, True)))
    code = torch.where(bad.unsqueeze(-1), 0, code | torch.signbit(g).to(torch.uint8) << 3).flatten(-2)
    return code[..., ::2] | code[..., 1::2] << 4, scale


def _run_store(s):
    """Returns the pools and their scales."""
    if own:
        s["F"].flowmm_nibble_store(s["p"], s["k"], s["v"], s["slots"], s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["ws"])
    else:
        page = s["case"]["page"]
        for u in range(0, s["slots"].shape[0], 8):
            slots = s["slots"][u:u + 8].long()
            for name in "kv":
                codes, scale = _quantised(s[name][u:u + 8])
                s[name + "_pages"][slots // page, :, slots % page] = codes.transpose(1, 2)
                s[name + "_scale"][slots // page, :, slots % page] = scale.transpose(1, 2)
    return s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"]


def _run_load(s):
    """Returns the dense rows; those behind a unit's last row are left as they were."""
    if own:
        s["F"].flowmm_nibble_load(s["p"], s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["table"], s["rows"], s["k"], s["v"], s["ws"])
        return s["k"], s["v"]
    there = (torch.arange(s["k"].shape[2], device=DEV) < s["rows"].unsqueeze(1))[:, None, :, None]
    return tuple(torch.where(there, _dense(s, name)[:, :, :s[name].shape[2]].to(s[name].dtype), s[name]) for name in "kv")


def _dense(s, name):
    """[units, KV heads, pages * page size, head_dim] float32."""
    ids = s["table"].long()
    codes, scale = s[name + "_pages"][ids], s[name + "_scale"][ids]
    sizes = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=DEV)
    values = torch.cat([sizes, -sizes])
    x = values[torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()]
    x = x.unflatten(-1, (-1, GROUP)) * (scale.to(torch.int16) << 7).view(torch.float16).float().unsqueeze(-1)
    x = x.flatten(-2)
    U, n, H, page, D = x.shape
    return x.transpose(1, 2).reshape(U, H, n * page, D)


def _run_attention(s):
    if own:
        s["F"].flowmm_nibble_attention(s["p"], s["q"], s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["table"], s["rows"], s["out"], s["ws"])
        return s["out"]
    U, Hq, D = s["q"].shape
    H = s["k_pages"].shape[1]
    k = _dense(s, "k")
    there = torch.arange(k.shape[2], device=DEV) < s["rows"].unsqueeze(1)
    z = torch.matmul(s["q"].float().view(U, H, Hq // H, D), k.transpose(2, 3)) * D ** -0.5
    del k
    z = torch.where(there[:, None, None], z, torch.full_like(z, -math.inf))
    w = torch.exp(z - z.amax(3, keepdim=True))
    v = torch.where(there[:, None, :, None], _dense(s, "v"), torch.zeros((), device=DEV))
    return (torch.matmul(w, v) / w.sum(3, keepdim=True)).view(U, Hq, D).to(s["q"].dtype)


def work(case):
    U, H, D = case["units"], case["heads"], case["dim"]
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "rotary":
        rows = U * (case["q_heads"] + H) * case["rows"]
        return {"bytes": 2 * rows * D * size + 4 * U * case["axes"] * case["rows"], "flops": 3 * rows * case["part"]}
    page, row = case["page"], D // 2 + D // GROUP                        # bytes of a row in a page
    if case["op"] == "store":
        rows = U * case["new"]
        return {"bytes": 2 * H * rows * (D * size + row) + 4 * rows, "flops": 2 * 2 * H * rows * D}
    most = case["most"]
    rows = most + (U - 1) * (most + max(1, most // 8)) // 2
    read = 2 * H * rows * row + 4 * _pages(rows, page) + 4 * U
    if case["op"] == "load":
        return {"bytes": read + 2 * H * rows * D * size, "flops": 2 * H * rows * D}
    Hq = H * case["group"]
    return {"bytes": read + U * Hq * D * 2 * size, "flops": 4 * Hq * rows * D}


# ---- the same from the definitions, in 64 bits ---------------------------------------------------


def _numbers(bits):
    """What a byte stands for, as float64: a table over all bytes of codes (4 bits) or of scales (8 bits)."""
    out = []
    for b in range(16 if bits == 4 else 256):
        if bits == 4:
            e, m = (b >> 1) & 3, b & 1
            size = (1 + m / 2) * 2.0 ** (e - 1) if e else m / 2
            out.append(-size if b & 8 else size)
        else:
            e, m = b >> 3, b & 7
            out.append((math.inf if m == 0 else math.nan) if e == 31 else (1 + m / 8) * 2.0 ** (e - 15) if e else m / 8 * 2.0 ** -14)
    return torch.tensor(out, dtype=torch.float64, device=DEV)


def exact(case, seed):
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "store": _exact_store, "load": _exact_load, "attention": _exact_attention}[case["op"]](s)


def _exact_rotary(s):
    case = s["case"]
    R, T = case["part"], case["rows"]
    axis = [a for a, n in enumerate(_sections(case)) for _ in range(n)]
    m = AMPLITUDE if case["scaling"] == BY_PARTS else 1.0
    out = s["q"].double(), s["k"].double()
    for i in range(R // 2):
        f = case["base"] ** (-2.0 * i / R)
        if case["scaling"] == LINEAR:
            f /= FACTOR
        if case["scaling"] == BY_PARTS:
            g = min(1.0, max(0.0, (TRAINED * f / (2 * math.pi) - LOW) / (HIGH - LOW)))
            f = g * f + (1 - g) * f / FACTOR
        angle = s["positions"][:, axis[i]].double() * (-f if case["adjoint"] else f)
        turn = torch.polar(torch.full_like(angle, m), angle).unsqueeze(1)       # [U, 1, T]
        at = (i, i + R // 2) if case["layout"] == HALVES else (2 * i, 2 * i + 1)
        for x in out:
            y = torch.complex(x[..., at[0]], x[..., at[1]]) * turn
            x[..., at[0]], x[..., at[1]] = y.real, y.imag
    return out


def _exact_store(s):
    """The nearest of all 16 codes, the even one of two that are as near; the scale the nearest of those that a store may write."""
    page = s["case"]["page"]
    number = _numbers(8)
    first, last = 8, 226                                                # the bytes of 2^-14 and 10240
    writable = number[first:last + 1]
    even = torch.arange(first, last + 1, device=DEV) % 2 == 0
    positive = _numbers(4)[:8]
    out = []
    for name in "kv":
        pages, scales = s[name + "_pages"].clone(), s[name + "_scale"].clone()
        for u in range(s["slots"].shape[0]):
            x = s[name][u].double()                                     # [H, T, D]
            H, T, D = x.shape
            g = x.view(H, T, D // GROUP, GROUP)
            want = g.abs().amax(3) / 6
            hi = torch.searchsorted(writable, want.flatten()).clamp(max=writable.numel() - 1).view(want.shape)
            lo = (hi - 1).clamp(min=0)
            up, down = (writable[hi] - want).abs(), (want - writable[lo]).abs()
            pick = torch.where((up < down) | ((up == down) & even[hi]), hi, lo)
            y = g / writable[pick].unsqueeze(3)
            dist = (y.abs().unsqueeze(4) - positive).abs()
            near = dist.argmin(4)                                       # the lower of two
            tied = dist.gather(4, (near + 1).clamp(max=7).unsqueeze(4)).squeeze(4) == dist.gather(4, near.unsqueeze(4)).squeeze(4)
            near = torch.where(tied & (near % 2 == 1) & (near < 7), near + 1, near)
            code = (near + 8 * torch.signbit(y)).view(H, T, D)
            slot = s["slots"][u].long()
            byte = (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8)
            for h in range(H):
                pages[slot // page, h, slot % page] = byte[h]
                scales[slot // page, h, slot % page] = (pick[h] + first).to(torch.uint8)
        out.append((pages, scales))
    return out[0][0], out[1][0], out[0][1], out[1][1]


def _unit(s, name, u, n):
    """[KV heads, n, head_dim] float64: the unit's first n rows."""
    page = s["case"]["page"]
    ids = s["table"][u, :_pages(n, page)].long()
    codes, scale = s[name + "_pages"][ids].long(), s[name + "_scale"][ids].long()
    x = torch.empty(*codes.shape[:3], 2 * codes.shape[3], dtype=torch.float64, device=DEV)
    x[..., 0::2], x[..., 1::2] = _numbers(4)[codes % 16], _numbers(4)[codes // 16]
    x *= _numbers(8)[scale].repeat_interleave(GROUP, 3)
    return x.transpose(0, 1).flatten(1, 2)[:, :n]


def _exact_load(s):
    out = tuple(s[name].double() for name in "kv")
    for u, n in enumerate(s["rows"].tolist()):
        for x, name in zip(out, "kv"):
            x[u, :, :n] = _unit(s, name, u, n)
    return out


def _exact_attention(s):
    U, Hq, D = s["q"].shape
    out = torch.zeros((U, Hq, D), dtype=torch.float64, device=DEV)
    for u, n in enumerate(s["rows"].tolist()):
        k, v = _unit(s, "k", u, n), _unit(s, "v", u, n)
        q = s["q"][u].double().view(k.shape[0], -1, D)
        w = torch.softmax(torch.einsum("hgd,hnd->hgn", q, k) / math.sqrt(D), 2)
        out[u] = torch.einsum("hgn,hnd->hgd", w, v).reshape(Hq, D)
    return out
