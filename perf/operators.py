"""The paged 8-bit cache's operators, as timed cases, with their plain forms.

  plan       flowmm_cache_plan: block tables and slot maps from the lengths of the requests
  store      flowmm_cache_store: rows of K and V into pages, e4m3 codes with one power-of-two scale per page and KV head
  load       flowmm_cache_load: pages back into dense rows, as flowmm_recompress takes them
  attention  flowmm_cache_attention: one new query per query head over the pages of every unit, lengths of their own

A unit is one (layer, sequence) pair, as in the rest of the library.  Head layouts, lengths and budgets are those of
`configs.WORKLOADS`.  Rows that no sequence holds (behind a unit's last row, pages nobody owns) hold arbitrary bytes, codes of
NaN among them, as memory that earlier requests have left does."""
import math
import random

import torch

own = False

DEV = "cuda"
E4M3 = torch.float8_e4m3fn
LOWEST, TOP = -96, 448.0                                # exponent of the smallest scale; the largest code


def listed():
    return [
        # every decode step: 48 sequences in service, each grows by a row, a few have ended and give their pages back
        dict(name="plan_step", op="plan", units=48, page=64, most=33792, grow=1, ended=4),
        # admission of compressed caches: all 80 layers of 4 sequences get the pages of 1690 rows
        dict(name="plan_admit", op="plan", units=320, page=64, most=1690, grow=1690, ended=0),
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
        # multi-head attention (a query head per KV head), eight sequences of up to a whole image prompt
        dict(name="attention_mha", op="attention", units=8, heads=32, group=1, dim=128, page=32, most=640, dtype="bf16"),
        # a batch of compressed long sequences of different lengths
        dict(name="attention_batch", op="attention", units=64, heads=8, group=8, dim=128, page=64, most=1690, dtype="bf16"),
        # full long caches, 16 sequences of different lengths: the large end
        dict(name="attention_long", op="attention", units=16, heads=8, group=8, dim=128, page=128, most=33792, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# Rows times KV heads of a drawn case: below the largest listed one's.
MOST_STORE, MOST_ATTENTION = 80 * 8 * 1690, 16 * 8 * 16000


def draw(rng):
    op = rng.choice(["plan", "store", "store", "load", "attention", "attention", "attention"])
    page = rng.choice([16, 32, 64, 64, 128])
    if op == "plan":
        if rng.random() < 0.5:
            units = _log_int(rng, 1, 2000)
            return dict(op=op, units=units, page=page, most=_log_int(rng, 64, 8000), grow=rng.choice([1, 1, 2, 5]), ended=units // rng.randint(8, 40))
        grow = _log_int(rng, 16, 1690)
        return dict(op=op, units=min(_log_int(rng, 1, 320), 320 * 1690 // grow), page=page, most=grow + rng.choice([0, rng.randint(1, 500)]), grow=grow, ended=0)
    heads, group, dim, dtype = rng.choice([(4, 1, 64, "f32"), (32, 1, 128, "bf16"), (4, 7, 128, "bf16"), (8, 8, 128, "bf16"), (8, 8, 128, "bf16"),
                                           (2, 5, 128, "bf16"), (8, 4, 64, "bf16")])
    if op == "attention":
        most = _log_int(rng, 1, 33792) if dim == 128 else _log_int(rng, 1, 2200)
        units = _log_int(rng, 1, 320)
        return dict(op=op, units=max(1, min(units, MOST_ATTENTION // (heads * most))), heads=heads, group=group, dim=dim, page=page, most=most, dtype=dtype)
    most = _log_int(rng, 1, 8000) if dim == 128 else _log_int(rng, 1, 1000)
    units = max(1, min(_log_int(rng, 1, 320), MOST_STORE // (heads * most)))
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
    codes = torch.randint(0, 256, (n_pages, heads, page, dim), generator=gen, device=DEV, dtype=torch.uint8)
    scales = torch.full((n_pages, heads), 2.0 ** LOWEST, device=DEV)
    step = max(1, (1 << 27) // (heads * page * dim))
    left = torch.zeros(n_pages, dtype=torch.int64, device=DEV)
    at = torch.arange(table.shape[1], device=DEV)
    held = (rows.long().unsqueeze(1) - at * page).clamp(0, page)
    left[table.long()[held > 0]] = held[held > 0]
    for i in range(0, n_pages, step):
        n = left[i:i + step]
        x = _gauss(gen, (n.numel(), heads, page, dim), keys)
        there = (torch.arange(page, device=DEV) < n.unsqueeze(1))[:, None, :, None]
        amax = torch.where(there, x.abs(), torch.zeros_like(x)).amax((2, 3))
        s = _scale_of(amax)
        q = (x / s[:, :, None, None]).to(E4M3).view(torch.uint8)
        codes[i:i + step] = torch.where(there, q, codes[i:i + step])
        scales[i:i + step] = s
    return codes.view(E4M3), scales


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    rng = random.Random(seed)
    op, page, U = case["op"], case["page"], case["units"]
    s = dict(op=op, case=case)
    F = None
    if own:
        from paper_2511_05534_b200 import binding as F
        s["F"] = F
    if op == "plan":
        _prepare_plan(s, case, rng, F)
        return s
    H, D = case["heads"], case["dim"]
    tdt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    if op == "store":
        rows = [case["held"] if case["new"] > 9 else rng.randint(0, max(0, 2 * case["held"])) for _ in range(U)]
        held = rows
        rows = [r + case["new"] for r in rows]
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
        s["out"] = torch.empty((U, H * case["group"], D), dtype=torch.float32, device=DEV)
    if own:
        s["p"] = F.CacheParams(U, H * case.get("group", 1), H, D, page, n_pages, wide, n_rows, dtype=F.BF16 if tdt == torch.bfloat16 else F.F32)
        s["ws"] = F.alloc_cache_workspace(s["p"])
    return s


def _prepare_plan(s, case, rng, F):
    page, U, grow = case["page"], case["units"], case["grow"]
    if grow > 9:                                            # admission: units without a row, or with a few
        rows = [rng.randint(0, case["most"] - grow) if case["most"] > grow else 0 for _ in range(U)]
    else:
        rows = [rng.randint(max(1, case["most"] // 8), case["most"]) for _ in range(U)]
    ended = set(rng.sample(range(U), case["ended"]))
    add = [-rows[u] if u in ended else grow for u in range(U)]
    held = [_pages(r, page) for r in rows]
    n_pages = U * _pages(case["most"] + (grow if grow < 10 else 0), page) + 21
    wide = _pages(case["most"] + grow, page)
    perm = list(range(n_pages))
    rng.shuffle(perm)
    table, at = [], 0
    for h in held:
        table.append(perm[at:at + h] + [0] * (wide - h))
        at += h
    free = perm[at:]
    head = rng.randrange(n_pages)
    ring = [0] * n_pages
    for i, x in enumerate(free):
        ring[(head + i) % n_pages] = x
    s.update(rows=_ints(rows), grow=_ints(add), ring=_ints(ring), state=_ints([head, len(free)]), table=_ints(table),
             rows_out=_ints([0] * U), state_out=_ints([0, 0]), slots=_ints([[0] * grow] * U))
    if own:
        s["p"] = F.CacheParams(U, 1, 1, 128, page, n_pages, wide, grow)
        s["ws"] = F.alloc_cache_workspace(s["p"])


def run(state):
    return {"plan": _run_plan, "store": _run_store, "load": _run_load, "attention": _run_attention}[state["op"]](state)


def _run_plan(s):
    """Returns (rows, state of the ring, table, ring, slots) after the step.  The rows and the ring's state go to arrays of their
    own, so that the step can be planned again from the same ones."""
    if own:
        s["F"].flowmm_cache_plan(s["p"], s["grow"], s["rows"], s["rows_out"], s["ring"], s["state"], s["state_out"], s["table"], s["slots"], s["ws"])
        return s["rows_out"], s["state_out"], s["table"], s["ring"], s["slots"]
    page, ring, table = s["case"]["page"], s["ring"], s["table"]
    U, wide = table.shape
    T, n = s["slots"].shape[1], ring.numel()
    rows, grow = s["rows"].long(), s["grow"].long()
    head, count = s["state"].long().unbind()
    new = (rows + grow).clamp(min=0)
    held, want = (rows + page - 1) // page, (new + page - 1) // page
    fits = (new <= wide * page) & (grow <= T)
    need = torch.where(fits, (want - held).clamp(min=0), 0)
    upto = need.cumsum(0)
    ok = fits & ((need == 0) | (upto <= count))
    taken = torch.where(ok & (need > 0), upto, 0).max()
    back = torch.where(ok, (held - want).clamp(min=0), 0)
    j = torch.arange(wide, device=DEV)
    mine = ok.unsqueeze(1) & (j >= held.unsqueeze(1)) & (j < want.unsqueeze(1))
    at = (head + (upto - need).unsqueeze(1) + j - held.unsqueeze(1)) % n
    out_table = torch.where(mine, ring[at], table)
    given = ok.unsqueeze(1) & (j >= want.unsqueeze(1)) & (j < held.unsqueeze(1))
    to = (head + count + (back.cumsum(0) - back).unsqueeze(1) + j - want.unsqueeze(1)) % n
    marked = torch.zeros(n + 1, dtype=torch.bool, device=DEV)
    marked[torch.where(given, to, n)] = True
    value = torch.zeros(n + 1, dtype=torch.int32, device=DEV)
    value[torch.where(given, to, n)] = table
    out_ring = torch.where(marked[:n], value[:n], ring)
    t = torch.arange(T, device=DEV)
    pos = rows.unsqueeze(1) + t
    fresh = ok.unsqueeze(1) & (t < grow.unsqueeze(1))
    ids = out_table.gather(1, (pos // page).clamp(max=wide - 1)).long()
    slots = torch.where(fresh, ids * page + pos % page, -1).to(torch.int32)
    left = torch.stack([(head + taken) % n, count - taken + back.sum()]).to(torch.int32)
    return torch.where(ok, new, rows).to(torch.int32), left, out_table, out_ring, slots


def _scale_of(amax):
    """The power of two that takes amax to at most 448 = 0.875 * 2^9."""
    m, e = torch.frexp(amax)
    e = torch.where(amax > 0, e - 9 + (m > 0.875).to(e.dtype), LOWEST).clamp(min=LOWEST)
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _run_store(s):
    """Returns the pools and their scales (codes as the e4m3 numbers they are, to be multiplied by their page's scale)."""
    if own:
        s["F"].flowmm_cache_store(s["p"], s["k"], s["v"], s["slots"], s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["ws"])
    else:
        for name in "kv":
            _store(s[name], s["slots"], s[name + "_pages"], s[name + "_scale"])
    return s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"]


def _store(x, slots, pages, scale):
    U, H, T, D = x.shape
    page = pages.shape[2]
    first = slots[:, :1].long() % page                              # rows that the first page holds already
    n = (T + 2 * page - 2) // page                                  # pages that T rows can touch
    at = torch.arange(n * page, device=DEV) - first                 # [U, n * page]: the new row at each place of those pages
    fresh = (at >= 0) & (at < T)
    old = (at < 0).view(U, 1, n, page, 1)
    src = at.clamp(0, T - 1)
    ids = torch.where(fresh, slots.long().gather(1, src) // page, -1).view(U, n, page).amax(2)
    img = x.float().gather(2, src[:, None, :, None].expand(U, H, n * page, D)).view(U, H, n, page, D)
    fresh = fresh.view(U, 1, n, page, 1)
    size = torch.where(fresh & torch.isfinite(img), img.abs(), torch.zeros_like(img)).amax((3, 4))
    want = _scale_of(size)
    had, codes = scale[ids.clamp(min=0)].transpose(1, 2), pages.view(torch.uint8)[ids.clamp(min=0)].transpose(1, 2)
    goes_on = old.any(3).squeeze(-1)                                # [U, 1, n]
    new = torch.where(goes_on, torch.maximum(want, had), want)
    kept = (codes.view(E4M3).float() * (had / new)[..., None, None]).to(E4M3).view(torch.uint8)
    put = (img / new[..., None, None]).to(E4M3).view(torch.uint8)
    codes = torch.where(fresh, put, torch.where(old, kept, codes)).transpose(1, 2)
    there = ids >= 0
    pages.view(torch.uint8)[ids[there]] = codes[there]
    scale[ids[there]] = new.transpose(1, 2)[there]


def _run_load(s):
    """Returns the dense rows; those behind a unit's last row are left as they were."""
    if own:
        s["F"].flowmm_cache_load(s["p"], s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["table"], s["rows"], s["k"], s["v"], s["ws"])
        return s["k"], s["v"]
    there = (torch.arange(s["k"].shape[2], device=DEV) < s["rows"].unsqueeze(1))[:, None, :, None]
    return tuple(torch.where(there, _dense(s, name)[:, :, :s[name].shape[2]].to(s[name].dtype), s[name]) for name in "kv")


def _dense(s, name):
    """[units, KV heads, pages * page size, head_dim] float32."""
    ids = s["table"].long()
    x = s[name + "_pages"].view(torch.uint8)[ids].view(E4M3).float() * s[name + "_scale"][ids][..., None, None]
    U, n, H, page, D = x.shape
    return x.transpose(1, 2).reshape(U, H, n * page, D)


def _run_attention(s):
    if own:
        s["F"].flowmm_cache_attention(s["p"], s["q"], s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["table"], s["rows"], s["out"], s["ws"])
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
    return (torch.matmul(w, v) / w.sum(3, keepdim=True)).view(U, Hq, D)


def work(case):
    page, U = case["page"], case["units"]
    if case["op"] == "plan":
        new = case["grow"] * U if case["grow"] > 9 else U
        table = U * _pages(case["grow"], page) if case["grow"] > 9 else _pages(U, page)
        back = case["ended"] * _pages(case["most"] * 9 // 16, page)
        return {"bytes": 4 * (3 * U + new + 2 * table + 2 * back + 4), "flops": 0}
    H, D = case["heads"], case["dim"]
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "store":
        rows = U * case["new"]
        return {"bytes": 2 * H * rows * D * (size + 1) + 4 * rows + 8 * H * U * _pages(case["new"], page), "flops": 2 * 2 * H * rows * D}
    most = case["most"]
    rows = most + (U - 1) * (most + max(1, most // 8)) // 2
    pages = _pages(rows, page)
    read = 2 * H * rows * D + 8 * H * pages + 4 * pages + 4 * U
    if case["op"] == "load":
        return {"bytes": read + 2 * H * rows * D * size, "flops": 2 * H * rows * D}
    Hq = H * case["group"]
    return {"bytes": read + U * Hq * D * (size + 4), "flops": 4 * case["group"] * H * rows * D}


# ---- the same from the definitions, in 64 bits ---------------------------------------------------


def _two(e):
    """2^e as float64, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _number(codes):
    """e4m3 codes as float64: sign, four exponent bits of bias 7, three mantissa bits; 127 and 255 are NaN."""
    c = torch.arange(256, dtype=torch.int64)
    e, m = (c >> 3) & 15, (c & 7).double()
    size = torch.where(e > 0, (1 + m / 8) * _two(e - 7), m * 2.0 ** -9)
    size[(c & 127) == 127] = math.nan
    return torch.where(c > 127, -size, size).to(codes.device)[codes.view(torch.uint8).long()]


def _nearest(x):
    """float64 numbers of at most 448 in size rounded to e4m3, ties to even; what is not finite becomes NaN."""
    m, e = torch.frexp(x.abs())
    step = _two(e.clamp(min=-5) - 4)      # four significant bits, 2^-9 at least
    r = torch.round(x / step) * step
    return torch.where(torch.isfinite(x), r, torch.full_like(r, math.nan))


def exact(case, seed):
    s = prepare(case, seed)
    return {"plan": _exact_plan, "store": _exact_store, "load": _exact_load, "attention": _exact_attention}[case["op"]](s)


def _exact_plan(s):
    page = s["case"]["page"]
    rows, grow, ring, table = (s[x].tolist() for x in ("rows", "grow", "ring", "table"))
    head, count = s["state"].tolist()
    n, wide, T = len(ring), len(table[0]), s["slots"].shape[1]
    slots = [[-1] * T for _ in rows]
    asked, taken, back = 0, 0, []
    for u, r in enumerate(rows):
        new = max(0, r + grow[u])
        if new > wide * page or grow[u] > T:
            continue
        held, want = _pages(r, page), _pages(new, page)
        if want > held:
            asked += want - held
            if asked > count:
                continue
            for j in range(held, want):
                table[u][j] = ring[(head + taken + j - held) % n]
            taken += want - held
        back += table[u][want:held]
        for t in range(grow[u]):
            slots[u][t] = table[u][(r + t) // page] * page + (r + t) % page
        rows[u] = new
    for i, x in enumerate(back):
        ring[(head + count + i) % n] = x
    return _ints(rows), _ints([(head + taken) % n, count - taken + len(back)]), _ints(table), _ints(ring), _ints(slots)


def _exact_store(s):
    out = []
    for name in "kv":
        x, pages, scale = s[name], s[name + "_pages"], s[name + "_scale"].double()
        page = pages.shape[2]
        value = _number(pages)
        slots = s["slots"].cpu()
        ids = slots // page
        for u in range(x.shape[0]):
            start = 0
            while start < x.shape[2]:                               # a run of rows that go into one page
                at, p = int(slots[u, start]) % page, int(ids[u, start])
                end = min(x.shape[2], start + page - at)
                rows = x[u, :, start:end].double()
                size = torch.where(torch.isfinite(rows), rows.abs(), torch.zeros_like(rows)).amax((1, 2))
                e = torch.ceil(torch.log2(size / TOP)).clamp(min=LOWEST)
                e = torch.where(TOP * _two(e - 1) >= size, e - 1, e).clamp(min=LOWEST)
                new = _two(torch.where(TOP * _two(e) < size, e + 1, e))
                if at:
                    new = torch.maximum(new, scale[p])
                    value[p, :, :at] = _nearest(value[p, :, :at] * (scale[p] / new)[:, None, None])
                value[p, :, at:at + end - start] = _nearest(rows / new[:, None, None])
                scale[p] = new
                start = end
        out.append((value, scale))
    return out[0][0], out[1][0], out[0][1], out[1][1]


def _unit(s, name, u, n):
    """[KV heads, n, head_dim] float64: the unit's first n rows."""
    page = s["case"]["page"]
    ids = s["table"][u, :_pages(n, page)].long()
    x = _number(s[name + "_pages"].view(torch.uint8)[ids]) * s[name + "_scale"][ids].double()[..., None, None]
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
