"""The paged-cache operators as a serving program calls them, beside their plain forms.

Four calls of one chain: page tables from request lengths, rows stored into pages, rotary positions of several axes, and
attention of new rows over the paged cache (with a sliding window and first tokens that stay visible, or without).
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
WORKSPACE_BYTES = 96 << 20  # zero-filled once and kept, as a serving program keeps it


# ---------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one decode step of a small batch: every request adds one row to a cache in pages of 16
        {"name": "tables decode 32", "op": "tables", "requests": 32, "cached_lo": 100, "cached_hi": 4000, "new_lo": 1, "new_hi": 1,
         "page": 16, "pad": 0},
        # a whole ragged calibration-sized batch of mapped caches enters the pool at once (lengths of the ragged build)
        {"name": "tables ragged 500", "op": "tables", "requests": 500, "cached_lo": 0, "cached_hi": 0, "new_lo": 512, "new_hi": 8192,
         "page": 16, "pad": 1000},
        # the new rows of a decode step, all 64 layers, into pages of 16
        {"name": "store decode 32", "op": "store", "layers": 64, "heads": 8, "dim": 128, "rows": 32, "pad": 0, "page": 16,
         "f32": False, "hnd": False},
        # a mapped cache of a 4,099-row prompt in fp32, rounded to bf16 on its way into pages of 64, head-major pages
        {"name": "store mapped f32", "op": "store", "layers": 64, "heads": 8, "dim": 128, "rows": 4099, "pad": 61, "page": 64,
         "f32": True, "hnd": True},
        # the queries of one layer over a prompt with images: time, height and width positions in three sections
        {"name": "rope queries 3 axes", "op": "rope", "layers": 1, "heads": 64, "dim": 128, "rows": 8190, "sections": "24,20,20",
         "interleaved": False, "inverse": False, "far": 40000},
        # cached keys of all layers taken back to content coordinates before they are mapped, interleaved axes
        {"name": "rope keys inverse", "op": "rope", "layers": 40, "heads": 8, "dim": 128, "rows": 1024, "sections": "24,20,20",
         "interleaved": True, "inverse": True, "far": 1000000},
        # one new token of one request over a short mapped prompt: latency
        {"name": "decode 1 x 1024", "op": "attention", "requests": 1, "q_lo": 1, "q_hi": 1, "kv_lo": 1024, "kv_hi": 1024, "kv_heads": 8,
         "group": 5, "dim": 128, "page": 16, "window": 0, "sinks": 0, "hnd": False},
        # a decode batch over ragged mapped contexts (lengths of the ragged build)
        {"name": "decode 64 ragged", "op": "attention", "requests": 64, "q_lo": 1, "q_hi": 1, "kv_lo": 512, "kv_hi": 8192, "kv_heads": 8,
         "group": 8, "dim": 128, "page": 16, "window": 0, "sinks": 0, "hnd": False},
        # a short question of each of four requests over its long transferred cache
        {"name": "chunk 4 x 200 over 8192", "op": "attention", "requests": 4, "q_lo": 77, "q_hi": 200, "kv_lo": 5000, "kv_hi": 8192,
         "kv_heads": 8, "group": 8, "dim": 128, "page": 32, "window": 0, "sinks": 0, "hnd": True},
        # one long chunk of a prompt over everything before it
        {"name": "chunk 4096 over 16384", "op": "attention", "requests": 1, "q_lo": 4096, "q_hi": 4096, "kv_lo": 16384, "kv_hi": 16384,
         "kv_heads": 8, "group": 8, "dim": 128, "page": 64, "window": 0, "sinks": 0, "hnd": False},
        # a layer with a window and four first tokens: long contexts, of which few rows are read
        {"name": "window decode 32", "op": "attention", "requests": 32, "q_lo": 1, "q_hi": 1, "kv_lo": 3000, "kv_hi": 16000, "kv_heads": 8,
         "group": 5, "dim": 128, "page": 16, "window": 1024, "sinks": 4, "hnd": False},
        # the same layer over a prompt's chunks, narrow heads
        {"name": "window chunk 2 x 2047", "op": "attention", "requests": 2, "q_lo": 1500, "q_hi": 2047, "kv_lo": 6000, "kv_hi": 8192,
         "kv_heads": 8, "group": 4, "dim": 64, "page": 16, "window": 1000, "sinks": 4, "hnd": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tables", "store", "rope", "attention", "attention", "attention"])
    page = rng.choice([8, 16, 32, 64, 128, 256])
    if op == "tables":
        n = _log(rng, 1, 2000)
        if rng.random() < 0.5:
            hi = _log(rng, 8, 8192)
            return {"op": op, "requests": n, "cached_lo": 0, "cached_hi": hi, "new_lo": 0, "new_hi": _log(rng, 1, 8), "page": page,
                    "pad": rng.randrange(0, 40)}
        hi = _log(rng, 16, max(17, min(8192, 2000000 // n)))
        return {"op": op, "requests": n, "cached_lo": 0, "cached_hi": rng.choice([0, 1000]), "new_lo": hi // 16, "new_hi": hi, "page": page,
                "pad": rng.randrange(0, 2000)}
    if op == "store":
        layers = rng.choice([1, 2, 36, 40, 64])
        heads = rng.choice([1, 2, 8])
        rows = _log(rng, 1, max(2, 64 * 8 * 4000 // (layers * heads)))
        return {"op": op, "layers": layers, "heads": heads, "dim": rng.choice([64, 128]), "rows": min(rows, 60000), "pad": rng.randrange(0, 70),
                "page": page, "f32": rng.random() < 0.5, "hnd": rng.random() < 0.5}
    if op == "rope":
        dim = rng.choice([64, 128])
        axes = rng.choice([1, 2, 3, 4])
        least = 2
        cut = sorted(rng.sample(range(least, dim // 2 - least, least), axes - 1))
        parts = [b - a for a, b in zip([0] + cut, cut + [dim // 2])]
        layers = rng.choice([1, 1, 36, 40])
        heads = rng.choice([1, 5, 8, 40, 64])
        rows = _log(rng, 1, max(2, 64 * 8190 // (layers * heads)))
        return {"op": op, "layers": layers, "heads": heads, "dim": dim, "rows": rows, "sections": ",".join(str(x) for x in parts),
                "interleaved": rng.random() < 0.5, "inverse": rng.random() < 0.5, "far": _log(rng, 100, 1000000)}
    group = rng.choice([1, 2, 4, 5, 8, 16])
    kv_heads = rng.choice([1, 2, 4, 8]) if group < 16 else rng.choice([1, 2, 4])
    window, sinks = (0, 0) if rng.random() < 0.5 else (_log(rng, 1, 4096), rng.choice([0, 1, 4, 130]))
    case = {"op": op, "kv_heads": kv_heads, "group": group, "dim": rng.choice([64, 128, 128]), "page": page, "window": window, "sinks": sinks,
            "hnd": rng.random() < 0.5}
    if rng.random() < 0.5:  # decode, or a few rows a request
        kv = _log(rng, 16, 100000)
        n = _log(rng, 1, max(1, min(256, 500000 // kv)))
        q = rng.choice([1, 1, 1, 2, 4, 8])
    else:  # chunks
        q = _log(rng, 9, 4096)
        kv = max(q, _log(rng, 64, 16384))
        n = _log(rng, 1, max(1, min(16, (1 << 32) // (q * kv * kv_heads * group))))
    case |= {"requests": n, "q_lo": max(1, q - q // 2) if n > 1 else q, "q_hi": q, "kv_lo": max(q, kv // 4) if n > 1 else kv, "kv_hi": max(q, kv)}
    return case


# --------------------------------------------------------------------------------------------------------------- lengths
def _lengths(case):
    """(cached, new) per request: a property of the case, so that its work is."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    n = case["requests"]
    if case["op"] == "tables":
        return [rng.randint(case["cached_lo"], case["cached_hi"]) for _ in range(n)], [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(n)]
    new = [rng.randint(case["q_lo"], case["q_hi"]) for _ in range(n)]
    total = [rng.randint(case["kv_lo"], case["kv_hi"]) for _ in range(n)]
    return [max(0, t - q) for t, q in zip(total, new)], new


def _pages(length, page):
    return -(-length // page)


def _seen(p, window, sinks):
    """How many keys the row at position p sees."""
    return p + 1 if not window else min(window, p + 1) + min(sinks, max(0, p + 1 - window))


def _read(first, last, window, sinks):
    """How many keys the rows at positions first..last see together."""
    lo = max(0, first - window + 1) if window else 0
    return last + 1 - lo + (min(sinks, lo) if window else 0)


def work(case):
    op = case["op"]
    if op == "tables":
        cached, new = _lengths(case)
        fresh = sum(_pages(c + n, case["page"]) - _pages(c, case["page"]) for c, n in zip(cached, new))
        rows = sum(new) + case["pad"]
        return {"bytes": 8 * len(new) + 8 * fresh + 8 * len(new) + 12 * rows, "flops": 0}
    if op == "store":
        values = 2 * case["layers"] * case["rows"] * case["heads"] * case["dim"]
        return {"bytes": values * ((4 if case["f32"] else 2) + 2) + 8 * (case["rows"] + case["pad"]), "flops": 0}
    if op == "rope":
        values = case["layers"] * case["rows"] * case["heads"] * case["dim"]
        return {"bytes": 4 * values + 4 * case["rows"] * len(case["sections"].split(",")), "flops": 3 * values}
    cached, new = _lengths(case)
    pairs = sum(_seen(c + i, case["window"], case["sinks"]) for c, n in zip(cached, new) for i in range(n))
    keys = sum(_read(c, c + n - 1, case["window"], case["sinks"]) for c, n in zip(cached, new))
    heads = case["kv_heads"] * case["group"]
    return {"bytes": 4 * keys * case["kv_heads"] * case["dim"] + 4 * sum(new) * heads * case["dim"], "flops": 4 * pairs * heads * case["dim"]}


# ---------------------------------------------------------------------------------------------------------------- inputs
def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _pool(case, layers, pages, g):
    """K and V pages indexed [layer][page][slot][head][channel], slots or heads outermost in a page's memory."""
    heads, dim, page = case["kv_heads" if "kv_heads" in case else "heads"], case["dim"], case["page"]
    shape = (layers, pages, heads, page, dim) if case["hnd"] else (layers, pages, page, heads, dim)
    both = [torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16) for _ in range(2)]
    return [x.transpose(2, 3) if case["hnd"] else x for x in both]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    op = case["op"]
    s = {"case": case}
    if op == "tables":
        cached, new = _lengths(case)
        page, n = case["page"], len(new)
        held = [_pages(c, page) for c in cached]
        need = [_pages(c + x, page) for c, x in zip(cached, new)]
        width = max(1, max(need)) + 2
        order = torch.randperm(sum(need) + 16, generator=g, device=DEV).to(torch.int32)
        table = torch.full((n, width), -7, dtype=torch.int32, device=DEV)
        at = torch.arange(width, device=DEV)[None, :] < _ints(held)[:, None]
        table[at] = order[:sum(held)]
        rows = sum(new) + case["pad"]
        s |= {"cached": _ints(cached), "new": _ints(new), "free": order[sum(held):].contiguous(), "table": table, "page": page,
              "cu": torch.empty(n + 1, dtype=torch.int32, device=DEV), "total": torch.empty(n, dtype=torch.int32, device=DEV),
              "pos": torch.empty(rows, dtype=torch.int32, device=DEV), "slot": torch.empty(rows, dtype=torch.int64, device=DEV),
              "used": torch.empty(1, dtype=torch.int32, device=DEV)}
    elif op == "store":
        rows, page = case["rows"] + case["pad"], case["page"]
        pages = _pages(case["rows"], page) + 3
        s["k"], s["v"] = _pool(case, case["layers"], pages, g)
        shape = (case["layers"], rows, case["heads"], case["dim"])
        s["rows_k"], s["rows_v"] = (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(torch.float32 if case["f32"] else torch.bfloat16)
                                    for _ in range(2))
        t = torch.arange(case["rows"], device=DEV)
        slot = torch.randperm(pages, generator=g, device=DEV)[t // page] * page + t % page
        s["slot"] = torch.cat([slot, torch.full((case["pad"],), -1, dtype=torch.int64, device=DEV)])
    elif op == "rope":
        parts = [int(x) for x in case["sections"].split(",")]
        s |= {"x": torch.randn(case["layers"], case["rows"], case["heads"], case["dim"], generator=g, device=DEV, dtype=torch.float32).bfloat16(),
              "parts": parts, "base": 1e6,
              "pos": torch.randint(0, case["far"], (len(parts), case["rows"]), generator=g, device=DEV, dtype=torch.int32)}
        s["out"] = torch.empty_like(s["x"])
    else:
        cached, new = _lengths(case)
        page, dim = case["page"], case["dim"]
        need = [_pages(c + n, page) for c, n in zip(cached, new)]
        width = max(need) + 1
        s["k"], s["v"] = _pool(case, 2, sum(need) + 2, g)
        spread = torch.exp(0.5 * torch.randn(case["kv_heads"], dim, generator=g, device=DEV)).bfloat16()  # channels of unlike scale
        s["k"].mul_(spread)
        order = torch.randperm(sum(need) + 2, generator=g, device=DEV).to(torch.int32)
        table = torch.full((len(new), width), -1, dtype=torch.int32, device=DEV)
        table[torch.arange(width, device=DEV)[None, :] < _ints(need)[:, None]] = order[:sum(need)]
        s |= {"table": table, "cu": torch.cat([_ints([0]), torch.cumsum(_ints(new), 0).to(torch.int32)]),
              "total": _ints([c + n for c, n in zip(cached, new)]), "most_new": max(new), "most_keys": max(c + n for c, n in zip(cached, new)),
              "q": torch.randn(sum(new), case["kv_heads"] * case["group"], dim, generator=g, device=DEV, dtype=torch.float32).bfloat16(),
              "scale": dim ** -0.5, "workspace": torch.zeros(WORKSPACE_BYTES, dtype=torch.uint8, device=DEV)}
        s["out"] = torch.empty_like(s["q"])
    return s


# ----------------------------------------------------------------------------------------------------------- one pass each
def run(state):
    op = state["case"]["op"]
    if own:
        return {"tables": _own_tables, "store": _own_store, "rope": _own_rope, "attention": _own_attention}[op](state)
    return {"tables": _plain_tables, "store": _plain_store, "rope": _plain_rope, "attention": _plain_attention}[op](state)


def _own_tables(s):
    from paper_2609_00891_b200 import binding as cb
    cb.cb_page_tables(s["cached"], s["new"], s["page"], s["free"], s["table"], s["cu"], s["total"], s["pos"], s["slot"], s["used"])
    return {n: s[n] for n in ("table", "cu", "total", "pos", "slot", "used")}


def _own_store(s):
    from paper_2609_00891_b200 import binding as cb
    cb.cb_paged_store(cb.PagePool(s["k"], s["v"]), s["rows_k"], s["rows_v"], s["slot"])
    return {"k": s["k"], "v": s["v"]}


def _own_rope(s):
    from paper_2609_00891_b200 import binding as cb
    cb.cb_rope_axes(s["x"], s["out"], s["pos"], s["parts"], s["base"], interleaved=s["case"]["interleaved"], inverse=s["case"]["inverse"])
    return s["out"]


def _own_attention(s):
    from paper_2609_00891_b200 import binding as cb
    cb.cb_paged_attention(s["q"], s["out"], cb.PagePool(s["k"], s["v"]), 1, s["table"], s["cu"], s["total"], s["scale"], s["workspace"],
                          max_new=s["most_new"], window=s["case"]["window"], n_sink=s["case"]["sinks"])
    return s["out"]


def _plain_tables(s):
    page, table = s["page"], s["table"]
    cached, new = s["cached"].long(), s["new"].long()
    held, need = (cached + page - 1) // page, (cached + new + page - 1) // page
    before = torch.cumsum(need - held, 0) - (need - held)
    column = torch.arange(table.shape[1], device=table.device)[None, :]
    fresh = (column >= held[:, None]) & (column < need[:, None])
    index = (before[:, None] + column - held[:, None]).clamp_(0, s["free"].numel() - 1)
    table.copy_(torch.where(fresh, s["free"][index], table))
    cu = torch.cat([torch.zeros(1, dtype=torch.int64, device=table.device), torch.cumsum(new, 0)])
    row = torch.arange(s["pos"].numel(), device=table.device)
    inside = row < cu[-1]
    b = (torch.searchsorted(cu, row, right=True) - 1).clamp_(0, new.numel() - 1)
    pos = torch.where(inside, cached[b] + row - cu[b], 0)
    slot = torch.where(inside, table[b, pos // page].long() * page + pos % page, -1)
    return {"table": table, "cu": cu.int(), "total": (cached + new).int(), "pos": pos.int(), "slot": slot,
            "used": (need - held).sum().int().reshape(1)}


def _plain_store(s):
    page = s["case"]["page"]
    row = torch.nonzero(s["slot"] >= 0)[:, 0]
    slot = s["slot"][row]
    s["k"][:, slot // page, slot % page] = s["rows_k"][:, row].bfloat16()
    s["v"][:, slot // page, slot % page] = s["rows_v"][:, row].bfloat16()
    return {"k": s["k"], "v": s["v"]}


def _axis_of_pair(parts, interleaved, device):
    """Which axis turns pair i: sections one after the other, or axis i % n while that axis has pairs left and the first after that."""
    n = torch.tensor(parts, device=device)
    if not interleaved:
        return torch.repeat_interleave(torch.arange(len(parts), device=device), n)
    i = torch.arange(sum(parts), device=device)
    a = i % len(parts)
    return torch.where(i < len(parts) * n[a], a, 0)


def _plain_rope(s):
    x, dim = s["x"], s["case"]["dim"]
    axis = _axis_of_pair(s["parts"], s["case"]["interleaved"], x.device)
    turn = s["base"] ** (-2.0 * torch.arange(dim // 2, device=x.device, dtype=torch.float64) / dim)
    angle = s["pos"].double()[axis].T * turn[None, :]  # far positions: in 64 bits until the sine is taken
    cos, sin = torch.cos(angle).float()[None, :, None, :], torch.sin(angle).float()[None, :, None, :]
    sin = -sin if s["case"]["inverse"] else sin
    a, b = x[..., :dim // 2].float(), x[..., dim // 2:].float()
    s["out"].copy_(torch.cat([a * cos - b * sin, a * sin + b * cos], -1))
    return s["out"]


def _plain_attention(s):
    c = s["case"]
    page, heads, group, dim, window, sinks = c["page"], c["kv_heads"], c["group"], c["dim"], c["window"], c["sinks"]
    cu, total, q = s["cu"].long(), s["total"].long(), s["q"]
    n, rows, keys, dev = total.numel(), s["most_new"], s["most_keys"], q.device
    new = cu[1:] - cu[:-1]
    j = torch.arange(keys, device=dev)
    at = s["table"][:, j // page].long().clamp_(min=0)  # pages of every request, padded to the longest
    live = j[None, :] < total[:, None]
    k = s["k"][1][at, j % page].float().mul_(live[:, :, None, None])
    i = torch.arange(rows, device=dev)
    row = (cu[:-1, None] + i[None, :]).clamp_(max=q.shape[0] - 1)
    qs = q[row].float().view(n, rows, heads, group, dim).permute(0, 2, 3, 1, 4).reshape(n, heads, group * rows, dim)
    score = torch.matmul(qs, k.permute(0, 2, 3, 1)).mul_(s["scale"]).view(n, heads, group, rows, keys)
    del k
    p = (total - new)[:, None] + i[None, :]
    see = (j[None, None, :] <= p[:, :, None]) & live[:, None, :]
    if window:
        see &= (p[:, :, None] - j[None, None, :] < window) | (j < sinks)[None, None, :]
    score.masked_fill_(~see[:, None, None], -math.inf)
    score.sub_(score.amax(-1, keepdim=True).clamp_(min=-1e30)).exp_()
    weight = score.sum(-1, keepdim=True)
    v = s["v"][1][at, j % page].float().mul_(live[:, :, None, None])
    out = torch.matmul(score.view(n, heads, group * rows, keys), v.permute(0, 2, 1, 3)).view(n, heads, group, rows, dim)
    out = torch.where(weight > 0, out / weight, 0.0).permute(0, 3, 1, 2, 4).reshape(n, rows, heads * group, dim)
    s["out"].copy_(out[i[None, :] < new[:, None]])
    return s["out"]


# ------------------------------------------------------------------------------------------------- the definitions in 64 bits
def _exact_tables(s, cached, new):
    page, table, free = s["page"], s["table"].cpu().numpy().copy(), s["free"].cpu().numpy()
    pos, slot = np.zeros(s["pos"].numel(), np.int32), np.full(s["slot"].numel(), -1, np.int64)
    cu, taken = [0], 0
    for b, (c, n) in enumerate(zip(cached, new)):
        held, need = _pages(c, page), _pages(c + n, page)
        table[b, held:need] = free[taken:taken + need - held]
        taken += need - held
        at = np.arange(c, c + n)
        pos[cu[-1]:cu[-1] + n] = at
        slot[cu[-1]:cu[-1] + n] = table[b].astype(np.int64)[at // page] * page + at % page
        cu.append(cu[-1] + n)
    return {"table": table, "cu": np.array(cu, np.int32), "total": np.array(cached, np.int32) + np.array(new, np.int32), "pos": pos,
            "slot": slot, "used": np.array([taken], np.int32)}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "tables":
        return _exact_tables(s, *_lengths(case))
    if op == "store":
        k, v = s["k"].double(), s["v"].double()
        slots = s["slot"].tolist()
        live = [t for t, x in enumerate(slots) if x >= 0]
        pages = torch.tensor([slots[t] // case["page"] for t in live], device=DEV)
        offsets = torch.tensor([slots[t] % case["page"] for t in live], device=DEV)
        for layer in range(case["layers"]):
            k[layer, pages, offsets] = s["rows_k"][layer, live].bfloat16().double()
            v[layer, pages, offsets] = s["rows_v"][layer, live].bfloat16().double()
        return {"k": k, "v": v}
    if op == "rope":
        x, half, n = s["x"].double(), case["dim"] // 2, len(s["parts"])
        out = torch.empty_like(x)
        owner = [a for a, size in enumerate(s["parts"]) for _ in range(size)]
        for i in range(half):
            a = owner[i]
            if case["interleaved"]:
                a = i % n if i < n * s["parts"][i % n] else 0
            angle = s["pos"][a].double() * s["base"] ** (-i / half) * (-1 if case["inverse"] else 1)
            z = torch.complex(x[..., i], x[..., i + half]) * torch.polar(torch.ones_like(angle), angle)[None, :, None]
            out[..., i], out[..., i + half] = z.real, z.imag
        return out
    cached, new = _lengths(case)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    window, sinks, group, page, start = case["window"], case["sinks"], case["group"], case["page"], 0
    for b, (c, n) in enumerate(zip(cached, new)):
        pages = s["table"][b, :_pages(c + n, page)].long()
        k = s["k"][1][pages].flatten(0, 1)[:c + n].double()
        v = s["v"][1][pages].flatten(0, 1)[:c + n].double()
        behind = torch.arange(c, c + n, device=DEV)[:, None] - torch.arange(c + n, device=DEV)[None, :]
        hidden = behind < 0
        if window:
            hidden |= (behind >= window) & (torch.arange(c + n, device=DEV) >= sinks)[None, :]
        for h in range(case["kv_heads"]):
            q = s["q"][start:start + n, h * group:(h + 1) * group].double()
            score = torch.einsum("tgd,jd->gtj", q, k[:, h]) * s["scale"]
            out[start:start + n, h * group:(h + 1) * group] = torch.einsum("gtj,jd->tgd", torch.softmax(score.masked_fill(hidden, -math.inf), -1), v[:, h])
        start += n
    return out
