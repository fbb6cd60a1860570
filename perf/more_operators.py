"""The paged cache held in 8 bits, as a serving program calls it, beside its plain forms.

Rows are quantised as they are written into pages (codes of e4m3 or int8, and one power of two for each block of rows and head),
read back, and attended to by new rows (with a sliding window and first tokens that stay visible, or without).
"""
import math
import random

import torch

own = False

DEV = "cuda"
WORKSPACE_BYTES = 96 << 20  # zero-filled once and kept, as a serving program keeps it
CODE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
MOST = {"e4m3": 448.0, "int8": 127.0}  # largest code
LEAST_EXP, MOST_EXP = -100, {"e4m3": 119, "int8": 121}  # exponents of a block


# ---------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one decode step of 32 requests, all 64 layers: every row joins a block that has rows already (some of them grow its exponent);
        # then the blocks are read back
        {"name": "store decode 32", "op": "store", "layers": 64, "heads": 8, "dim": 128, "requests": 32, "new": 1, "held": 4000, "page": 16,
         "block": 16, "format": "e4m3", "f32": False, "hnd": False, "pad": 0},
        # a mapped cache of a 4,099-row prompt in fp32 enters head-major pages of 64, and is read back as later rows will see it
        {"name": "store mapped f32", "op": "store", "layers": 64, "heads": 8, "dim": 128, "requests": 1, "new": 4099, "held": 0, "page": 64,
         "block": 64, "format": "int8", "f32": True, "hnd": True, "pad": 61},
        # a chunk of one layer's new rows of a ragged batch, in a model's step
        {"name": "store layer 8 x 500", "op": "store", "layers": 1, "heads": 8, "dim": 128, "requests": 8, "new": 500, "held": 1001, "page": 32,
         "block": 16, "format": "e4m3", "f32": False, "hnd": False, "pad": 0},
        # a cached prompt of 8,191 rows, 40 layers, read back to be mapped to another model
        {"name": "load prompt 8191", "op": "load", "layers": 40, "heads": 8, "dim": 128, "rows": 8191, "page": 16, "block": 16, "format": "e4m3",
         "f32": False, "hnd": False, "pad": 0},
        # one layer's rows of a short prompt in 32 bits: latency
        {"name": "load layer 300 f32", "op": "load", "layers": 1, "heads": 8, "dim": 128, "rows": 300, "page": 64, "block": 32, "format": "int8",
         "f32": True, "hnd": True, "pad": 7},
        # one new token of one request over a short mapped prompt: latency
        {"name": "decode 1 x 1024", "op": "attention", "requests": 1, "q_lo": 1, "q_hi": 1, "kv_lo": 1024, "kv_hi": 1024, "kv_heads": 8,
         "group": 5, "dim": 128, "page": 16, "block": 16, "format": "e4m3", "window": 0, "sinks": 0, "hnd": False},
        # a decode batch over ragged mapped contexts (lengths of the ragged build)
        {"name": "decode 64 ragged", "op": "attention", "requests": 64, "q_lo": 1, "q_hi": 1, "kv_lo": 512, "kv_hi": 8192, "kv_heads": 8,
         "group": 8, "dim": 128, "page": 16, "block": 16, "format": "e4m3", "window": 0, "sinks": 0, "hnd": False},
        # a few long contexts, two rows each (the last token and a guess)
        {"name": "decode 3 x 2 over 99999", "op": "attention", "requests": 3, "q_lo": 2, "q_hi": 2, "kv_lo": 60000, "kv_hi": 99999, "kv_heads": 8,
         "group": 8, "dim": 128, "page": 64, "block": 64, "format": "int8", "window": 0, "sinks": 0, "hnd": True},
        # a short question of each of four requests over its long transferred cache
        {"name": "chunk 4 x 200 over 8192", "op": "attention", "requests": 4, "q_lo": 77, "q_hi": 200, "kv_lo": 5000, "kv_hi": 8192,
         "kv_heads": 8, "group": 8, "dim": 128, "page": 32, "block": 32, "format": "e4m3", "window": 0, "sinks": 0, "hnd": True},
        # one long chunk of a prompt over everything before it
        {"name": "chunk 4096 over 16384", "op": "attention", "requests": 1, "q_lo": 4096, "q_hi": 4096, "kv_lo": 16384, "kv_hi": 16384,
         "kv_heads": 8, "group": 8, "dim": 128, "page": 64, "block": 64, "format": "e4m3", "window": 0, "sinks": 0, "hnd": False},
        # a layer with a window and four first tokens: long contexts, of which few rows are read
        {"name": "window decode 32", "op": "attention", "requests": 32, "q_lo": 1, "q_hi": 1, "kv_lo": 3000, "kv_hi": 16000, "kv_heads": 8,
         "group": 5, "dim": 128, "page": 16, "block": 8, "format": "int8", "window": 1024, "sinks": 4, "hnd": False},
        # the same layer over a prompt's chunks, narrow heads
        {"name": "window chunk 2 x 2047", "op": "attention", "requests": 2, "q_lo": 1500, "q_hi": 2047, "kv_lo": 6000, "kv_hi": 8192,
         "kv_heads": 8, "group": 4, "dim": 64, "page": 16, "block": 16, "format": "e4m3", "window": 1000, "sinks": 4, "hnd": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["store", "load", "attention", "attention", "attention"])
    page = rng.choice([8, 16, 32, 64, 128, 256])
    block = rng.choice([b for b in (8, 16, 32, 64, 128, 256) if b <= page])
    case = {"op": op, "dim": rng.choice([64, 128, 128]), "page": page, "block": block, "format": rng.choice(["e4m3", "int8"]), "hnd": rng.random() < 0.5}
    if op != "attention":
        layers, heads = rng.choice([1, 2, 36, 40, 64]), rng.choice([1, 2, 8])
        case |= {"layers": layers, "heads": heads, "f32": rng.random() < 0.5, "pad": rng.randrange(0, 70)}
        if op == "load":
            return case | {"rows": min(60000, _log(rng, 1, 64 * 8 * 4000 // (layers * heads)))}
        rows = _log(rng, 1, min(20000, 64 * 8 * 3000 // (layers * heads)))
        new = 1 if rng.random() < 0.4 else _log(rng, 1, rows)
        n = max(1, min(rows // new, 500, 64 * 8 * 3000 // (layers * heads * block)))
        return case | {"requests": n, "new": new, "held": rng.choice([0, _log(rng, 1, 5000)])}
    group = rng.choice([1, 2, 4, 5, 8, 16])
    kv_heads = rng.choice([1, 2, 4, 8]) if group < 16 else rng.choice([1, 2, 4])
    window, sinks = (0, 0) if rng.random() < 0.5 else (_log(rng, 1, 4096), rng.choice([0, 1, 4, 130]))
    case |= {"kv_heads": kv_heads, "group": group, "window": window, "sinks": sinks}
    if rng.random() < 0.5:  # decode, or a few rows a request
        kv = _log(rng, 16, 100000)
        n = _log(rng, 1, max(1, min(256, 300000 // kv)))
        q = rng.choice([1, 1, 1, 2, 4, 8])
    else:  # chunks
        q = _log(rng, 9, 4096)
        kv = max(q, _log(rng, 64, 16384))
        n = _log(rng, 1, max(1, min(16, (1 << 32) // (q * kv * kv_heads * group))))
    return case | {"requests": n, "q_lo": max(1, q - q // 2) if n > 1 else q, "q_hi": q, "kv_lo": max(q, kv // 4) if n > 1 else kv, "kv_hi": max(q, kv)}


# --------------------------------------------------------------------------------------------------------------- lengths
def _lengths(case):
    """(cached, new) per request: a property of the case, so that its work is."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    n = case["requests"]
    if case["op"] == "store":
        new = [rng.randint(max(1, case["new"] - case["new"] // 3), case["new"]) if n > 1 else case["new"] for _ in range(n)]
        return [rng.randint(case["held"] // 2, case["held"]) for _ in range(n)], new
    new = [rng.randint(case["q_lo"], case["q_hi"]) for _ in range(n)]
    total = [rng.randint(case["kv_lo"], case["kv_hi"]) for _ in range(n)]
    return [max(0, t - q) for t, q in zip(total, new)], new


def _up(n, unit):
    return -(-n // unit)


def _kept(case):
    """For each request of a store: (first row of the first block that is written to, rows behind the new ones' last)."""
    b = case["block"]
    return [(c // b * b, c + n) for c, n in zip(*_lengths(case))]


def _seen(p, window, sinks):
    """How many keys the row at position p sees."""
    return p + 1 if not window else min(window, p + 1) + min(sinks, max(0, p + 1 - window))


def _read(first, last, window, sinks):
    """How many keys the rows at positions first..last see together."""
    lo = max(0, first - window + 1) if window else 0
    return last + 1 - lo + (min(sinks, lo) if window else 0)


def work(case):
    op, block = case["op"], case["block"]
    if op == "attention":
        cached, new = _lengths(case)
        pairs = sum(_seen(c + i, case["window"], case["sinks"]) for c, n in zip(cached, new) for i in range(n))
        keys = sum(_read(c, c + n - 1, case["window"], case["sinks"]) for c, n in zip(cached, new))
        heads = case["kv_heads"] * case["group"]
        return {"bytes": 2 * keys * case["kv_heads"] * case["dim"] + 2 * (keys // block) * case["kv_heads"] + 4 * sum(new) * heads * case["dim"],
                "flops": 4 * pairs * heads * case["dim"]}
    size, lh = 4 if case["f32"] else 2, 2 * case["layers"] * case["heads"]
    if op == "load":
        return {"bytes": lh * (case["rows"] * case["dim"] * (1 + size) + _up(case["rows"], block)) + 8 * (case["rows"] + case["pad"]), "flops": 0}
    rows, back = sum(_lengths(case)[1]), sum(b - a for a, b in _kept(case))
    blocks = sum(_up(b - a, block) for a, b in _kept(case))
    return {"bytes": lh * (case["dim"] * (rows * (size + 1) + back * (1 + size)) + 3 * blocks) + 8 * (rows + case["pad"] + back), "flops": 0}


# ---------------------------------------------------------------------------------------------------------------- inputs
def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _two(e):
    """2^e in fp32, exactly (a power function is off by a step here and there), for whole e in -126 .. 127."""
    return ((e.clamp(-126, 127).int() + 127) << 23).view(torch.float32)


def _codes(x, e, form):
    """Codes of x (fp32) in blocks of exponent e, broadcast against it."""
    y = (x * _two(-e)).clamp_(-MOST[form], MOST[form])
    return y.round_().to(torch.int8) if form == "int8" else y.to(torch.float8_e4m3fn)


def _need(most, form):
    """The least exponent under which `most` fits the codes: most = m 2^x with m in [1/2, 1)."""
    m, x = torch.frexp(most)
    x = torch.where(m <= MOST[form] / 2.0 ** (9 if form == "e4m3" else 7), x, x + 1) - (9 if form == "e4m3" else 7)
    return torch.where(most > 0, x, LEAST_EXP).clamp_(LEAST_EXP, MOST_EXP[form])


def _pool(case, layers, pages, g, spread=None):
    """Codes [layer][page][slot][head][channel] (heads before slots in memory with "hnd") and exponents [layer][page][block][head]."""
    heads, dim, page, block, form = case["kv_heads" if "kv_heads" in case else "heads"], case["dim"], case["page"], case["block"], case["format"]
    out = []
    for comp in range(2):
        codes = torch.empty((layers, pages, heads, page, dim) if case["hnd"] else (layers, pages, page, heads, dim), dtype=CODE[form], device=DEV)
        codes = codes.transpose(2, 3) if case["hnd"] else codes
        exps = torch.empty((layers, pages, page // block, heads), dtype=torch.int8, device=DEV)
        for layer in range(layers):
            x = torch.randn((pages, page // block, block, heads, dim), generator=g, device=DEV, dtype=torch.float32)
            if spread is not None and comp == 0:
                x.mul_(spread)
            e = _need(x.abs().amax((2, 4)), form)
            exps[layer] = e.to(torch.int8)
            codes[layer].view(torch.int8).copy_(_codes(x, e[:, :, None, :, None], form).view(pages, page, heads, dim).view(torch.int8))
        out += [codes, exps]
    return {"k": out[0], "k_exp": out[1], "v": out[2], "v_exp": out[3]}


def _slots(cached, new, order, page):
    """Slots of rows cached .. cached + new - 1 of every request, whose pages stand in `order` one request after the other."""
    at, out = 0, []
    for c, n in zip(cached, new):
        p = torch.arange(c, c + n, device=DEV)
        out.append(order[at + p // page] * page + p % page)
        at += _up(c + n, page)
    return torch.cat(out)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    op, page, dim = case["op"], case["page"], case["dim"]
    s = {"case": case}
    if op == "attention":
        cached, new = _lengths(case)
        need = [_up(c + n, page) for c, n in zip(cached, new)]
        spread = torch.exp(0.5 * torch.randn(case["kv_heads"], dim, generator=g, device=DEV))  # channels of unlike scale
        s |= _pool(case, 2, sum(need) + 2, g, spread)
        order = torch.randperm(sum(need) + 2, generator=g, device=DEV).to(torch.int32)
        table = torch.full((len(new), max(need) + 1), -1, dtype=torch.int32, device=DEV)
        table[torch.arange(max(need) + 1, device=DEV)[None, :] < _ints(need)[:, None]] = order[:sum(need)]
        s |= {"table": table, "cu": torch.cat([_ints([0]), torch.cumsum(_ints(new), 0).to(torch.int32)]),
              "total": _ints([c + n for c, n in zip(cached, new)]), "most_new": max(new), "most_keys": max(c + n for c, n in zip(cached, new)),
              "q": torch.randn(sum(new), case["kv_heads"] * case["group"], dim, generator=g, device=DEV, dtype=torch.float32).bfloat16(),
              "scale": dim ** -0.5, "workspace": torch.zeros(WORKSPACE_BYTES, dtype=torch.uint8, device=DEV)}
        s["out"] = torch.empty_like(s["q"])
        return s
    layers, heads, kind = case["layers"], case["heads"], torch.float32 if case["f32"] else torch.bfloat16
    behind = torch.full((case["pad"],), -1, dtype=torch.int64, device=DEV)  # rows behind the last request's
    if op == "load":
        pages = _up(case["rows"], page) + 3
        s |= _pool(case, layers, pages, g)
        s["slot"] = torch.cat([_slots([0], [case["rows"]], torch.randperm(pages, generator=g, device=DEV), page), behind])
    else:
        cached, new = _lengths(case)
        cached = [c % page for c in cached]  # of a request's earlier pages only the last one matters here
        pages = sum(_up(c + n, page) for c, n in zip(cached, new)) + 3
        s |= _pool(case, layers, pages, g)
        order = torch.randperm(pages, generator=g, device=DEV)
        s["slot"] = torch.cat([_slots(cached, new, order, page), behind])
        begin = [c // case["block"] * case["block"] for c in cached]
        s["back"] = _slots(begin, [c + n - b for c, n, b in zip(cached, new, begin)], order, page)
        grow = torch.exp(0.25 * torch.randn(sum(new) + case["pad"], 1, 1, generator=g, device=DEV))  # rows of unlike scale
        s |= {n: (grow * torch.randn(layers, sum(new) + case["pad"], heads, dim, generator=g, device=DEV, dtype=torch.float32)).to(kind)
              for n in ("rows_k", "rows_v")}
    out_rows = s["back"].numel() if op == "store" else s["slot"].numel()
    s |= {n: torch.zeros(layers, out_rows, heads, dim, dtype=kind, device=DEV) for n in ("out_k", "out_v")}
    return s


# ----------------------------------------------------------------------------------------------------------- one pass each
def run(state):
    op = state["case"]["op"]
    if own:
        return {"store": _own_store, "load": _own_load, "attention": _own_attention}[op](state)
    return {"store": _plain_store, "load": _plain_load, "attention": _plain_attention}[op](state)


def _own_pool(s):
    from paper_2609_00891_b200 import binding as cb
    return cb.PagePool8(s["k"], s["v"], s["k_exp"], s["v_exp"])


def _own_store(s):
    from paper_2609_00891_b200 import binding as cb
    pool = _own_pool(s)
    cb.cb_paged_store8(pool, s["rows_k"], s["rows_v"], s["slot"])
    cb.cb_paged_load8(pool, s["out_k"], s["out_v"], s["back"])
    return {n: s[n] for n in ("out_k", "out_v", "k_exp", "v_exp")}


def _own_load(s):
    from paper_2609_00891_b200 import binding as cb
    cb.cb_paged_load8(_own_pool(s), s["out_k"], s["out_v"], s["slot"])
    return {"k": s["out_k"], "v": s["out_v"]}


def _own_attention(s):
    from paper_2609_00891_b200 import binding as cb
    cb.cb_paged_attention8(s["q"], s["out"], _own_pool(s), 1, s["table"], s["cu"], s["total"], s["scale"], s["workspace"],
                           max_new=s["most_new"], window=s["case"]["window"], n_sink=s["case"]["sinks"])
    return s["out"]


def _values(codes, exps, block, page, slot):
    """fp32 values of the rows at `page`, `slot` (any shape) of codes [page][slot][head][channel]; leading layers stay."""
    layered = codes.dim() == 5
    c = (codes.view(torch.int8)[:, page, slot] if layered else codes.view(torch.int8)[page, slot]).view(codes.dtype).float()
    e = exps[:, page, slot // block] if layered else exps[page, slot // block]
    return c * _two(e.int())[..., None]


def _plain_load(s):
    c = s["case"]
    row = torch.nonzero(s["slot"] >= 0)[:, 0]
    slot = s["slot"][row]
    for n, out in (("k", s["out_k"]), ("v", s["out_v"])):
        out[:, row] = _values(s[n], s[n + "_exp"], c["block"], slot // c["page"], slot % c["page"]).to(out.dtype)
    return {"k": s["out_k"], "v": s["out_v"]}


def _plain_store(s):
    c = s["case"]
    page, block, form = c["page"], c["block"], c["format"]
    row = torch.nonzero(s["slot"] >= 0)[:, 0]
    slot = s["slot"][row]
    at, mine = torch.unique(slot // block, return_inverse=True)  # blocks that are written to
    pg, bl = at // (page // block), at % (page // block)
    begun = torch.zeros(at.numel(), dtype=torch.bool, device=DEV)
    begun[mine[slot % block == 0]] = True  # its first slot is written: the block begins anew
    inside = bl[:, None] * block + torch.arange(block, device=DEV)[None, :]
    for n in ("k", "v"):
        x, codes, exps = s["rows_" + n][:, row].float(), s[n], s[n + "_exp"]
        most = torch.zeros((x.shape[0], at.numel(), x.shape[2]), device=DEV)
        most.scatter_reduce_(1, mine[None, :, None].expand(x.shape[0], -1, x.shape[2]), x.abs().amax(-1), "amax")
        old = exps[:, pg, bl].int()
        e = torch.where(begun[None, :, None], _need(most, form), torch.maximum(old, _need(most, form)))
        held = codes.view(torch.int8)[:, pg[:, None], inside].view(codes.dtype).float()
        held = _codes(held, (e - old)[:, :, None, :, None], form).view(torch.int8)
        codes.view(torch.int8)[:, pg[:, None], inside] = held
        codes.view(torch.int8)[:, slot // page, slot % page] = _codes(x, e[:, mine][..., None], form).view(torch.int8)
        exps[:, pg, bl] = e.to(torch.int8)
        s["out_" + n].copy_(_values(codes, exps, block, s["back"] // page, s["back"] % page))
    return {n: s[n] for n in ("out_k", "out_v", "k_exp", "v_exp")}


def _plain_attention(s):
    c = s["case"]
    page, heads, group, dim, window, sinks = c["page"], c["kv_heads"], c["group"], c["dim"], c["window"], c["sinks"]
    cu, total, q = s["cu"].long(), s["total"].long(), s["q"]
    n, rows, keys, dev = total.numel(), s["most_new"], s["most_keys"], q.device
    new = cu[1:] - cu[:-1]
    j = torch.arange(keys, device=dev)
    at = s["table"][:, j // page].long().clamp_(min=0)  # pages of every request, padded to the longest
    slot = (j % page)[None, :].expand(n, -1)
    live = j[None, :] < total[:, None]
    k = _values(s["k"][1], s["k_exp"][1], c["block"], at, slot).mul_(live[:, :, None, None])
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
    v = _values(s["v"][1], s["v_exp"][1], c["block"], at, slot).mul_(live[:, :, None, None])
    out = torch.matmul(score.view(n, heads, group * rows, keys), v.permute(0, 2, 1, 3)).view(n, heads, group, rows, dim)
    out = torch.where(weight > 0, out / weight, 0.0).permute(0, 3, 1, 2, 4).reshape(n, rows, heads * group, dim)
    s["out"].copy_(out[i[None, :] < new[:, None]])
    return s["out"]


# ------------------------------------------------------------------------------------------------- the definitions in 64 bits
def _power(e):
    """2^e in 64 bits, exactly, for whole e."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _grid(y, form):
    """y (64 bits, within the codes' range) to the nearest code, ties to even."""
    if form == "int8":
        return torch.round(y)
    step = _power(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)  # 8 steps from one power of two to the next
    return torch.round(y / step) * step


def _exact_store(s):
    c = s["case"]
    page, block, form = c["page"], c["block"], c["format"]
    groups = {}
    for t, x in enumerate(s["slot"].tolist()):
        if x >= 0:
            groups.setdefault(x // block, []).append((t, x % block))
    # every block that is written to, in 64-bit numbers: [layer][block][slot][head][channel]
    ids = sorted(groups)
    where = torch.tensor([[b // (page // block), b % (page // block)] for b in ids], device=DEV)
    place = {b: i for i, b in enumerate(ids)}
    t_of, b_of, s_of = (torch.tensor(v, device=DEV) for v in zip(*((t, place[b], o) for b in ids for t, o in groups[b])))
    begun = torch.tensor([any(o == 0 for _, o in groups[b]) for b in ids], device=DEV)
    back_b = torch.tensor([place[x // block] for x in s["back"].tolist()], device=DEV)
    res = {}
    for n in ("k", "v"):
        exps, out = s[n + "_exp"].clone(), torch.empty(s["out_" + n].shape, dtype=torch.float64, device=DEV)
        for layer in range(c["layers"]):
            codes = s[n][layer].view(torch.int8).reshape(-1, page // block, block, c["heads"], c["dim"])[where[:, 0], where[:, 1]].view(s[n].dtype).double()
            x = s["rows_" + n][layer].double()[t_of]
            top = torch.zeros(len(ids), c["heads"], dtype=torch.float64, device=DEV).index_reduce_(0, b_of, x.abs().amax(-1), "amax")
            e = torch.ceil(torch.log2(top.clamp(min=2.0 ** -140) / MOST[form])).clamp(LEAST_EXP, MOST_EXP[form])
            e = e + (top > MOST[form] * _power(e)).double() - (top <= MOST[form] * _power(e - 1)).double()  # the logarithm's last bit
            e = e.clamp(LEAST_EXP, MOST_EXP[form])
            old = exps[layer][where[:, 0], where[:, 1]].double()
            e = torch.where(begun[:, None], e, torch.maximum(e, old))
            value = _grid((codes * _power(old - e)[:, None, :, None]).clamp(-MOST[form], MOST[form]), form)
            value[b_of, s_of] = _grid(x * _power(-e[b_of])[:, :, None], form)
            out[layer] = value[back_b, s["back"] % block] * _power(e[back_b])[:, :, None]
            exps[layer][where[:, 0], where[:, 1]] = e.to(torch.int8)
        res["out_" + n], res[n + "_exp"] = out, exps
    return res


def exact(case, seed):
    s = prepare(case, seed)
    page, block = case["page"], case["block"]
    if case["op"] == "store":
        return _exact_store(s)
    if case["op"] == "load":
        at = [x for x in s["slot"].tolist() if x >= 0]
        pages, slots = torch.tensor(at, device=DEV) // page, torch.tensor(at, device=DEV) % page
        res = {}
        for n in ("k", "v"):
            res[n] = torch.zeros(s["out_" + n].shape, dtype=torch.float64, device=DEV)
            for layer in range(case["layers"]):
                scale = _power(s[n + "_exp"][layer][pages, slots // block])
                res[n][layer, :len(at)] = s[n][layer].view(torch.int8)[pages, slots].view(s[n].dtype).double() * scale[:, :, None]
        return res
    cached, new = _lengths(case)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    window, sinks, group, start = case["window"], case["sinks"], case["group"], 0
    for b, (c, n) in enumerate(zip(cached, new)):
        pages = s["table"][b, :_up(c + n, page)].long()
        kv = [s[x][1].view(torch.int8)[pages].view(s[x].dtype).double() * _power(s[x + "_exp"][1][pages]).repeat_interleave(block, 1)[..., None]
              for x in ("k", "v")]
        k, v = (x.flatten(0, 1)[:c + n] for x in kv)
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
