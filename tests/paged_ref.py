"""Plain 64-bit forms of the paged-cache operators, written from their definitions, for the tests."""
import numpy as np
import torch


def tables(cached, new, page, free, table, n_rows):
    """Lists of lengths, the free list, the incoming table (numpy [B][cols]) -> dict of expected outputs (numpy)."""
    table = table.copy()
    pos, slot = np.zeros(n_rows, np.int32), np.full(n_rows, -1, np.int64)
    cu, total, taken, t = [0], [], 0, 0
    for b, (c, n) in enumerate(zip(cached, new)):
        c, n = max(c, 0), max(n, 0)
        held, need = -(-c // page), -(-(c + n) // page)
        fresh = {}
        for col in range(held, need):
            fresh[col] = free[taken] if taken < len(free) else -1
            if col < table.shape[1]:
                table[b, col] = fresh[col]
            taken += 1
        for i in range(n):
            p = c + i
            col = p // page
            if t < n_rows:
                pos[t] = p
                if col < table.shape[1]:
                    pg = fresh[col] if col in fresh else table[b, col]
                    slot[t] = int(pg) * page + p % page if pg >= 0 else -1
            t += 1
        cu.append(t)
        total.append(c + n)
    return {"table": table, "cu": np.array(cu, np.int32), "total": np.array(total, np.int32), "pos": pos, "slot": slot, "used": taken}


def rope(x, positions, sections, base, interleaved, inverse):
    """x [L][T][H][d] (any float), positions [A][T] int -> float64."""
    d, n = x.shape[-1], len(sections)
    x = x.double()
    out = torch.empty_like(x)
    owner = [a for a, s in enumerate(sections) for _ in range(s)]
    for i in range(d // 2):
        a = owner[i]
        if interleaved:
            a = i % n if i < n * sections[i % n] else 0
        ang = positions[a].double() * float(base) ** (-2.0 * i / d)
        c, s = torch.cos(ang)[None, :, None], torch.sin(ang)[None, :, None]
        s = -s if inverse else s
        lo, hi = x[..., i], x[..., i + d // 2]
        out[..., i], out[..., i + d // 2] = lo * c - hi * s, lo * s + hi * c
    return out


def attention(q, k_pool, v_pool, table, cu, total, scale, window=0, n_sink=0):
    """q [T][Hq][d], pools [pages][slot][H][d], lists cu / total -> (out float64, tolerance float64): rows of no request are NaN.

    Tolerance, element by element: the output's rounding to bf16 (2^-8 of it); every weight's rounding to bf16 (2^-8 of
    sum w |v| / sum w); the score's fp32 product over d channels, in the worst order, 2 d 2^-24 of scale sum |q||k| on the
    exponent, and 2^-20 for the exponential, its argument (scores below 16 here) and the sums."""
    T, Hq, d = q.shape
    page, H = k_pool.shape[1], k_pool.shape[2]
    g = Hq // H
    out = torch.full((T, Hq, d), float("nan"), dtype=torch.float64, device=q.device)
    tol = torch.zeros_like(out)
    for b in range(len(total)):
        t0, t1 = cu[b], cu[b + 1]
        if t0 == t1:
            continue
        n = total[b]
        pages = table[b, : -(-n // page)].long()
        # a page id outside the pool reads as zeros
        ok = (pages >= 0) & (pages < k_pool.shape[0])
        at = torch.where(ok, pages, 0)
        k = torch.where(ok[:, None, None, None], k_pool[at], 0).flatten(0, 1)[:n].double()
        v = torch.where(ok[:, None, None, None], v_pool[at], 0).flatten(0, 1)[:n].double()
        p = torch.arange(n - (t1 - t0), n, device=q.device)[:, None]
        j = torch.arange(n, device=q.device)[None, :]
        see = j <= p
        if window:
            see &= (p - j < window) | (j < n_sink)
        used = see.any(0)
        k = torch.where(used[:, None, None], k, 0)
        v = torch.where(used[:, None, None], v, 0)
        for h in range(Hq):
            qh, kh, vh = q[t0:t1, h].double(), k[:, h // g], v[:, h // g]
            s = (qh @ kh.T) * scale
            s = torch.where(see, s, -torch.inf)
            m = s.amax(-1, keepdim=True) if n else torch.full((t1 - t0, 1), -torch.inf, dtype=torch.float64, device=q.device)
            w = torch.exp(s - torch.where(m == -torch.inf, 0, m))
            l = w.sum(-1, keepdim=True)
            safe = torch.where(l > 0, l, 1)
            out[t0:t1, h] = torch.where(l > 0, (w @ vh) / safe, 0)
            size = torch.where(l > 0, (w @ vh.abs()) / safe, 0)
            worst = float((qh.abs() @ kh.abs().T).max()) * scale if n else 0.0
            tol[t0:t1, h] = out[t0:t1, h].abs() * 2.0 ** -8 + size * (2.0 ** -8 + 2 * (2 * d * 2.0 ** -24 * worst + 2.0 ** -20)) + 1e-30
    return out, tol
