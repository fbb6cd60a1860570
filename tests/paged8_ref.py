"""Plain 64-bit forms of the operators of a paged cache held in 8 bits, written from their definitions, for the tests (CPU)."""
import numpy as np
import torch

LARGEST = {torch.float8_e4m3fn: 448.0, torch.int8: 127.0}
EXPS = {torch.float8_e4m3fn: (-100, 119), torch.int8: (-100, 121)}


def to_grid(y, kind):
    """64-bit numbers to the nearest code value (ties to even), the largest code at most; NaN: NaN, or 0 for int8."""
    y = np.clip(y, -LARGEST[kind], LARGEST[kind])
    if kind is torch.int8:
        return np.rint(np.nan_to_num(y, nan=0.0))
    _, x = np.frexp(np.maximum(np.abs(np.nan_to_num(y)), 2.0 ** -6))
    step = np.exp2(x - 4.0)                                # 8 steps from one power of two to the next, 2^-9 below 2^-6
    return np.rint(y / step) * step


def need(most, kind):
    """Least exponent e with most * 2^-e <= largest code, clamped."""
    lo, hi = EXPS[kind]
    e = np.full(most.shape, lo)
    for x in range(lo, hi):
        e = np.where(most > LARGEST[kind] * 2.0 ** x, x + 1, e)
    return e


def numbers(codes):
    """Codes (torch, any device) as float64 numpy."""
    return np.ascontiguousarray(codes.detach().cpu().double().numpy())


def store(codes, exps, x, slot, kind, page, block):
    """codes [L][pages][page][H][d] (float64 code values), exps [L][pages][page / block][H] (int), x [L][T][H][d], slot list:
    updated in place."""
    codes = codes.reshape(codes.shape[0], -1, block, *codes.shape[3:])          # [L][block id][row][H][d]
    flat = exps.reshape(exps.shape[0], -1, exps.shape[3])
    groups = {}
    for t, s in enumerate(slot):
        if 0 <= s < codes.shape[1] * block:
            groups.setdefault(s // block, []).append((t, s % block))
    for b, rows in groups.items():
        t = [r[0] for r in rows]
        most = np.nanmax(np.abs(np.nan_to_num(x[:, t], nan=0.0, posinf=np.inf, neginf=-np.inf)), axis=(1, 3))   # [L][H]
        e = need(most, kind)
        if not any(o == 0 for _, o in rows):
            old = np.clip(flat[:, b], *EXPS[kind])
            e = np.maximum(e, old)
            codes[:, b] = np.where((e > old)[:, None, :, None], to_grid(codes[:, b] * np.exp2((old - e).astype(float))[:, None, :, None], kind), codes[:, b])
        flat[:, b] = e
        for r, o in rows:
            codes[:, b, o] = to_grid(x[:, r] * np.exp2(-e.astype(float))[:, :, None], kind)


def values(codes, exps, block):
    """Code values and exponents as above -> float64 values [L][pages][page][H][d]."""
    return codes * np.exp2(np.repeat(exps, block, axis=2).astype(float))[..., None]


def attention(q, k, v, table, cu, total, scale, window=0, n_sink=0, weight=2.0 ** -11):
    """q [T][Hq][d], k and v [pages][slot][H][d] in float64, lists cu / total -> (out, tolerance) in float64; rows of no request are NaN.

    Tolerance, element by element: the output's rounding to bf16 (2^-8 of it); every weight's rounding (`weight`, of
    sum w |v| / sum w); the score's fp32 product over d channels, in the worst order, 2 d 2^-24 of scale sum |q||k| on the
    exponent, q held to 2^-20 of its row's largest magnitude (2^-20 of scale max|q| sum |k|), 2^-20 for the exponential, its argument
    (scores below 16 here) and the sums; and fp16's 2^-27 of the largest weight for every key (half a subnormal step, 2^-25, under
    2^6 for the largest weight and 2^-4 for a value's exponent)."""
    T, Hq, d = q.shape
    page, H = k.shape[1], k.shape[2]
    g = Hq // H
    out = torch.full((T, Hq, d), float("nan"), dtype=torch.float64, device=q.device)
    tol = torch.zeros_like(out)
    for b in range(len(total)):
        t0, t1 = cu[b], cu[b + 1]
        if t0 == t1:
            continue
        n = total[b]
        pages = table[b, : -(-n // page)].long()
        ok = (pages >= 0) & (pages < k.shape[0])           # a page id outside the pool reads as zeros
        at = torch.where(ok, pages, 0)
        kb, vb = (torch.where(ok[:, None, None, None], x[at], 0).flatten(0, 1)[:n] for x in (k, v))
        p = torch.arange(n - (t1 - t0), n, device=q.device)[:, None]
        j = torch.arange(n, device=q.device)[None, :]
        see = j <= p
        if window:
            see &= (p - j < window) | (j < n_sink)
        used = see.any(0)
        kb, vb = torch.where(used[:, None, None], kb, 0), torch.where(used[:, None, None], vb, 0)
        for h in range(Hq):
            qh, kh, vh = q[t0:t1, h].double(), kb[:, h // g], vb[:, h // g]
            s = torch.where(see, (qh @ kh.T) * scale, -torch.inf)
            m = s.amax(-1, keepdim=True) if n else torch.full((t1 - t0, 1), -torch.inf, dtype=torch.float64, device=q.device)
            w = torch.exp(s - torch.where(m == -torch.inf, 0, m))
            l = w.sum(-1, keepdim=True)
            safe = torch.where(l > 0, l, 1)
            out[t0:t1, h] = torch.where(l > 0, (w @ vh) / safe, 0)
            size = torch.where(l > 0, (w @ vh.abs()) / safe, 0)
            small = (see.double() @ vh.abs()) / safe * 2.0 ** -27
            worst = float((qh.abs() @ kh.abs().T).max()) * scale if n else 0.0
            parts = qh.abs().amax(-1, keepdim=True) * (float(kh.abs().sum(-1).max()) * scale * 2.0 ** -20) if n else 0.0
            tol[t0:t1, h] = out[t0:t1, h].abs() * 2.0 ** -8 + size * (weight + 2 * (2 * d * 2.0 ** -24 * worst + parts + 2.0 ** -20)) + small + 1e-30
    return out, tol
