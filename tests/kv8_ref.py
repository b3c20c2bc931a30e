"""64-bit restatement of the 8-bit cache's operators and of the page tables, one sequence, page and row at a time.

Test infrastructure only. Formulas as in include/cod.h: a page's scale is 2^e with the least e >= -100 for which the largest finite
magnitude appended to it is at most 448 * 2^e; held values are rounded again when it grows.
"""
from __future__ import annotations

import math

import numpy as np

PAGE = 16


def e4m3(x):
    """Nearest e4m3 value (ties to even) of float64 values, saturating at 448; NaN stays NaN."""
    x = np.asarray(x, dtype=np.float64)
    y = np.clip(x, -448.0, 448.0)
    _, k = np.frexp(np.where(np.isfinite(y), y, 0.0))
    step = np.ldexp(1.0, np.maximum(k - 1, -6) - 3)
    return np.where(np.isnan(x), np.nan, np.rint(y / step) * step)


def scale_for(amax: float) -> float:
    e = -100
    if amax > 0:
        e = max(-100, math.frexp(amax)[1] - 10)
        while amax > math.ldexp(448.0, e):
            e += 1
    return math.ldexp(1.0, e)


def append(pool, scale, rows, slot):
    """pool [Ld, n_pages, n_kv, 2, 16, hd] values of the bytes, scale [Ld, n_pages, n_kv, 2], rows [Ld, R, 2, n_kv, hd]; in place."""
    Ld, n_pages, n_kv = pool.shape[:3]
    r = 0
    while r < len(slot):
        if slot[r] < 0:
            r += 1
            continue
        pg, off = divmod(int(slot[r]), PAGE)
        n = 1
        while r + n < len(slot) and slot[r + n] == slot[r] + n and off + n < PAGE:
            n += 1
        follows_badly = r > 0 and slot[r - 1] >= 0 and slot[r - 1] // PAGE == pg
        if pg < n_pages and not follows_badly:
            for l in range(Ld):
                for h in range(n_kv):
                    for kv in range(2):
                        x = rows[l, r:r + n, kv, h]
                        fin = np.abs(x[np.isfinite(x)])
                        old = float(scale[l, pg, h, kv]) if off else 0.0
                        new = max(old, scale_for(float(fin.max()) if fin.size else 0.0))
                        if off and new != old:
                            pool[l, pg, h, kv, :off] = e4m3(pool[l, pg, h, kv, :off] * (old / new))
                        pool[l, pg, h, kv, off:off + n] = e4m3(x / new)
                        scale[l, pg, h, kv] = new
        r += n


def rope(x, pos, theta):
    """Rotate-half of x [..., hd] at positions pos (broadcast over the leading axes)."""
    hd = x.shape[-1]
    f = theta ** (-2.0 * np.arange(hd // 2) / hd)
    a = np.asarray(pos, dtype=np.float64)[..., None] * f
    lo, hi = x[..., :hd // 2], x[..., hd // 2:]
    return np.concatenate([lo * np.cos(a) - hi * np.sin(a), hi * np.cos(a) + lo * np.sin(a)], -1)


def attention(q, kb, vb, pool, scale, table, lens, carry, carry_len, theta):
    """q [S, W, n_q, hd], kb / vb [S, W, n_kv, hd], one layer's pool [n_pages, n_kv, 2, 16, hd]; all float64.
    Returns out, the largest score error that rounding the rotated q and k to `eps` relative would give per unit of eps,
    the largest |v| and the carried mass."""
    S, W, n_q, hd = q.shape
    n_kv = kb.shape[2]
    rep = n_q // n_kv
    out = np.zeros_like(q)
    mass = np.zeros((S, W, n_q))
    swing, vmax = 0.0, 0.0
    for s in range(S):
        L, c = int(lens[s]), int(carry_len[s])
        pos = (L + np.arange(W))[:, None]
        qs, ks = rope(q[s], pos, theta), rope(kb[s], pos, theta)
        pages = table[s, :(L + PAGE - 1) // PAGE]
        for h in range(n_kv):
            body = [(pool[pages, h, kv] * scale[pages, h, kv][:, None, None]).reshape(-1, hd)[:L] for kv in range(2)]
            k = np.concatenate([body[0], carry[s, h, 0, :c], ks[:, h]])
            v = np.concatenate([body[1], carry[s, h, 1, :c], vb[s, :, h]])
            for g in range(h * rep, (h + 1) * rep):
                sc = qs[:, g] @ k.T / math.sqrt(hd)
                p = np.exp(sc - sc.max(1, keepdims=True))
                p /= p.sum(1, keepdims=True)
                out[s, :, g] = p @ v
                mass[s, :, g] = p[:, L:L + c].sum(1)
                swing = max(swing, float((np.abs(qs[:, g]) @ np.abs(k).T).max() / math.sqrt(hd)))
            vmax = max(vmax, float(np.abs(v).max()))
    return out, swing, vmax, mass


class Tables:
    """Page tables kept by hand: what cod_pages_reserve and cod_pages_release are to do."""

    def __init__(self, n_pages, S, width, lens, page=PAGE):
        self.page, self.width, self.n_pages = page, width, n_pages
        self.free = list(range(n_pages - 1, -1, -1))
        self.table = [[-1] * width for _ in range(S)]
        self.held = [0] * S
        self.lens = [int(n) for n in lens]
        self.carry_len = [0] * S

    def reserve(self, n_new, max_rows=None, advance=False):
        total, slots, pos, seq, off, served = 0, [], [], [], [0], []
        n_free, lens = len(self.free), list(self.lens)
        for s, n in enumerate(n_new):
            n = int(n)
            ok, need = n >= 0 and 0 <= lens[s] + n <= self.width * self.page, 0
            if ok:
                need = max(0, -(-(lens[s] + n) // self.page) - self.held[s])
                total += need
                ok = need == 0 or total <= n_free
            if ok:
                for _ in range(need):
                    self.table[s][self.held[s]] = self.free.pop()
                    self.held[s] += 1
                if advance:
                    self.lens[s] += n
            served.append(ok)
            n = max(n, 0)
            for i in range(n):
                p = lens[s] + i
                slots.append(self.table[s][p // self.page] * self.page + p % self.page if ok else -1)
                pos.append(p)
                seq.append(s)
            off.append(off[-1] + n)
        if max_rows is not None:
            pad = [-1] * max(0, max_rows - len(slots))
            slots, pos, seq = (slots + pad)[:max_rows], (pos + pad)[:max_rows], (seq + pad)[:max_rows]
        return {"row_off": off, "slot": slots, "row_pos": pos, "row_seq": seq, "served": served}

    def release(self, keep=None):
        gone = []
        for s in range(len(self.held)):
            k = self.lens[s] if keep is None else max(0, int(keep[s]))
            first = min(self.held[s], -(-k // self.page))
            gone += self.table[s][first:self.held[s]]
            for j in range(first, self.held[s]):
                self.table[s][j] = -1
            self.held[s] = first
            if k < self.lens[s] or (keep is not None and k == 0):
                self.lens[s] = k
                self.carry_len[s] = 0
        self.free += gone[::-1]
