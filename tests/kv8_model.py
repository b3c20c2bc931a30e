"""Attention over the 8-bit cache in 64 bits, with the error that the kernels' roundings are to cause.

Test infrastructure only. With p the soft-max weights of a row, o = sum p_j v_j its output and d_j a small error of the j-th score,
the output moves by sum_j p_j d_j (v_j - o). Roundings are taken as independent and uniform within half a step of relative size u,
so with variance u^2 / 3 at most:
  q          one rounding per element (u = 2^-8: bf16, or two e4m3 terms: 2^-4 of a rest of 2^-4), the same for all keys of the row:
             d_j = sum_d e_d q_d k_jd / sqrt(hd), and the output moves by sum_d e_d q_d c_d with c_d = sum_j p_j k_jd (v_j - o) / sqrt(hd)
  block keys rounded to bf16 after the rotation, one rounding per element and key
  weights    f16 (u = 2^-11), one per key
  output     bf16, one per element
`noise` is the root of the expected square of the row's 2-norm, `mass_noise` the same for the carried share. Cached and carried
keys and all values are exact in what they are held in.
"""
from __future__ import annotations

import math

import numpy as np

from tests.kv8_ref import PAGE, rope

U_BF16, U_F16 = 2.0 ** -8, 2.0 ** -11


def attend(q, kb, vb, pool, scale, table, lens, carry, carry_len, theta, drop=None):
    """q [S, W, n_q, hd], kb / vb [S, W, n_kv, hd], one layer's pool [n_pages, n_kv, 2, 16, hd] and scale [n_pages, n_kv, 2]; float64.
    Table entries outside the pool: their keys do not count. drop: {(sequence, head): key} left out, too.
    Returns out, noise [S, W, n_q], mass, mass_noise."""
    S, W, n_q, hd = q.shape
    n_kv, n_pages = kb.shape[2], pool.shape[0]
    rep = n_q // n_kv
    out, noise, mass, mass_noise = np.zeros_like(q), *(np.zeros((S, W, n_q)) for _ in range(3))
    for s in range(S):
        L, c = int(lens[s]), int(carry_len[s])
        pos = (L + np.arange(W))[:, None]
        qs, ks = rope(q[s], pos, theta), rope(kb[s], pos, theta)
        pages = np.asarray(table[s, :(L + PAGE - 1) // PAGE])
        real = (pages >= 0) & (pages < n_pages)
        at = np.where(real, pages, 0)
        for h in range(n_kv):
            body = [(pool[at, h, kv] * scale[at, h, kv][:, None, None]).reshape(-1, hd)[:L] for kv in range(2)]
            k = np.concatenate([body[0], carry[s, h, 0, :c], ks[:, h]])
            v = np.concatenate([body[1], carry[s, h, 1, :c], vb[s, :, h]])
            keep = np.concatenate([np.repeat(real, PAGE)[:L], np.ones(c + W, bool)])
            kind = np.concatenate([np.zeros(L, int), np.ones(c, int), np.full(W, 2)])
            if drop is not None and (s, h) in drop:
                keep[drop[s, h]] = False
            k, v, kind = k[keep], v[keep], kind[keep]
            for g in range(h * rep, (h + 1) * rep):
                sc = qs[:, g] @ k.T / math.sqrt(hd)
                p = np.exp(sc - sc.max(1, keepdims=True))
                p /= p.sum(1, keepdims=True)
                o = p @ v
                out[s, :, g] = o
                mass[s, :, g] = p[:, kind == 1].sum(1)
                for i in range(W):
                    away, qi, blk = v - o[i], qs[i, g], kind == 2
                    pk = p[i][:, None] * k / math.sqrt(hd)
                    spread = ((pk.T @ away) ** 2).sum(1)                        # |c_d|^2
                    own = p[i, blk] ** 2 * ((qi * k[blk]) ** 2).sum(1) / hd      # p_j^2 var(d_j) / (u^2 / 3), block keys
                    far = (away ** 2).sum(1)
                    noise[s, i, g] = math.sqrt((U_BF16 ** 2 * ((qi ** 2 * spread).sum() + own @ far[blk] + (o[i] ** 2).sum())
                                                + U_F16 ** 2 * (p[i] ** 2 @ (v ** 2).sum(1))) / 3)
                    tilt = (kind == 1) - mass[s, i, g]
                    mass_noise[s, i, g] = math.sqrt((U_BF16 ** 2 * ((qi ** 2 * (pk.T @ tilt) ** 2).sum() + own @ tilt[blk] ** 2)) / 3)
    return out, noise, mass, mass_noise


def check(got, want, noise, mass=None, want_mass=None, mass_noise=None):
    """Every row within three times its expected error (a sum of bounded errors: even a row that one of them rules stays within 1.8),
    and 2^-18 of it for sums in float; the same for the carried share, four times (a single number). Raises AssertionError."""
    assert np.isfinite(got).all()
    off = np.linalg.norm(got - want, axis=-1)
    room = 3 * noise + 2.0 ** -18 * np.linalg.norm(want, axis=-1)
    assert (off <= room).all(), float((off / room).max())
    if mass is not None:
        assert np.isfinite(mass).all()
        off, room = np.abs(mass - want_mass), 4 * mass_noise + 2.0 ** -18
        assert (off <= room).all(), float((off / room).max())
