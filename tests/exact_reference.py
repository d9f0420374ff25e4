"""Exact attention and the 8-bit cache in 64 bits, one row and one block at a time (test infrastructure only)."""
import math

import numpy as np
import torch

E4M3_MAX, SCALE_MIN = 448.0, -118
TINY = 2.0 ** -126        # matrix instructions may take what is smaller as 0


def half_step(dtype):
    return torch.finfo({"f32": torch.float32, "bf16": torch.bfloat16}[dtype]).eps / 2


def attend(q, k, v, limit, scale, dtype):
    """q [n, d], k, v [keys, d] (64 bits), limit [n]: keys that a row sees.  O, lse, weights [n, keys], and how far the library
    may be off from each: the bounds of the roundings it makes, in the order it makes them.
      score: d products and sums in 32 bits, scaled, its reference taken off: |ds| <= eps (d + 8) scale sum |q k|
      weight: |dp| / p <= 2 |ds| (its own and the sum's) + eps (keys + 32); for the product with V in bf16 one rounding more
      output: sum |dp| |v|, one rounding to the tensor's type"""
    n, keys = q.shape[0], k.shape[0]
    eps = 2.0 ** -24
    O, lse, P = np.zeros((n, v.shape[1])), np.full(n, -np.inf), np.zeros((n, keys))
    dO, dlse, dP = np.zeros_like(O), np.zeros(n), np.zeros_like(P)
    for i in range(n):
        c = int(limit[i])
        if c <= 0:
            continue
        with np.errstate(invalid="ignore", over="ignore"):
            s = scale * (k[:c] @ q[i])
            m = s.max()
            if m == -np.inf:
                continue
            e = np.exp(s - m)
            p = e / e.sum()
            P[i, :c], lse[i] = p, m + math.log(e.sum()) if np.isfinite(m) else np.nan
            O[i] = (p[:, None] * v[:c]).sum(0)
            vis = p > 0                                     # (a key of weight 0 is none: its value has no bound)
            if not vis.any():                               # NaN throughout
                continue
            ds = eps * (q.shape[1] + 8) * scale * (np.abs(k[:c][vis]) @ np.abs(q[i])).max()
            w = 2 * ds + eps * (keys + 32)
            dP[i, :c] = w * p + TINY
            dlse[i] = ds + eps * (keys + 32) + 2 * eps * abs(lse[i])
            wv = w + (half_step(dtype) if dtype == "bf16" else 0.0)
            dO[i] = wv * (p[vis][:, None] * np.abs(v[:c][vis])).sum(0) + half_step(dtype) * np.abs(O[i]) * (1 + wv) + 2 * TINY
    return O, lse, P, dO, dlse, dP


def check(name, got, want, bound):
    got, want = np.asarray(got, dtype=np.float64), np.asarray(want, dtype=np.float64)
    assert got.shape == want.shape, (name, got.shape, want.shape)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        ok = same | (np.abs(got - want) <= bound)
    if not ok.all():
        at = tuple(int(x) for x in np.argwhere(~ok)[0])
        raise AssertionError(f"{name}: {(~ok).sum()} of {ok.size} off, first at {at}: {got[at]} for {want[at]}, bound {np.broadcast_to(bound, ok.shape)[at]}")


def limits(nq, nk, causal):
    return [max(0, min(nk, i + nk - nq + 1)) if causal else nk for i in range(nq)]


def packed(Q, K, V, q_off, k_off, scale, causal, dtype, O0, lse0):
    """Q [n_q, Hq, d] .. in 64 bits; O0, lse0: what rows of no sequence hold."""
    Hq, Hkv = Q.shape[1], K.shape[1]
    O, lse = O0.copy(), lse0.copy()
    dO, dlse = np.zeros_like(O), np.zeros_like(lse)
    for b in range(len(q_off) - 1):
        q0, q1, k0, k1 = q_off[b], q_off[b + 1], k_off[b], k_off[b + 1]
        for h in range(Hq):
            kv = h // (Hq // Hkv)
            o, l, _, do, dl, _ = attend(Q[q0:q1, h], K[k0:k1, kv], V[k0:k1, kv], limits(q1 - q0, k1 - k0, causal), scale, dtype)
            O[q0:q1, h], lse[h, q0:q1], dO[q0:q1, h], dlse[h, q0:q1] = o, l, do, dl
    return O, lse, dO, dlse


def e4m3(x):
    """Nearest e4m3 value, ties to even, of |x| <= 448; NaN for what is not finite."""
    x = np.asarray(x, dtype=np.float64)
    fine = np.isfinite(x)
    e = np.frexp(np.where(fine, x, 1.0))[1] - 1
    step = np.ldexp(1.0, np.maximum(e, -6) - 3)
    return np.where(fine, np.rint(np.where(fine, x, 0.0) / step) * step, np.nan)


def block_scale(x):
    """Smallest 2^e, e >= -118, with every finite |x| <= 448 2^e."""
    x = np.abs(x[np.isfinite(x)])
    most = float(x.max()) if x.size else 0.0
    e = SCALE_MIN
    while E4M3_MAX * 2.0 ** e < most:
        e += 1
    return 2.0 ** e


class Cache:
    """Codes as the values they are; K and V both [pages, Hkv, page, d] here."""

    def __init__(self, K, V, Ks, Vs):
        self.x = {"K": K.copy(), "V": V.copy()}
        self.s = {"K": Ks.astype(np.float64), "V": Vs.astype(np.float64)}
        self.page = K.shape[2]

    def store(self, name, pages, start, rows):
        """rows [n, Hkv, d] behind `start` tokens of the sequence with these pages."""
        n, P = rows.shape[0], self.page
        for j in range(start // P, -(-(start + n) // P)):
            lo, hi = max(start, j * P), min(start + n, (j + 1) * P)
            for h in range(rows.shape[1]):
                new = rows[lo - start:hi - start, h]
                s, old = block_scale(new), lo - j * P
                x, was = self.x[name][pages[j], h], self.s[name][pages[j], h]
                if old:
                    s = max(s, was)
                    x[:old] = e4m3(x[:old] * (was / s))
                x[old:old + hi - lo] = e4m3(new / s)
                self.s[name][pages[j], h] = s

    def tokens(self, name, pages, n, h):
        P = self.page
        return np.concatenate([self.x[name][pages[j], h] * self.s[name][pages[j], h] for j in range(-(-n // P))] or [np.zeros((0, self.x[name].shape[3]))])[:n]


def keep(w, budget, recent):
    """Slots that stay of a sequence with weights w: the last ones, and the heaviest others, lowest slot first among equals."""
    n = len(w)
    k = min(n, budget)
    r = min(recent, k)
    key = [math.inf if math.isnan(x) else x + 0.0 for x in w[:n - r]]
    nan = [0 if math.isnan(x) else 1 for x in w[:n - r]]
    best = sorted(range(n - r), key=lambda t: (nan[t], -key[t], t))[:k - r]
    return sorted(best) + list(range(n - r, n))
