"""Plain CPU oracle of the paged serving calls, in float64: norms and rotation,
the paged cache, its causal attention with the weight each key received, and
eviction by that weight.  Written from the formulas, slot by slot, with no code
of the HIP path.

Pages are float64 arrays of the values they hold ([n_pages, Hkv, page, D]);
``quantize_row`` gives what an 8-bit page keeps of a row.
"""
from __future__ import annotations

import numpy as np

from oracle import hyq_oracle as orc

POS_PAD = 0x7FFFFFFF


def bf16(x):
    """Values of bf16 bit patterns (uint16) in float64."""
    u = np.asarray(x, dtype=np.uint16).astype(np.uint32) << 16
    return u.view(np.float32).astype(np.float64)


def norm_rope_row(x, weight, pos, inv_freq, rot, interleaved, eps):
    """One head row x [D]: RMS norm (weight None: none), then the rotation."""
    y = np.array(x, dtype=np.float64)
    if weight is not None:
        y = y * weight / np.sqrt(np.mean(y * y) + eps)
    out = y.copy()
    for f in range(rot // 2):
        ang = float(pos) * float(inv_freq[f])
        a, c = (2 * f, 2 * f + 1) if interleaved else (f, f + rot // 2)
        out[a] = y[a] * np.cos(ang) - y[c] * np.sin(ang)
        out[c] = y[c] * np.cos(ang) + y[a] * np.sin(ang)
    return out


def norm_rope(x, weight, pos, inv_freq, rot, interleaved=False, eps=1e-6):
    """Rows x [T, H, D] at positions pos [T]."""
    return np.stack([np.stack([norm_rope_row(r, weight, pos[t], inv_freq, rot, interleaved, eps)
                               for r in x[t]]) for t in range(x.shape[0])])


def quantize_row(x, fmt):
    """(codes, scale, values) of a row x [..., D] in an 8-bit page: float32 scale
    max|x| / c, code nearest to x / scale."""
    x = np.asarray(x, dtype=np.float32)
    c = np.float32(127 if fmt == "int" else 448)
    s = (np.abs(x).max(axis=-1) / c).astype(np.float32)
    safe = np.where(s > 0, s, np.float32(1))[..., None]
    y = (x / safe).astype(np.float32)
    if fmt == "int":
        code = np.clip(np.rint(y), -127, 127).astype(np.int8)
        val = code.astype(np.float64)
    else:
        code = orc.e4m3_encode(np.clip(y, np.float32(-448), np.float32(448)))
        val = orc.e4m3_decode(code).astype(np.float64)
    zero = (s == 0)[..., None]
    code, val = np.where(zero, 0, code).astype(code.dtype), np.where(zero, 0.0, val)
    return code, s, val * s.astype(np.float64)[..., None]


def place(table, b, n, page, n_pages):
    """(page, offset) of slot n of sequence b, or None where the table has none."""
    i = n // page
    if i >= table.shape[1]:
        return None
    p = int(table[b, i])
    return (p, n % page) if 0 <= p < n_pages else None


def attention(q, k, v, cu, lens, table, Hkv, scale, mass=None, mode="none"):
    """Causal attention of the new tokens' queries q [T, Hq, D] over pages k, v.
    Rows that are nobody's stay NaN.  ``mode`` "add" or "set" changes ``mass``."""
    T, Hq, D = q.shape
    n_pages, _, page, _ = k.shape
    g = Hq // Hkv
    out = np.full((T, Hq, D), np.nan)
    for b in range(len(lens)):
        t0, t1 = int(cu[b]), int(cu[b + 1])
        if t1 == t0:
            continue
        total = int(lens[b]) + t1 - t0
        at = [place(table, b, n, page, n_pages) for n in range(total)]
        here = [n for n in range(total) if at[n] is not None]
        for j in range(Hkv):
            K = np.stack([k[at[n][0], j, at[n][1]] for n in here]) if here else np.zeros((0, D))
            V = np.stack([v[at[n][0], j, at[n][1]] for n in here]) if here else np.zeros((0, D))
            got = np.zeros(len(here))
            for i in range(t1 - t0):
                seen = np.array([n <= int(lens[b]) + i for n in here], dtype=bool)
                for h in range(j * g, (j + 1) * g):
                    if not seen.any():
                        out[t0 + i, h] = 0.0
                        continue
                    z = scale * (K[seen] @ q[t0 + i, h])
                    w = np.exp(z - z.max())
                    w /= w.sum()
                    out[t0 + i, h] = w @ V[seen]
                    got[seen] += w
            if mode != "none":
                for x, n in zip(got, here):
                    p, o = at[n]
                    mass[p, j, o] = x + (mass[p, j, o] if mode == "add" else 0.0)
    return out


def evict_slots(m, n, budget, recent):
    """Kept slots, ascending, of n slots with masses m [n]."""
    if n <= budget:
        return list(range(n))
    # NaN (and a missing page) below every number, -inf among them
    order = sorted(range(n - recent), key=lambda s: (np.isnan(m[s]), -float(m[s]) if m[s] == m[s] else 0.0, s))
    return sorted(order[:budget - recent] + list(range(n - recent, n)))


def evict(mass, lens, table, budget, recent):
    """keep [B, Hkv, budget] and new_lens [B]."""
    n_pages, Hkv, page = mass.shape
    B = len(lens)
    keep = np.full((B, Hkv, budget), POS_PAD, dtype=np.int32)
    for b in range(B):
        n = int(lens[b])
        at = [place(table, b, s, page, n_pages) for s in range(n)]
        for j in range(Hkv):
            m = np.array([np.nan if a is None else mass[a[0], j, a[1]] for a in at], dtype=np.float64)
            kept = evict_slots(m, n, budget, recent)
            keep[b, j, :len(kept)] = kept
    return keep, np.minimum(np.asarray(lens), budget).astype(np.int32)
