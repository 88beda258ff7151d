"""Pins of the paged serving oracle: closed forms, torch's float64 softmax, and
brute force, all on the CPU."""
import itertools
import math

import numpy as np
import pytest

from oracle import paged_oracle as po

D = 128
INV = (1e4 ** -(np.arange(0, D, 2) / D)).astype(np.float32)


@pytest.mark.parametrize("inter", [False, True])
def test_rotation(inter):
    rng = np.random.default_rng(0)
    x, y = rng.standard_normal((2, D))
    assert np.array_equal(po.norm_rope_row(x, None, 0, INV, D, inter, 0.0), x)      # position 0
    r = po.norm_rope_row(x, None, 77, INV, 64, inter, 0.0)
    assert np.array_equal(r[64:], x[64:])                                           # partial
    a, c = (r[0:64:2], r[1:64:2]) if inter else (r[:32], r[32:64])
    u, v = (x[0:64:2], x[1:64:2]) if inter else (x[:32], x[32:64])
    np.testing.assert_allclose(a * a + c * c, u * u + v * v)                        # lengths of pairs
    z = (u + 1j * v) * np.exp(1j * 77 * INV[:32].astype(np.float64))
    np.testing.assert_allclose(a + 1j * c, z)
    # products depend on the distance alone
    d = [po.norm_rope_row(x, None, p, INV, D, inter, 0.0) @ po.norm_rope_row(y, None, p + 9, INV, D, inter, 0.0)
         for p in (0, 5, 100000)]
    np.testing.assert_allclose(d, d[0], rtol=1e-9)


def test_norm():
    rng = np.random.default_rng(1)
    x, w = rng.standard_normal(D) * 50, rng.standard_normal(D)
    y = po.norm_rope_row(x, w, 3, INV, 0, False, 0.0)
    np.testing.assert_allclose(np.sqrt(np.mean((y / w) ** 2)), 1.0)
    np.testing.assert_allclose(po.norm_rope_row(7 * x, w, 3, INV, 0, False, 0.0), y)
    np.testing.assert_allclose(po.norm_rope_row(np.zeros(D), w, 3, INV, D, False, 1e-6), 0.0)


@pytest.mark.parametrize("fmt", ["int", "fp8"])
def test_quantized_rows(fmt):
    rng = np.random.default_rng(2)
    x = rng.standard_normal((5, D)).astype(np.float32)
    x[3] = 0
    code, s, val = po.quantize_row(x, fmt)
    assert s[3] == 0 and np.all(val[3] == 0) and np.all(code[3] == 0)
    top = 127 if fmt == "int" else 448
    np.testing.assert_allclose(s, np.abs(x).max(-1) / top, rtol=1e-6)
    assert np.all(np.abs(val).max(-1) == top * s.astype(np.float64))
    step = 0.5 * s[:, None] if fmt == "int" else np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * s[:, None])
    assert np.all(np.abs(val - x) <= step * (1 + 1e-6))


def random_cache(rng, lens, news, Hkv, page):
    total = np.add(lens, news)
    used = [-(-int(n) // page) for n in total]
    n_pages = sum(used) + 2
    perm = rng.permutation(n_pages)
    table = np.full((len(lens), max(used) + 1), -1)
    at = 0
    for b, u in enumerate(used):
        table[b, :u] = perm[at:at + u]
        at += u
    k, v = rng.standard_normal((2, n_pages, Hkv, page, D))
    return table, k, v


def test_attention_against_torch():
    import torch
    rng = np.random.default_rng(3)
    lens, news, Hq, Hkv, page = [5, 0, 33], [3, 4, 1], 4, 2, 4
    table, k, v = random_cache(rng, lens, news, Hkv, page)
    cu = np.concatenate([[0], np.cumsum(news)])
    q = rng.standard_normal((cu[-1] + 2, Hq, D))
    mass = np.zeros(k.shape[:3])
    out = po.attention(q, k, v, cu, lens, table, Hkv, 0.1, mass, "add")
    assert np.isnan(out[cu[-1]:]).all()                     # rows of nobody
    for b in range(3):
        n = lens[b] + news[b]
        K = np.stack([k[table[b, s // page], :, s % page] for s in range(n)], 1)   # [Hkv, n, D]
        V = np.stack([v[table[b, s // page], :, s % page] for s in range(n)], 1)
        Q = q[cu[b]:cu[b + 1]].transpose(1, 0, 2)
        z = torch.tensor(Q) @ torch.tensor(K).repeat_interleave(2, 0).transpose(1, 2) * 0.1
        hid = torch.arange(n)[None] > lens[b] + torch.arange(news[b])[:, None]
        w = torch.softmax(z.masked_fill(hid, -math.inf), -1)
        np.testing.assert_allclose(out[cu[b]:cu[b + 1]], (w @ torch.tensor(V).repeat_interleave(2, 0))
                                   .transpose(0, 1).numpy(), rtol=1e-12, atol=1e-12)
        got = np.stack([mass[table[b, s // page], :, s % page] for s in range(n)], 1)
        np.testing.assert_allclose(got, w.sum(1).view(2, 2, n).sum(1).numpy(), rtol=1e-12, atol=1e-14)
        np.testing.assert_allclose(got.sum(), news[b] * Hq)  # every row's weights sum to 1
    again = po.attention(q, k, v, cu, lens, table, Hkv, 0.1, mass.copy(), "set")
    np.testing.assert_array_equal(again[:cu[-1]], out[:cu[-1]])


def test_attention_ignores_where_pages_lie():
    rng = np.random.default_rng(4)
    table, k, v = random_cache(rng, [21], [2], 1, 8)
    q = rng.standard_normal((2, 2, D))
    a = po.attention(q, k, v, [0, 2], [21], table, 1, 0.2)
    order = rng.permutation(len(k))
    inv = np.argsort(order)
    b = po.attention(q, k[order], v[order], [0, 2], [21], np.where(table >= 0, inv[table], -1), 1, 0.2)
    np.testing.assert_array_equal(a, b)


def test_holes():
    rng = np.random.default_rng(5)
    table, k, v = random_cache(rng, [20], [2], 1, 8)
    q = rng.standard_normal((2, 1, D))
    cut = table.copy()
    cut[0, 1] = 9999                                         # slots 8..15 are gone
    a = po.attention(q, k, v, [0, 2], [20], cut, 1, 0.2)
    z = np.array([q[0, 0] @ k[table[0, s // 8], 0, s % 8] * 0.2 for s in range(21) if not 8 <= s < 16])
    w = np.exp(z) / np.exp(z).sum()
    V = np.stack([v[table[0, s // 8], 0, s % 8] for s in range(21) if not 8 <= s < 16])
    np.testing.assert_allclose(a[0, 0], w @ V)
    none = po.attention(q, k, v, [0, 2], [20], np.full_like(table, -1), 1, 0.2)
    assert np.all(none == 0)


def test_eviction_brute_force():
    """The kept set is the recent slots and the best choice of the others: no
    slot outside has a larger mass than one inside, equal ones by slot."""
    rng = np.random.default_rng(6)
    for n, budget, recent in itertools.product((1, 5, 9, 12), (1, 4, 9), (0, 1, 4)):
        if recent > budget:
            continue
        m = rng.integers(0, 4, n).astype(np.float64)
        m[rng.random(n) < 0.2] = np.nan
        kept = po.evict_slots(m, n, budget, recent)
        assert kept == sorted(set(kept)) and len(kept) == min(n, budget)
        if n <= budget:
            continue
        assert set(range(n - recent, n)) <= set(kept)
        rank = [(-np.inf if np.isnan(m[s]) else m[s], -s) for s in range(n)]
        inside = [rank[s] for s in kept if s < n - recent]
        outside = [rank[s] for s in range(n - recent) if s not in kept]
        assert not inside or not outside or min(inside) > max(outside)
    keep, lens = po.evict(np.ones((3, 1, 4)), [0, 6], np.array([[0, 1], [2, 0]]), 4, 1)
    assert lens.tolist() == [0, 4] and keep[1, 0].tolist() == [0, 1, 2, 5]
    assert np.all(keep[0] == po.POS_PAD)
