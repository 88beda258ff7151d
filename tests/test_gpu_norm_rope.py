"""hyq_norm_rope and hyq_paged_append on the GPU against the float64 oracle.

Tolerance: outputs are rounded to bf16 once (2^-8 of the value); the float32
work before that is within 2^-18 of the row's largest entry (a mean of 128
squares 2^-18 worst and 2^-22 typical halved by the root, weight, sine and
cosine products 2^-23 each; two products cancel in a rotated pair)."""
import numpy as np
import pytest

import paged_common as pc
import paper_2608_27875_amd as hyq
from oracle import paged_oracle as po

pytestmark = pytest.mark.gpu
D = 128


def close(got, want, what):
    tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -18 * np.abs(want).max(axis=-1, keepdims=True)
    bad = np.abs(got - want) > tol
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.abs(got - want)[bad].max()}"


def inv_freq(rot):
    return (1e4 ** -(np.arange(0, rot, 2) / max(rot, 1))).astype(np.float32)


def rope_of(rot, interleaved, qw, kw, eps=1e-6):
    f = inv_freq(rot)
    r = hyq.Rope(rot_dim=rot, interleaved=interleaved, eps=eps,
                 q_weight=None if qw is None else pc.dev(qw),
                 k_weight=None if kw is None else pc.dev(kw),
                 inv_freq=pc.dev(f) if rot else None)
    return r, f


def weights(rng, norm):
    w = [pc.bits(rng, D) if n else None for n in norm]
    return w, [None if x is None else po.bf16(x) for x in w]


CASES = [
    # B, Hq, Hkv, L, rot, interleaved, (q norm, k norm), packed
    (1, 1, 1, 1, 128, False, (True, True), True),
    (2, 8, 2, 3, 128, False, (True, True), True),
    (1, 5, 1, 7, 64, False, (True, False), False),
    (3, 4, 4, 1, 128, True, (False, True), True),
    (1, 40, 8, 5, 16, True, (True, True), True),
    (2, 6, 3, 11, 32, False, (False, False), True),
    (1, 8, 8, 2, 0, False, (True, True), False),
    (1, 32, 8, 130, 96, False, (True, True), True),
    (1, 3, 1, 4, 112, False, (True, True), True),
]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_dense(case):
    import torch
    B, Hq, Hkv, L, rot, inter, norm, packed = case
    rng = np.random.default_rng(hash(case[:5]) % 1000)
    T, H = B * L, Hq + 2 * Hkv
    raw = pc.bits(rng, T, H, D, scale=3.0)
    w, wv = weights(rng, norm)
    rope, f = rope_of(rot, inter, *w)
    pos = rng.integers(-5, 100000, size=T).astype(np.int32)
    x = pc.dev(raw)
    q, k, v = x.split([Hq, Hkv, Hkv], dim=1)
    if not packed:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    shape = hyq.Shape(B=B, Hq=Hq, Hkv=Hkv, L=L)
    Q, K, V = (torch.full((B, h, L, D), float("nan"), dtype=torch.bfloat16, device="cuda")
               for h in (Hq, Hkv, Hkv))
    hyq.hyq_norm_rope(shape, rope, q, k, v, pc.dev(pos), Q, K, V)
    torch.cuda.synchronize()
    xv = po.bf16(raw)

    def dense(r):
        return r.reshape(B, L, -1, D).transpose(0, 2, 1, 3)
    close(pc.host(Q), dense(po.norm_rope(xv[:, :Hq], wv[0], pos, f, rot, inter)), "Q")
    close(pc.host(K), dense(po.norm_rope(xv[:, Hq:Hq + Hkv], wv[1], pos, f, rot, inter)), "K")
    assert np.array_equal(pc.host(V), dense(xv[:, Hq + Hkv:])), "V is copied"


def test_without_keys_and_values():
    import torch
    rng = np.random.default_rng(3)
    raw = pc.bits(rng, 6, 4, D)
    (qw, kw), (qv, _) = weights(rng, (True, True))
    rope, f = rope_of(128, False, qw, kw)
    pos = np.arange(6, dtype=np.int32)
    Q = torch.empty((1, 4, 6, D), dtype=torch.bfloat16, device="cuda")
    hyq.hyq_norm_rope(hyq.Shape(B=1, Hq=4, Hkv=2, L=6), rope, pc.dev(raw), None, None, pc.dev(pos),
                      Q, None, None)
    close(pc.host(Q)[0].transpose(1, 0, 2), po.norm_rope(po.bf16(raw), qv, pos, f, 128), "Q")


def test_far_positions():
    """Angles of positions beyond 2^24, where a float32 product is off by radians."""
    import torch
    rng = np.random.default_rng(4)
    raw = pc.bits(rng, 4, 3, D)
    rope, f = rope_of(128, False, None, None)
    pos = np.array([2 ** 31 - 1, 16777217, 123456789, -2 ** 31], dtype=np.int32)
    Q, K, V = (torch.empty((4, 1, 1, D), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    x = pc.dev(raw)
    hyq.hyq_norm_rope(hyq.Shape(B=4, Hq=1, Hkv=1, L=1), rope, x[:, :1], x[:, 1:2], x[:, 2:],
                      pc.dev(pos), Q, K, V)
    want = po.norm_rope(po.bf16(raw)[:, :1], None, pos, f, 128)
    close(pc.host(Q)[:, :, 0], want, "Q")


def test_zero_rows_and_tiny_ones():
    """mean(x^2) = 0 with eps: zeros; eps = 0 on tiny rows: still unit rows."""
    import torch
    raw = np.zeros((2, 3, D), dtype=np.uint16)
    raw[1] = pc.bits(np.random.default_rng(5), 3, D, scale=1e-12)
    one = np.full(D, 0x3F80, dtype=np.uint16)
    for eps in (1e-6, 1e-30):
        rope, f = rope_of(128, False, one, one, eps)
        Q, K, V = (torch.empty((2, 1, 1, D), dtype=torch.bfloat16, device="cuda") for _ in range(3))
        x = pc.dev(raw)
        pos = np.array([3, 4], dtype=np.int32)
        hyq.hyq_norm_rope(hyq.Shape(B=2, Hq=1, Hkv=1, L=1), rope, x[:, :1], x[:, 1:2], x[:, 2:],
                          pc.dev(pos), Q, K, V)
        want = po.norm_rope(po.bf16(raw)[:, :1], np.ones(D), pos, f, 128, eps=eps)
        assert np.all(pc.host(Q)[0] == 0)
        close(pc.host(Q)[:, :, 0], want, "Q")


APPEND = [
    # lens, news, Hq, Hkv, page, fmt, rot, interleaved, tail rows nobody owns
    ([0], [1], 1, 1, 16, "bf16", 128, False, 0),
    ([5, 0, 40], [3, 17, 1], 8, 2, 16, "bf16", 128, False, 2),
    ([63, 64, 1], [2, 0, 70], 4, 4, 64, "int8", 64, True, 3),
    ([30, 200], [5, 31], 5, 1, 32, "fp8", 128, False, 0),
    ([255, 256], [2, 1], 16, 2, 256, "fp8", 128, True, 1),
    ([100], [129], 6, 3, 128, "int8", 0, False, 0),
]


@pytest.mark.parametrize("case", APPEND, ids=str)
def test_append(case):
    import torch
    lens, news, Hq, Hkv, page, fmt, rot, inter, tail = case
    rng = np.random.default_rng(sum(lens) + sum(news))
    cu = np.concatenate([[0], np.cumsum(news)])
    T = int(cu[-1]) + tail
    table, n_pages = pc.tables(rng, np.add(lens, news), page)
    bufs, vals = pc.pool(rng, fmt, n_pages, Hkv, page)
    mass = rng.random((n_pages, Hkv, page)).astype(np.float32)
    cache = pc.cache_of(bufs, fmt, Hq, mass)
    raw = pc.bits(rng, T, Hq + 2 * Hkv, D, scale=2.0)
    (qw, kw), (qv, kv) = weights(rng, (True, True))
    rope, f = rope_of(rot, inter, qw, kw)
    pos = rng.integers(0, 5000, size=T).astype(np.int32)
    x = pc.dev(raw)
    q, k, v = x.split([Hq, Hkv, Hkv], dim=1)
    q_out = torch.full((T, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    before = {n: t.clone() for n, t in cache.bufs.items() if t is not None}
    hyq.hyq_paged_append(cache, pc.batch_of(cu, lens, table), rope, q, k, v, pc.dev(pos), q_out)
    torch.cuda.synchronize()
    xv = po.bf16(raw)
    n = T - tail
    close(pc.host(q_out)[:n], po.norm_rope(xv[:n, :Hq], qv, pos, f, rot, inter), "q")
    assert np.all(pc.host(q_out)[n:] == 7.0), "rows of nobody are left"
    want_k = po.norm_rope(xv[:n, Hq:Hq + Hkv], kv, pos, f, rot, inter)
    want_v = xv[:n, Hq + Hkv:]
    untouched = np.ones((n_pages, page), dtype=bool)
    after = {m: t.cpu().numpy() if m != "k" and m != "v" or fmt != "bf16" else pc.host(t)
             for m, t in cache.bufs.items() if t is not None}
    for b in range(len(lens)):
        for i in range(news[b]):
            p, o = po.place(table, b, lens[b] + i, page, n_pages)
            untouched[p, o] = False
            t = int(cu[b]) + i
            assert np.all(after["mass"][p, :, o] == 0.0)
            for name, want in (("k", want_k[t]), ("v", want_v[t])):
                got = after[name][p, :, o]
                if fmt == "bf16":
                    (close if name == "k" else lambda a, c, w: np.testing.assert_array_equal(a, c))(got, want, name)
                    continue
                kind = "int" if fmt == "int8" else "fp8"
                code, s, val = po.quantize_row(want, kind)
                sc = after[name + "_scale"][p, :, o]
                if name == "v":   # exact inputs: the same codes and scales, bit for bit
                    np.testing.assert_array_equal(got, code.view(np.uint8))
                    np.testing.assert_array_equal(sc, s)
                else:   # within half a code step (of the value with E4M3), and of float32's work
                    np.testing.assert_allclose(sc, s, rtol=2.0 ** -18)
                    dec = got.view(np.int8).astype(np.float64) if kind == "int" else po.orc.e4m3_decode(got)
                    dec = dec * sc[:, None].astype(np.float64)
                    step = sc[:, None] * (0.5 if kind == "int" else 2.0 ** -10) + \
                        (0.0 if kind == "int" else 2.0 ** -4) * np.abs(want)
                    assert np.all(np.abs(dec - want) <= step * (1 + 2.0 ** -10) +
                                  2.0 ** -17 * np.abs(want).max(-1, keepdims=True))
    for name, t in before.items():   # every other slot keeps its bytes
        was = t.view(torch.int16 if t.dtype == torch.bfloat16 else t.dtype).cpu().numpy()
        now = cache.bufs[name].view(torch.int16 if t.dtype == torch.bfloat16 else t.dtype).cpu().numpy()
        mask = untouched[:, None, :].repeat(Hkv, 1)
        np.testing.assert_array_equal(now[mask], was[mask], err_msg=name)


def test_append_keys_only_and_holes():
    """q may be left out; rows of a missing page and beyond the table go nowhere."""
    import torch
    rng = np.random.default_rng(9)
    bufs, _ = pc.pool(rng, "bf16", 2, 2, 16)
    cache = pc.cache_of(bufs, "bf16", 4)
    table = np.array([[1, -1], [7, 0]], dtype=np.int32)   # 7 is no page
    raw = pc.bits(rng, 40, 4, D)
    x = pc.dev(raw)
    rope, _ = rope_of(0, False, None, None)
    batch = pc.batch_of([0, 20, 40], [10, 14], table)
    was = pc.host(cache.bufs["k"])
    hyq.hyq_paged_append(cache, batch, rope, None, x[:, :2], x[:, 2:], pc.dev(np.zeros(40, np.int32)), None)
    torch.cuda.synchronize()
    want = was.copy()
    v = po.bf16(raw)
    for i in range(6):           # slots 10..15 of sequence 0; 16.. are in the hole
        want[1, :, 10 + i] = v[i, :2]
    for i in range(2, 18):       # slots 16..31 of sequence 1; 14, 15 in a bad page, 32.. beyond
        want[0, :, i - 2] = v[20 + i, :2]
    np.testing.assert_array_equal(pc.host(cache.bufs["k"]), want)


def test_prefill_and_decode_on_its_output():
    """The dense outputs are the prefill's and the decode calls' inputs."""
    import torch
    rng = np.random.default_rng(11)
    B, Hq, Hkv, L = 1, 8, 2, 300
    (qw, kw), (qv, kv) = weights(rng, (True, True))
    rope, f = rope_of(128, False, qw, kw)
    raw = pc.bits(rng, B * L, Hq + 2 * Hkv, D)
    x = pc.dev(raw)
    shape = hyq.Shape(B=B, Hq=Hq, Hkv=Hkv, L=L, window=64, budget_ppm=20000, bits_kv=8)
    Q, K, V = (torch.empty((B, h, L, D), dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv))
    pos = torch.arange(L, dtype=torch.int32, device="cuda")
    hyq.hyq_norm_rope(shape, rope, *x.split([Hq, Hkv, Hkv], dim=1), pos, Q, K, V)
    bufs = hyq.alloc_buffers(shape, Q.device)
    out = hyq.prefill(shape, Q, K, V, bufs)
    cache = hyq.DecodeCache(shape, L + 64, Q.device)
    hyq.hyq_freeze(shape, Q, K, V, cache)
    new = pc.dev(pc.bits(rng, B, Hq + 2 * Hkv, D))
    q1, k1, v1 = (torch.empty((B, h, D), dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv))
    hyq.hyq_norm_rope(hyq.Shape(B=B, Hq=Hq, Hkv=Hkv, L=1), rope, *new.split([Hq, Hkv, Hkv], dim=1),
                      torch.full((B,), L, dtype=torch.int32, device="cuda"), q1, k1, v1)
    hyq.hyq_decode_append(cache, k1, v1)
    o1 = torch.empty((B, Hq, D), dtype=torch.float32, device="cuda")
    hyq.hyq_decode_attn(cache, q1, o1)
    torch.cuda.synchronize()
    from oracle import hyq_oracle as orc

    def raw_bits(t):
        return t.view(torch.int16).cpu().numpy().view(np.uint16)
    qb, kb, vb = raw_bits(Q), raw_bits(K), raw_bits(V)
    idx, _ = orc.select_vertical(qb, kb, Hkv, 64, 20000)
    O = orc.attention(qb, kb, vb, 64, 8, idx, orc.quantize(qb, kb, vb, idx, 64, 8))
    assert np.abs(pc.host(out) - O).max() <= 2e-3
    oc = orc.freeze(qb, kb, vb, Hkv, 64, 20000, 8)
    orc.decode_append(oc, raw_bits(k1), raw_bits(v1))
    assert np.abs(pc.host(o1) - orc.decode_attention(raw_bits(q1), oc)).max() <= 2e-3
