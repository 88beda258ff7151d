"""hyq_norm_rope and hyq_paged_append over the whole range of their values and
sizes: rows whose squares leave float32's range, rows of zeros without eps, more
rows than 2^24.

Tolerance as in test_gpu_norm_rope: one bf16 rounding, and float32's work
relative to the row's largest entry."""
import numpy as np
import pytest

import paged_common as pc
import paper_2608_27875_amd as hyq
from oracle import paged_oracle as po
from paper_2608_27875_amd import gen
from test_gpu_norm_rope import close, rope_of

pytestmark = pytest.mark.gpu
D = 128


def ranged(scales, heads=3, seed=5):
    """bf16 rows [len(scales), heads, D] of normal values times each scale."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((len(scales), heads, D)) * np.array(scales)[:, None, None]
    return gen.f32_to_bf16_bits(np.clip(x, -3e38, 3e38).astype(np.float32))


def want_rows(x, w, pos, f, inter, eps):
    """The oracle's rows; a row of zeros stays zero (with eps = 0 the formula is 0 / 0)."""
    dead = ~x.any(-1)
    y = po.norm_rope(np.where(dead[..., None], 1.0, x), w, pos, f, D, inter, eps)
    return np.where(dead[..., None], 0.0, y)


SCALES = [0.0, 1e-38, 1e-30, 1e-22, 1e-15, 1e-12, 1.0, 1e12, 1e20, 1e25, 1e37]


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("eps", [0.0, 1e-35, 1e-30, 1e-6])
def test_dense_rows_of_any_size(eps, inter):
    """RMS norms of rows from 1e-38 to 1e37 (their squares are zero or infinite
    in float32), and of zeros."""
    import torch
    raw = ranged(SCALES)
    T = len(SCALES)
    w = pc.bits(np.random.default_rng(6), D)
    rope, f = rope_of(D, inter, w, w, eps)
    pos = np.arange(T, dtype=np.int32) * 7
    Q, K, V = (torch.empty((T, 1, 1, D), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    x = pc.dev(raw)
    hyq.hyq_norm_rope(hyq.Shape(B=T, Hq=1, Hkv=1, L=1), rope, x[:, :1], x[:, 1:2], x[:, 2:], pc.dev(pos), Q, K, V)
    torch.cuda.synchronize()
    xv = po.bf16(raw)
    for got, h in ((Q, 0), (K, 1)):
        got = pc.host(got)[:, 0]
        want = want_rows(xv[:, h:h + 1], po.bf16(w), pos, f, inter, eps)
        assert np.isfinite(got).all()
        assert np.all(got[0] == 0)
        close(got, want, "QK"[h])
    assert np.array_equal(pc.host(V)[:, 0], xv[:, 2:])


@pytest.mark.parametrize("fmt", ["bf16", "int8", "fp8"])
def test_appended_rows_of_any_size(fmt):
    """The same into pages, without eps: keys stay finite, zero rows are zero
    rows in every format."""
    import torch
    scales = [s for s in SCALES if s < 1e30]   # values are kept as they are: their scales stay normal
    T = len(scales)
    raw = ranged(scales, heads=4, seed=8)
    w = pc.bits(np.random.default_rng(9), D)
    rope, f = rope_of(D, False, w, w, 0.0)
    bufs, _ = pc.pool(np.random.default_rng(10), fmt, 2, 1, 16)
    cache = pc.cache_of(bufs, fmt, 2, np.ones((2, 1, 16), np.float32))
    pos = np.arange(T, dtype=np.int32)
    x = pc.dev(raw)
    q_out = torch.empty((T, 2, D), dtype=torch.bfloat16, device="cuda")
    hyq.hyq_paged_append(cache, pc.batch_of([0, T], [0], [[1]]), rope, x[:, :2], x[:, 2:3], x[:, 3:],
                         pc.dev(pos), q_out)
    torch.cuda.synchronize()
    xv = po.bf16(raw)
    want = want_rows(xv[:, 2:3], po.bf16(w), pos, f, False, 0.0)[:, 0]
    close(pc.host(q_out), want_rows(xv[:, :2], po.bf16(w), pos, f, False, 0.0), "q")
    if fmt == "bf16":
        got = pc.host(cache.bufs["k"])[1, 0, :T]
        close(got, want, "k")
    else:
        kind = "int" if fmt == "int8" else "fp8"
        code = cache.bufs["k"].cpu().numpy()[1, 0, :T]
        s = cache.bufs["k_scale"].cpu().numpy()[1, 0, :T].astype(np.float64)
        got = (code.view(np.int8).astype(np.float64) if kind == "int" else po.orc.e4m3_decode(code)) * s[:, None]
        _, ws, _ = po.quantize_row(want, kind)
        np.testing.assert_allclose(s, ws, rtol=2.0 ** -18)
        # half a code step (of the value, with E4M3, and of its smallest step), and float32's work
        half = s[:, None] * (0.5 if kind == "int" else 2.0 ** -10) + (0.0 if kind == "int" else 2.0 ** -4) * np.abs(want)
        assert np.all(np.abs(got - want) <= half * (1 + 2.0 ** -10) + 2.0 ** -17 * np.abs(want).max(-1, keepdims=True))
    assert np.isfinite(got).all() and np.all(got[0] == 0)


def test_more_rows_than_24_bits_count():
    """17.5 million head rows, byte offsets beyond 2^32: values are copied, and
    queries and keys are right at tokens all over the call."""
    import torch
    B, Hq, Hkv, L = 2, 8, 1, 875011
    T, H = B * L, Hq + 2 * Hkv
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty((T, H, D), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    q, k, v = x.split([Hq, Hkv, Hkv], dim=1)
    w = pc.bits(np.random.default_rng(6), D)
    rope, f = rope_of(D, False, w, w)
    pos = torch.arange(T, device="cuda", dtype=torch.int32)
    Q, K, V = (torch.full((B, h, L, D), float("nan"), dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv))
    hyq.hyq_norm_rope(hyq.Shape(B=B, Hq=Hq, Hkv=Hkv, L=L), rope, q, k, v, pos, Q, K, V)
    torch.cuda.synchronize()
    assert torch.equal(V.view(torch.int16).view(T, D), v.contiguous().view(torch.int16).view(T, D))
    assert bool(torch.isfinite(Q).all()) and bool(torch.isfinite(K).all())
    at = np.unique(np.concatenate([[0, 1, L - 1, L, T - 1], np.random.default_rng(7).integers(0, T, 60)]))
    rows = pc.host(x[torch.from_numpy(at).cuda()])
    got_q = pc.host(Q.transpose(1, 2).reshape(T, Hq, D)[torch.from_numpy(at).cuda()])
    got_k = pc.host(K.transpose(1, 2).reshape(T, Hkv, D)[torch.from_numpy(at).cuda()])
    close(got_q, po.norm_rope(rows[:, :Hq], po.bf16(w), at, f, D), "Q")
    close(got_k, po.norm_rope(rows[:, Hq:Hq + Hkv], po.bf16(w), at, f, D), "K")
    del x, q, k, v, Q, K, V
    torch.cuda.empty_cache()
