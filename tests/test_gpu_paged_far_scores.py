"""hyq_paged_attn where scores are so large that float32 holds no fraction of
them: the largest ones still share all the weight.

Scores come from one channel, in powers of two, so equal keys have equal scores
and any two others are at least 2^-7 of the score apart: from 2^20 on the weights
are 0 and 1 / count, whatever the rounding.  At 2^12 that is 32, and the lesser
weights (e^-32) carry the error of their distance in log2 units, up to 2^12 1.46:
the factor log2 e, a row scale, and the product are rounded, 2^-24 of it each, and
a distance has two of them."""
import numpy as np
import pytest

import paged_common as pc
import paper_2608_27875_amd as hyq
from oracle import paged_oracle as po
from paper_2608_27875_amd import gen

pytestmark = pytest.mark.gpu
D = 128

PATTERNS = {
    # channel 0 of key s, times 2^a; all keys, or from the least to the largest and back
    "below": lambda s: np.where(s % 5 == 2, -1.0, -1.0078125),
    "above": lambda s: np.where(s % 5 == 2, 1.0, 1.0078125),
    "rising": lambda s: np.select([s < 70, s < 140, s < 210], [-1.0, 0.0, 2.0 ** -40], 1.0),
    "falling": lambda s: np.select([s < 70, s < 140, s < 210], [1.0, 2.0 ** -40, 0.0], -1.0),
    "late": lambda s: np.where(s == 295, -0.5, -1.0),
}


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "int8"])
@pytest.mark.parametrize("new,g,max_len", [(1, 2, 300), (4, 4, 9000), (40, 2, 300), (80, 2, 9000)])
@pytest.mark.parametrize("power", [12, 20, 33, 64, 120, 126])
def test_scores_of_any_size(power, new, g, max_len, fmt):
    import torch
    rng = np.random.default_rng(power + new)
    page, len0 = 32, 300
    n = len0 + new
    table, n_pages = pc.tables(rng, [n], page)
    a = power // 2
    cu = np.array([0, new])
    q = np.zeros((new, g, D), np.float32)
    q[..., 0] = 2.0 ** (power - a)
    qb = gen.f32_to_bf16_bits(q)
    for name, pattern in PATTERNS.items():
        bufs, vals = pc.pool(rng, fmt, n_pages, 1, page)
        k = np.zeros((n_pages, 1, page, D))
        for s in range(n):
            p, o = po.place(table, 0, s, page, n_pages)
            k[p, 0, o, 0] = float(pattern(np.array(s))) * 2.0 ** a
        if fmt == "bf16":
            bufs["k"] = gen.f32_to_bf16_bits(k.astype(np.float32))
            vals["k"] = po.bf16(bufs["k"])
        else:
            code, bufs["k_scale"], vals["k"] = po.quantize_row(k, "int" if fmt == "int8" else "fp8")
            bufs["k"] = code.view(np.uint8)
        mass = rng.random((n_pages, 1, page)).astype(np.float32)
        wm = mass.astype(np.float64)
        want = po.attention(po.bf16(qb), vals["k"], vals["v"], cu, [len0], table, 1, 1.0, wm, "set")
        cache = pc.cache_of(bufs, fmt, g, mass)
        batch = pc.batch_of(cu, [len0], table, max_len=max_len)
        out = torch.empty((new, g, D), device="cuda")
        hyq.hyq_paged_attn(cache, batch, pc.dev(qb), out, softmax_scale=1.0, mass=hyq.MASS_SET,
                           ws=pc.workspace(cache, batch, True, new))
        torch.cuda.synchronize()
        # the weights' rounding (bf16 beyond 16 rows); float32 sums of n equal weights and of the
        # rows' shares, one rounding a step, and a few around them
        w = 2.0 ** -16 if new * g <= 16 else 2.0 ** -8
        sums = (n + new * g + 16) * 2.0 ** -24
        lesser = 0.0 if power >= 20 else 6 * 2.0 ** -24 * 2.0 ** power * 1.46
        got = pc.host(out)
        assert np.isfinite(got).all(), (name, "not finite")
        np.testing.assert_allclose(got, want, rtol=0, atol=(w + sums) * np.abs(vals["v"]).max(), err_msg=name)
        np.testing.assert_allclose(pc.host(cache.bufs["mass"]), wm, rtol=sums + lesser, atol=0, err_msg=name)
