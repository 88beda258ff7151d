"""hyq_paged_attn on the GPU against the float64 oracle: outputs and the weight
every cached key received.  Tolerances are derived in paged_common."""
import math

import numpy as np
import pytest

import paged_common as pc
import paper_2608_27875_amd as hyq
from oracle import paged_oracle as po

pytestmark = pytest.mark.gpu
D = 128
SCALE = 1 / math.sqrt(D)

CASES = [
    # lens, news, Hq, Hkv, page, fmt, out_dtype, mass
    ([0], [1], 1, 1, 16, "bf16", 0, "set"),                    # the first token
    ([1], [1], 4, 1, 16, "bf16", 1, "none"),
    ([31, 32, 33], [1, 1, 1], 8, 2, 16, "bf16", 0, "add"),     # around a unit of 32
    ([700, 3], [1, 1], 8, 1, 64, "fp8", 0, "set"),
    ([500, 129], [1, 1], 5, 1, 32, "int8", 1, "add"),
    ([300], [4], 8, 2, 128, "bf16", 0, "set"),                 # drafted tokens, 16 rows
    ([77, 260], [2, 3], 15, 3, 256, "int8", 0, "add"),
    ([40], [5], 4, 1, 16, "bf16", 0, "set"),                   # 20 rows: the other kernel
    ([0], [33], 4, 1, 16, "bf16", 0, "set"),                   # a prompt from nothing
    ([63, 64], [65, 64], 4, 2, 64, "bf16", 1, "add"),          # around a tile of 64
    ([300, 0, 21], [70, 130, 1], 8, 2, 32, "fp8", 0, "set"),   # mixed: both kernels
    ([10, 400, 50], [1, 40, 0], 6, 3, 16, "int8", 0, "add"),   # one without new tokens
    ([129], [127], 1, 1, 128, "fp8", 1, "set"),
]


def reference(case, seed=0, tail=0, hole=None):
    lens, news, Hq, Hkv, page, fmt, _, mode = case
    rng = np.random.default_rng([seed, sum(lens), sum(news), Hq, page])
    cu = np.concatenate([[0], np.cumsum(news)])
    T = int(cu[-1]) + tail
    table, n_pages = pc.tables(rng, np.add(lens, news), page)
    if hole is not None:
        table[hole[0], hole[1]] = hole[2]
    bufs, vals = pc.pool(rng, fmt, n_pages, Hkv, page)
    q = pc.bits(rng, T, Hq, D)
    mass = rng.random((n_pages, Hkv, page)).astype(np.float32)
    want_mass = mass.astype(np.float64)
    want = po.attention(po.bf16(q), vals["k"], vals["v"], cu, lens, table, Hkv, SCALE, want_mass, mode)
    return dict(cu=cu, T=T, table=table, bufs=bufs, vals=vals, q=q, mass=mass, want=want,
                want_mass=want_mass, lens=lens, news=news)


def check(case, r, cache, out):
    lens, news, Hq, Hkv, page, fmt, odt, mode = case
    qv = po.bf16(r["q"])
    n = int(r["cu"][-1])
    got = pc.host(out)
    for b in range(len(lens)):
        s = slice(int(r["cu"][b]), int(r["cu"][b + 1]))
        if not news[b]:
            continue
        atol, rtol = pc.out_tolerance(qv, r["vals"], SCALE, news[b] * Hq // Hkv, odt == 1)
        np.testing.assert_allclose(got[s], r["want"][s], rtol=rtol, atol=atol)
    e = pc.logit_error(qv, r["vals"]["k"], SCALE)
    if mode != "none":
        m = pc.host(cache.bufs["mass"])
        # a weight is off by 2e of its value; sums of float32 and exponentials 2^-18
        np.testing.assert_allclose(m, r["want_mass"], rtol=2 * e + 2.0 ** -18, atol=2.0 ** -40)
        same = r["want_mass"] == r["mass"]
        assert np.array_equal(m[same], r["mass"][same].astype(np.float64))
    return got[n:]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_against_oracle(case):
    import torch
    odt, mode = case[6], case[7]
    r = reference(case, tail=2)
    cache = pc.cache_of(r["bufs"], case[5], case[2], r["mass"])
    batch = pc.batch_of(r["cu"], r["lens"], r["table"])
    out = torch.full((r["T"], case[2], D), 7.0, device="cuda",
                     dtype=torch.float32 if odt == 0 else torch.bfloat16)
    hyq.hyq_paged_attn(cache, batch, pc.dev(r["q"]), out, out_dtype=odt,
                       mass={"none": hyq.MASS_NONE, "add": hyq.MASS_ADD, "set": hyq.MASS_SET}[mode],
                       ws=pc.workspace(cache, batch, mode != "none", r["T"]))
    torch.cuda.synchronize()
    rest = check(case, r, cache, out)
    assert np.all(rest == 7.0), "rows of nobody are left as they were"
    for n in ("k", "v"):   # the pages are only read
        assert torch.equal(cache.bufs[n].view(torch.uint8), pc.dev(r["bufs"][n]).view(torch.uint8))


@pytest.mark.parametrize("case", [CASES[3], CASES[5], CASES[10]], ids=str)
def test_looser_bounds_change_nothing(case):
    """max_new, max_len and the table's width are bounds: larger ones (other
    splits, other kernels) give results within the same tolerances, and a
    step without mass leaves the mass alone."""
    import torch
    r = reference(case)
    cache = pc.cache_of(r["bufs"], case[5], case[2], r["mass"])
    wide = np.concatenate([r["table"], np.full((len(r["lens"]), 70), -5, np.int32)], axis=1)
    batch = pc.batch_of(r["cu"], r["lens"], wide, max_new=max(r["news"]) + 37, max_len=max(r["lens"]) + 9000)
    out = torch.empty((r["T"], case[2], D), dtype=torch.float32, device="cuda")
    hyq.hyq_paged_attn(cache, batch, pc.dev(r["q"]), out, ws=pc.workspace(cache, batch, False, r["T"]))
    torch.cuda.synchronize()
    check(case[:6] + (0, "none"), r, cache, out)
    assert np.array_equal(cache.bufs["mass"].cpu().numpy(), r["mass"])


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "int8"])
@pytest.mark.parametrize("new,max_len", [(1, 100), (40, 100), (40, 9000)])
def test_holes_and_poison(fmt, new, max_len):
    """Keys of missing pages take no part; what lies behind the sequences and in
    pages of nobody may be NaN.  (A bound of 9000 slots: workgroups of 8 waves.)"""
    import torch
    for hole in ((0, 0, -1), (0, 2, 1 << 29), (0, 6, -7)):
        case = ([100], [new], 4, 1, 16, fmt, 0, "set")
        r = reference(case, seed=hole[1], hole=hole)
        owned = np.zeros(r["bufs"]["k"].shape[:1] + (16,), dtype=bool)
        for n in range(100 + new):
            at = po.place(r["table"], 0, n, 16, len(owned))
            if at:
                owned[at] = True
        for name in ("k", "v"):
            if fmt == "bf16":
                r["bufs"][name].transpose(0, 2, 1, 3)[~owned] = 0x7FC0   # NaN
            else:
                if fmt == "fp8":
                    r["bufs"][name].transpose(0, 2, 1, 3)[~owned] = 0x7F   # NaN
                r["bufs"][name + "_scale"].transpose(0, 2, 1)[~owned] = np.nan
        cache = pc.cache_of(r["bufs"], fmt, 4, r["mass"])
        batch = pc.batch_of(r["cu"], r["lens"], r["table"], max_len=max_len)
        out = torch.empty((new, 4, D), dtype=torch.float32, device="cuda")
        hyq.hyq_paged_attn(cache, batch, pc.dev(r["q"]), out, mass=hyq.MASS_SET,
                           ws=pc.workspace(cache, batch, True, new))
        torch.cuda.synchronize()
        check(case, r, cache, out)


@pytest.mark.parametrize("new", [1, 30])
def test_rows_that_see_nothing(new):
    """Every page missing: zero output, untouched mass."""
    import torch
    case = ([50], [new], 8, 2, 32, "bf16", 0, "set")
    r = reference(case)
    cache = pc.cache_of(r["bufs"], "bf16", 8, r["mass"])
    batch = pc.batch_of(r["cu"], r["lens"], np.full_like(r["table"], -1))
    out = torch.full((new, 8, D), 3.0, device="cuda")
    hyq.hyq_paged_attn(cache, batch, pc.dev(r["q"]), out, mass=hyq.MASS_SET,
                       ws=pc.workspace(cache, batch, True, new))
    torch.cuda.synchronize()
    assert torch.all(out == 0)
    assert np.array_equal(cache.bufs["mass"].cpu().numpy(), r["mass"])


@pytest.mark.parametrize("new,max_len", [(2, 90), (60, 90), (80, 9000)])
def test_extreme_logits(new, max_len):
    """Logits of a few thousand either way: one key takes all the weight, and
    rows whose logits are all far below zero are still a softmax."""
    import torch
    rng = np.random.default_rng(1)
    lens, page, n = [90], 16, 90 + new
    table, n_pages = pc.tables(rng, [n], page)
    bufs, vals = pc.pool(rng, "bf16", n_pages, 1, page)
    q = pc.bits(rng, new, 2, D, scale=30.0)
    q[:, 1] = pc.bits(rng, new, D, scale=0.01)
    cu = np.array([0, new])
    want = po.attention(po.bf16(q), vals["k"], vals["v"], cu, lens, table, 1, SCALE)
    cache = pc.cache_of(bufs, "bf16", 2)
    batch = pc.batch_of(cu, lens, table, max_len=max_len)
    out = torch.empty((new, 2, D), device="cuda")
    hyq.hyq_paged_attn(cache, batch, pc.dev(q), out, ws=pc.workspace(cache, batch, False, new))
    atol, rtol = pc.out_tolerance(po.bf16(q), vals, SCALE, 2 * new, False)
    np.testing.assert_allclose(pc.host(out), want, rtol=rtol, atol=atol)


@pytest.mark.parametrize("new,max_len", [(1, 400), (30, 400), (70, 9000)])
def test_rising_and_falling_logits(new, max_len):
    """Keys along the query, each hundred far larger (or smaller) than the one
    before: the reference of a row's weights has to follow."""
    import torch
    rng = np.random.default_rng(2)
    g, page, n = 4, 32, 400
    table, n_pages = pc.tables(rng, [n + new], page)
    for sign in (1, -1):
        bufs, _ = pc.pool(rng, "bf16", n_pages, 1, page)
        q = np.zeros((new, g, D), dtype=np.float32)
        q[..., 0] = 1 + rng.random((new, g))
        k = po.bf16(bufs["k"])
        for s in range(n + new):
            p, o = po.place(table, 0, s, page, n_pages)
            k[p, 0, o, 0] = sign * 700.0 * (s // 100) + 8 * rng.standard_normal()
        bufs["k"] = hyq_bits(k)
        qb = hyq_bits(q)
        vals = dict(k=po.bf16(bufs["k"]), v=po.bf16(bufs["v"]))
        mass = np.zeros((n_pages, 1, page), np.float32)
        wm = mass.astype(np.float64)
        cu = np.array([0, new])
        want = po.attention(po.bf16(qb), vals["k"], vals["v"], cu, [n], table, 1, 1.0, wm, "set")
        cache = pc.cache_of(bufs, "bf16", g, mass)
        batch = pc.batch_of(cu, [n], table, max_len=max_len)
        out = torch.empty((new, g, D), device="cuda")
        hyq.hyq_paged_attn(cache, batch, pc.dev(qb), out, softmax_scale=1.0, mass=hyq.MASS_SET,
                           ws=pc.workspace(cache, batch, True, new))
        # one product (channel 0) carries the logits: exact to float32, up to 6000 (2^-11 absolute)
        w = 2.0 ** -16 if new * g <= 16 else 2.0 ** -8
        atol = (2.0 ** -9 + w) * np.abs(vals["v"]).max()
        np.testing.assert_allclose(pc.host(out), want, rtol=2.0 ** -20, atol=atol)
        got = pc.host(cache.bufs["mass"])
        np.testing.assert_allclose(got[wm > 1e-30], wm[wm > 1e-30], rtol=2.0 ** -8)
        assert np.all(got[wm < 1e-60] < 1e-30)


def hyq_bits(x):
    from paper_2608_27875_amd import gen
    return gen.f32_to_bf16_bits(np.asarray(x, dtype=np.float32))


def test_mixed_batch_with_splits():
    """A long chunk and single tokens whose keys are split too: both kernels
    leave partials in one workspace; masses of both."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(3)
    Hq, Hkv, page = 8, 2, 32
    lens, news = [5000, 3001, 0, 4100], [33, 1, 20, 2]
    cu = [0, 33, 34, 54, 56]
    used = [-(-(a + n) // page) for a, n in zip(lens, news)]
    perm = torch.randperm(sum(used) + 1, generator=g, device="cuda").to(torch.int32)
    k = torch.randn((sum(used) + 1, Hkv, page, D), generator=g, device="cuda").bfloat16()
    v = torch.randn((sum(used) + 1, Hkv, page, D), generator=g, device="cuda").bfloat16()
    q = torch.randn((56, Hq, D), generator=g, device="cuda").bfloat16()
    mass = torch.zeros((sum(used) + 1, Hkv, page), device="cuda")
    table = torch.full((4, max(used)), -1, dtype=torch.int32, device="cuda")
    for b, u in enumerate(used):
        table[b, :u] = perm[sum(used[:b]):sum(used[:b + 1])]
    cache = hyq.PagedCache(Hq=Hq, Hkv=Hkv, page=page, n_pages=k.shape[0], device=k.device,
                           bufs=dict(k=k, v=v, mass=mass))
    batch = pc.batch_of(cu, lens, table.cpu().numpy())
    out = torch.empty((56, Hq, D), device="cuda")
    hyq.hyq_paged_attn(cache, batch, q, out, mass=hyq.MASS_SET, ws=pc.workspace(cache, batch, True, 56))
    e = 130 * 2.0 ** -24 * SCALE * 128 * 30   # as in test_long
    for b in range(4):
        p = table[b, :used[b]].long()
        n = lens[b] + news[b]
        kk, vv = (x[p].transpose(0, 1).reshape(Hkv, -1, D)[:, :n] for x in (k, v))
        want, wm = plain(q[cu[b]:cu[b + 1]], kk, vv, lens[b])
        w = 2.0 ** -16 if news[b] * 4 <= 16 else 2.0 ** -8
        off = (out[cu[b]:cu[b + 1]].double() - want).abs().max()
        assert float(off) <= (2 * e + w) * float(v.float().abs().max())
        got = mass[p].transpose(0, 1).reshape(Hkv, -1)[:, :n]
        np.testing.assert_allclose(pc.host(got), wm.cpu().numpy(), rtol=2 * e + 2.0 ** -18)


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
def test_long_codes(fmt):
    """8-bit pages in a long chunk (eight waves, splits): against float64 on
    what the codes stand for."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(9)
    Hq, Hkv, page, len0, new = 5, 1, 64, 6500, 301
    pages = -(-(len0 + new) // page)
    rows = (pages, Hkv, page)
    if fmt == "int8":
        codes = [torch.randint(-127, 128, rows + (D,), generator=g, device="cuda").to(torch.int8) for _ in "kv"]
        vals = [c.double() for c in codes]
    else:
        codes = [(torch.randn(rows + (D,), generator=g, device="cuda") * 150).clamp(-448, 448)
                 .to(torch.float8_e4m3fn) for _ in "kv"]
        vals = [c.float().double() for c in codes]
    scales = [torch.rand(rows, generator=g, device="cuda") / 60 for _ in "kv"]
    scales[0][0, 0, 3] = 0   # a row of zeros
    codes = [c.view(torch.uint8) for c in codes]
    codes[0][0, 0, 3] = 0
    vals[0][0, 0, 3] = 0
    k, v = (x * s[..., None].double() for x, s in zip(vals, scales))
    bits, kind = pc.FORMATS[fmt]
    mass = torch.zeros(rows, device="cuda")
    cache = hyq.PagedCache(Hq=Hq, Hkv=Hkv, page=page, n_pages=pages, device=mass.device, bits_kv=bits,
                           kv_format=kind, bufs=dict(k=codes[0], v=codes[1], k_scale=scales[0],
                                                     v_scale=scales[1], mass=mass))
    q = torch.randn((new, Hq, D), generator=g, device="cuda").bfloat16()
    batch = pc.batch_of([0, new], [len0], np.arange(pages, dtype=np.int32)[None])
    out = torch.empty((new, Hq, D), device="cuda")
    hyq.hyq_paged_attn(cache, batch, q, out, mass=hyq.MASS_SET, ws=pc.workspace(cache, batch, True, new))
    kk, vv = (x.transpose(0, 1).reshape(Hkv, -1, D)[:, :len0 + new] for x in (k, v))
    want, wm = plain(q, kk, vv, len0)
    big = float(q.double().abs().amax((0, 1)) @ kk[0].abs().amax(0))
    e = SCALE * big * 130 * 2.0 ** -24
    # the worst case of 2^-8 a weight, and a mean error far below it
    assert float((out.double() - want).abs().max()) <= (2 * e + 2.0 ** -8) * float(vv.abs().max())
    assert float((out.double() - want).norm()) <= 2.0 ** -8 * float(want.norm()) + 2 * e * float(vv.abs().max())
    got = mass.transpose(0, 1).reshape(Hkv, -1)[:, :len0 + new]
    np.testing.assert_allclose(pc.host(got), wm.cpu().numpy(), rtol=2 * e + 2.0 ** -18)


def test_two_streams_at_once():
    """Two steps in flight on two streams, each with its own workspace."""
    import torch
    r = [reference(c, seed=4) for c in (CASES[10], CASES[3])]
    cases = [CASES[10], CASES[3]]
    jobs = []
    for c, x in zip(cases, r):
        cache = pc.cache_of(x["bufs"], c[5], c[2], x["mass"])
        batch = pc.batch_of(x["cu"], x["lens"], x["table"], max_len=6000)
        out = torch.empty((x["T"], c[2], D), device="cuda")
        jobs.append((cache, batch, pc.dev(x["q"]), out, pc.workspace(cache, batch, True, x["T"]),
                     torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for cache, batch, q, out, ws, st in jobs:
            hyq.hyq_paged_attn(cache, batch, q, out, mass=hyq.MASS_SET, ws=ws, stream=st)
    torch.cuda.synchronize()
    for c, x, (cache, _, _, out, _, _) in zip(cases, r, jobs):
        check(c[:6] + (0, "set"), x, cache, out)


def plain(q, k, v, len0):
    """float64 attention of q [n, Hq, D] over k, v [Hkv, N, D], and the masses."""
    import torch
    n, Hq, _ = q.shape
    Hkv, N, _ = k.shape
    g = Hq // Hkv
    out = torch.empty((n, Hq, D), dtype=torch.float64, device=q.device)
    mass = torch.zeros((Hkv, N), dtype=torch.float64, device=q.device)
    hidden = torch.arange(N, device=q.device) > len0 + torch.arange(n, device=q.device)[:, None]
    for h in range(Hq):
        z = (q[:, h].double() @ k[h // g].double().T.contiguous()) * SCALE
        w = torch.softmax(z.masked_fill(hidden, -math.inf), -1)
        out[:, h] = w @ v[h // g].double()
        mass[h // g] += w.sum(0)
    return out, mass


@pytest.mark.parametrize("len0,new,Hq,Hkv,page,fmt", [
    (32749, 1, 8, 2, 64, "bf16"), (20011, 3, 10, 2, 16, "bf16"), (9000, 777, 8, 2, 128, "bf16"),
    (40001, 130, 5, 1, 256, "bf16"), (0, 1500, 4, 1, 32, "bf16"), (131071, 1, 8, 1, 64, "bf16"),
    (70003, 2, 4, 1, 16, "bf16"),
])
def test_long(len0, new, Hq, Hkv, page, fmt):
    """Long sequences (many splits, many tiles), every output and mass."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(len0 + new)
    N = len0 + new
    pages = -(-N // page)
    perm = torch.randperm(pages + 2, generator=g, device="cuda")[:pages].to(torch.int32)
    k = torch.randn((pages + 2, Hkv, page, D), generator=g, device="cuda").bfloat16()
    v = torch.randn((pages + 2, Hkv, page, D), generator=g, device="cuda").bfloat16()
    q = torch.randn((new, Hq, D), generator=g, device="cuda").bfloat16()
    mass = torch.zeros((pages + 2, Hkv, page), device="cuda")
    cache = hyq.PagedCache(Hq=Hq, Hkv=Hkv, page=page, n_pages=pages + 2, device=k.device,
                           bufs=dict(k=k, v=v, mass=mass))
    batch = pc.batch_of([0, new], [len0], perm.cpu().numpy()[None])
    out = torch.empty((new, Hq, D), device="cuda")
    hyq.hyq_paged_attn(cache, batch, q, out, mass=hyq.MASS_ADD, ws=pc.workspace(cache, batch, True, new))
    kk = k[perm.long()].transpose(0, 1).reshape(Hkv, -1, D)[:, :N]
    vv = v[perm.long()].transpose(0, 1).reshape(Hkv, -1, D)[:, :N]
    want, wm = plain(q, kk, vv, len0)
    # here |z| <= 130 2^-24 SCALE sum |q k|, of at most 128 * 5.5 * 5.5 (normal values)
    e = 130 * 2.0 ** -24 * SCALE * 128 * 30
    w = 2.0 ** -16 if new * Hq // Hkv <= 16 else 2.0 ** -8
    # weights' roundings are independent: the worst case of them all is 2^-8 max |V|
    assert float((out.double() - want).abs().max()) <= (2 * e + w) * float(v.float().abs().max())
    got = mass[perm.long()].transpose(0, 1).reshape(Hkv, -1)
    np.testing.assert_allclose(pc.host(got[:, :N]), wm.cpu().numpy(), rtol=2 * e + 2.0 ** -18)
    assert torch.all(got[:, N:] == 0)
    # a mean error far below the worst case: no systematic loss
    assert float((out.double() - want).abs().mean()) <= 2.0 ** -9 * float(want.abs().mean()) + 2 * e


def test_offsets_beyond_32_bits():
    """Pages whose byte and element offsets pass 2^32."""
    import torch
    Hkv, page = 8, 256
    n_pages = (1 << 32) // (Hkv * page * D) + 40   # elements beyond 2^32
    k = torch.zeros((n_pages, Hkv, page, D), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    g = torch.Generator(device="cuda").manual_seed(1)
    ids = torch.tensor([n_pages - 1, 0, n_pages - 20], dtype=torch.int32)
    for p in ids.tolist():
        k[p] = torch.randn((Hkv, page, D), generator=g, device="cuda").bfloat16()
        v[p] = torch.randn((Hkv, page, D), generator=g, device="cuda").bfloat16()
    cache = hyq.PagedCache(Hq=8, Hkv=Hkv, page=page, n_pages=n_pages, device=k.device,
                           bufs=dict(k=k, v=v))
    for new in (1, 100):
        len0 = 700 - new
        q = torch.randn((new, 8, D), generator=g, device="cuda").bfloat16()
        batch = pc.batch_of([0, new], [len0], ids.numpy()[None])
        out = torch.empty((new, 8, D), device="cuda")
        hyq.hyq_paged_attn(cache, batch, q, out, ws=pc.workspace(cache, batch, False, new))
        kk = k[ids.long().cuda()].transpose(0, 1).reshape(Hkv, -1, D)[:, :700]
        vv = v[ids.long().cuda()].transpose(0, 1).reshape(Hkv, -1, D)[:, :700]
        want, _ = plain(q, kk, vv, len0)
        assert float((out.double() - want).abs().max()) <= (2.0 ** -13 if new == 1 else 2.0 ** -8) * 6
    del k, v, cache
    torch.cuda.empty_cache()


def test_shared_pages():
    """Two sequences with the same prompt pages (only read) and own last pages."""
    import torch
    rng = np.random.default_rng(5)
    bufs, vals = pc.pool(rng, "bf16", 6, 2, 16)
    table = np.array([[3, 1, 0], [3, 1, 5]], dtype=np.int32)
    cu, lens = np.array([0, 1, 2]), [40, 36]
    q = pc.bits(rng, 2, 4, D)
    want = po.attention(po.bf16(q), vals["k"], vals["v"], cu, lens, table, 2, SCALE)
    cache = pc.cache_of(bufs, "bf16", 4)
    batch = pc.batch_of(cu, lens, table)
    out = torch.empty((2, 4, D), device="cuda")
    hyq.hyq_paged_attn(cache, batch, pc.dev(q), out, ws=pc.workspace(cache, batch, False, 2))
    atol, rtol = pc.out_tolerance(po.bf16(q), vals, SCALE, 2, False)
    np.testing.assert_allclose(pc.host(out), want, rtol=rtol, atol=atol)


def test_no_new_tokens():
    """T = 0 enqueues nothing; a batch of sequences without new tokens changes nothing."""
    import torch
    rng = np.random.default_rng(6)
    bufs, _ = pc.pool(rng, "bf16", 4, 1, 16)
    mass = rng.random((4, 1, 16)).astype(np.float32)
    cache = pc.cache_of(bufs, "bf16", 1, mass)
    empty = torch.empty((0, 1, D), dtype=torch.bfloat16, device="cuda")
    hyq.hyq_paged_attn(cache, pc.batch_of([0, 0], [10], [[1]], max_new=0), empty, empty.float())
    for max_new in (1, 50):
        batch = pc.batch_of([0, 0, 0], [10, 0], [[1], [2]], max_new=max_new)
        out = torch.full((3, 1, D), 2.0, device="cuda")
        q = torch.zeros((3, 1, D), dtype=torch.bfloat16, device="cuda")
        hyq.hyq_paged_attn(cache, batch, q, out, mass=hyq.MASS_SET, ws=pc.workspace(cache, batch, True, 3))
        torch.cuda.synchronize()
        assert torch.all(out == 2.0)
    assert np.array_equal(cache.bufs["mass"].cpu().numpy(), mass)


def test_same_bits_every_time():
    """Nothing depends on the order of workgroups."""
    import torch
    for case in (CASES[10], CASES[3]):
        r = reference(case)
        got = []
        for _ in range(4):
            cache = pc.cache_of(r["bufs"], case[5], case[2], r["mass"])
            batch = pc.batch_of(r["cu"], r["lens"], r["table"], max_len=5000)
            out = torch.empty((r["T"], case[2], D), device="cuda")
            hyq.hyq_paged_attn(cache, batch, pc.dev(r["q"]), out, mass=hyq.MASS_SET,
                               ws=pc.workspace(cache, batch, True, r["T"]))
            got.append((out.clone(), cache.bufs["mass"].clone()))
        for o, m in got[1:]:
            assert torch.equal(o, got[0][0]) and torch.equal(m, got[0][1])


@pytest.mark.parametrize("lens", [[-3, 40], [400, 40]])
def test_lengths_beyond_their_bounds(lens):
    """Device lengths outside [0, max_len] count as the nearest bound."""
    import torch
    rng = np.random.default_rng(7)
    bufs, vals = pc.pool(rng, "bf16", 12, 1, 16)
    table = rng.permutation(12).reshape(2, 6).astype(np.int32)
    cu = np.array([0, 1, 2])
    q = pc.bits(rng, 2, 2, D)
    clipped = np.clip(lens, 0, 60)
    want = po.attention(po.bf16(q), vals["k"], vals["v"], cu, clipped, table, 1, SCALE)
    cache = pc.cache_of(bufs, "bf16", 2)
    batch = pc.batch_of(cu, lens, table, max_len=60)
    out = torch.empty((2, 2, D), device="cuda")
    hyq.hyq_paged_attn(cache, batch, pc.dev(q), out, ws=pc.workspace(cache, batch, False, 2))
    atol, rtol = pc.out_tolerance(po.bf16(q), vals, SCALE, 2, False)
    np.testing.assert_allclose(pc.host(out), want, rtol=rtol, atol=atol)
