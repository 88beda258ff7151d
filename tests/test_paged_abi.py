"""The paged serving calls without a GPU: sizes, and every refusal before
anything is enqueued (no device exists here)."""
import ctypes
import os

import pytest

import paper_2608_27875_amd as hyq

EINVAL, EUNSUP = hyq.HYQ_EINVAL, hyq.HYQ_EUNSUPPORTED
FAKE = 0x1000   # never dereferenced: the calls fail first
OUT, WS = 1 << 40, 1 << 44   # outputs and a workspace elsewhere


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(hyq.LIB_PATH):
        from paper_2608_27875_amd import build
        build.build()
    return hyq.lib()


def cache(**kw):
    c = hyq._PCache(8, 2, 128, 16, 10, 16, 0, FAKE, FAKE, FAKE, FAKE, FAKE)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def batch(**kw):
    b = hyq._PBatch(2, 6, 4, 100, 8, FAKE, FAKE, FAKE)
    for k, v in kw.items():
        setattr(b, k, v)
    return b


def rope(**kw):
    r = hyq._Rope(128, 0, 1e-6, FAKE, FAKE, FAKE)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


BAD_CACHE = [
    (dict(Hq=0), EINVAL), (dict(Hkv=0), EINVAL), (dict(Hq=7), EINVAL), (dict(n_pages=0), EINVAL),
    (dict(page=8), EINVAL), (dict(page=48), EINVAL), (dict(page=512), EINVAL),
    (dict(bits_kv=4), EUNSUP), (dict(bits_kv=8, kv_format=hyq.FMT_FP4), EUNSUP),
    (dict(D=64), EUNSUP), (dict(Hq=18), EUNSUP),
]
BAD_BUFFERS = [(dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(k=FAKE + 8), EINVAL),
               (dict(mass=FAKE + 4), EINVAL), (dict(bits_kv=8, k_scale=None), EINVAL),
               (dict(bits_kv=8, v_scale=None), EINVAL)]
BAD_BATCH = [
    (dict(B=0), EINVAL), (dict(T=-1), EINVAL), (dict(max_new=-1), EINVAL), (dict(max_len=-1), EINVAL),
    (dict(max_pages=0), EINVAL), (dict(max_len=1 << 23), EUNSUP), (dict(T=1 << 24), EUNSUP),
    (dict(B=20000), EUNSUP), (dict(B=16000, T=1 << 20, max_new=1 << 20), EUNSUP), (dict(cu_new=None), EINVAL), (dict(lens=None), EINVAL),
    (dict(table=None), EINVAL),
]
BAD_ROPE = [
    (dict(rot_dim=-16), EINVAL), (dict(rot_dim=144), EINVAL), (dict(rot_dim=24), EINVAL),
    (dict(interleaved=2), EINVAL), (dict(eps=-1.0), EINVAL), (dict(eps=float("nan")), EINVAL),
    (dict(eps=float("inf")), EINVAL), (dict(inv_freq=None), EINVAL), (dict(q_weight=FAKE + 2), EINVAL),
]


def append(lib, c=None, b=None, r=None, q=FAKE, qs=1024, k=FAKE, ks=256, v=FAKE, vs=256, pos=FAKE, out=OUT):
    return lib.hyq_paged_append(c or cache(), b or batch(), r or rope(), q, qs, k, ks, v, vs, pos, out, None)


def attn(lib, c=None, b=None, q=FAKE, scale=0.1, mass=0, out=OUT, odt=0, ws=WS, wsb=1 << 40):
    return lib.hyq_paged_attn(c or cache(), b or batch(), q, ctypes.c_float(scale), mass, out, odt, ws,
                              ctypes.c_size_t(wsb), None)


def evict(lib, c=None, B=2, lens=FAKE, table=FAKE, max_pages=8, max_len=100, budget=40, recent=4,
          new_table=FAKE, new_pages=3, keep=FAKE, new_lens=0x9000):
    return lib.hyq_evict(c or cache(), B, lens, table, max_pages, max_len, budget, recent, new_table,
                         new_pages, keep, new_lens, None)


def norm_rope(lib, s=None, r=None, q=FAKE, qs=1024, k=FAKE, ks=256, v=FAKE, vs=256, pos=FAKE, Q=OUT,
              K=OUT << 1, V=OUT << 2):
    s = s or hyq.Shape(B=1, Hq=8, Hkv=2, L=4)
    return lib.hyq_norm_rope(s.c(), r or rope(), q, qs, k, ks, v, vs, pos, Q, K, V, None)


@pytest.mark.parametrize("kw,code", BAD_CACHE + BAD_BUFFERS)
def test_bad_caches(lib, kw, code):
    assert append(lib, c=cache(**kw)) == code
    assert attn(lib, c=cache(**kw)) == code
    assert evict(lib, c=cache(**kw)) == code
    assert hyq.hyq_last_error()
    if (kw, code) in BAD_CACHE:
        n = ctypes.c_size_t()
        assert lib.hyq_paged_ws_bytes(cache(**kw), batch(), 0, ctypes.byref(n)) == code
        c = cache(**kw)
        out = hyq._PCache()
        assert lib.hyq_pcache_init(c.Hq, c.Hkv, c.D, c.page, c.n_pages, c.bits_kv, c.kv_format, out,
                                   None) == code


@pytest.mark.parametrize("kw,code", BAD_BATCH)
def test_bad_batches(lib, kw, code):
    assert append(lib, b=batch(**kw)) == code
    assert attn(lib, b=batch(**kw)) == code


@pytest.mark.parametrize("kw,code", BAD_ROPE)
def test_bad_ropes(lib, kw, code):
    assert append(lib, r=rope(**kw)) == code
    assert norm_rope(lib, r=rope(**kw)) == code


@pytest.mark.parametrize("kw", [dict(q=None), dict(out=None), dict(k=None), dict(v=None), dict(pos=None),
                                dict(qs=1023), dict(qs=1020), dict(ks=255), dict(vs=-256),
                                dict(q=FAKE + 2), dict(k=FAKE + 8), dict(v=FAKE + 4), dict(out=FAKE + 8)])
def test_bad_append_arguments(lib, kw):
    assert append(lib, **kw) == EINVAL


@pytest.mark.parametrize("kw", [dict(q=None), dict(Q=None), dict(pos=None), dict(K=None), dict(k=None),
                                dict(v=None), dict(V=None), dict(qs=1016), dict(ks=8), dict(vs=257),
                                dict(q=FAKE + 2), dict(Q=FAKE + 2), dict(K=FAKE + 2), dict(V=FAKE + 2)])
def test_bad_norm_rope_arguments(lib, kw):
    assert norm_rope(lib, **kw) == EINVAL


def test_bad_norm_rope_shapes(lib):
    assert norm_rope(lib, s=hyq.Shape(B=0, Hq=8, Hkv=2, L=4)) == EINVAL
    assert norm_rope(lib, s=hyq.Shape(B=1, Hq=8, Hkv=2, L=4, D=64)) == EUNSUP
    assert norm_rope(lib, s=hyq.Shape(B=1 << 12, Hq=8, Hkv=2, L=1 << 12)) == EUNSUP


@pytest.mark.parametrize("kw", [dict(q=None), dict(out=None), dict(scale=0.0), dict(scale=-1.0),
                                dict(scale=float("nan")), dict(scale=float("inf")), dict(mass=3),
                                dict(mass=-1), dict(odt=2), dict(q=FAKE + 2), dict(out=FAKE + 8),
                                dict(ws=None, mass=1), dict(wsb=15, mass=1), dict(ws=FAKE + 8, mass=1)])
def test_bad_attention_arguments(lib, kw):
    assert attn(lib, **kw) == EINVAL


APART = 6 * 8 * 256    # bytes of q's rows in `batch`: T = 6, 8 heads


@pytest.mark.parametrize("kw", [dict(out=FAKE), dict(out=FAKE + APART - 16), dict(q=OUT + 2 * APART - 16),
                                dict(odt=1, out=FAKE), dict(mass=1, ws=FAKE), dict(mass=1, ws=OUT + 16)])
def test_attention_outputs_apart_from_inputs(lib, kw):
    assert attn(lib, **kw) == EINVAL
    assert "overlap" in hyq.hyq_last_error()


@pytest.mark.parametrize("kw", [dict(out=FAKE), dict(k=OUT + APART - 16), dict(v=OUT),
                                dict(q=OUT - 5 * 4096 * 2, qs=4096), dict(k=OUT - 16, ks=4096)])
def test_appended_queries_apart_from_inputs(lib, kw):
    assert append(lib, **kw) == EINVAL
    assert "overlap" in hyq.hyq_last_error()


@pytest.mark.parametrize("kw", [dict(Q=FAKE), dict(K=FAKE), dict(V=FAKE), dict(q=OUT + 4 * 8 * 256 - 16),
                                dict(v=(OUT << 1) - 3 * 8192, vs=4096), dict(k=(OUT << 2) + 16)])
def test_norm_rope_outputs_apart_from_inputs(lib, kw):
    assert norm_rope(lib, **kw) == EINVAL
    assert "overlap" in hyq.hyq_last_error()


def test_mass_needs_a_buffer(lib):
    assert attn(lib, c=cache(mass=None), mass=hyq.MASS_ADD) == EINVAL
    assert evict(lib, c=cache(mass=None)) == EINVAL


@pytest.mark.parametrize("kw", [dict(B=0), dict(max_pages=0), dict(max_len=-1), dict(new_pages=0),
                                dict(budget=0), dict(recent=-1), dict(recent=41), dict(budget=49),
                                dict(lens=None), dict(table=None), dict(new_table=None), dict(keep=None),
                                dict(new_lens=None), dict(new_lens=FAKE), dict(new_lens=FAKE + 4)])
def test_bad_evictions(lib, kw):
    assert evict(lib, **kw) == EINVAL


def test_too_large_evictions(lib):
    assert evict(lib, max_len=(1 << 22) + 1) == EUNSUP
    assert evict(lib, B=20000) == EUNSUP


def test_null_structs(lib):
    n = ctypes.c_size_t()
    assert lib.hyq_paged_append(None, batch(), rope(), *[FAKE, 1024, FAKE, 256, FAKE, 256, FAKE, FAKE], None) == EINVAL
    assert lib.hyq_paged_append(cache(), None, rope(), *[FAKE, 1024, FAKE, 256, FAKE, 256, FAKE, FAKE], None) == EINVAL
    assert lib.hyq_paged_append(cache(), batch(), None, *[FAKE, 1024, FAKE, 256, FAKE, 256, FAKE, FAKE], None) == EINVAL
    assert lib.hyq_paged_ws_bytes(cache(), None, 0, ctypes.byref(n)) == EINVAL
    assert lib.hyq_paged_ws_bytes(cache(), batch(), 7, ctypes.byref(n)) == EINVAL
    assert lib.hyq_paged_ws_bytes(cache(), batch(), 0, None) == EINVAL
    assert lib.hyq_pcache_init(8, 2, 128, 16, 10, 16, 0, None, None) == EINVAL


def test_nothing_to_do_is_no_error(lib):
    """No token rows: no array is read, nothing is enqueued."""
    for kw in (dict(T=0), dict(max_new=0)):
        b = batch(cu_new=None, lens=None, table=None, **kw)
        n = ctypes.c_size_t(5)
        assert lib.hyq_paged_ws_bytes(cache(), b, 1, ctypes.byref(n)) == 0 and n.value == 0
        assert append(lib, b=b, q=None, k=None, v=None, pos=None, out=None) == 0
        assert attn(lib, b=b, q=None, out=None, ws=None, wsb=0) == 0


@pytest.mark.parametrize("bits,fmt", [(16, 0), (8, hyq.FMT_INT), (8, hyq.FMT_FP8)])
def test_sizes(lib, bits, fmt):
    c, z = hyq.hyq_pcache_init(40, 8, 64, 1000, bits, fmt)
    rows = 1000 * 8 * 64
    assert z == dict(kv_bytes=rows * 128 * bits // 8, scale_bytes=rows * 4 if bits == 8 else 0,
                     mass_bytes=rows * 4)
    assert (c.Hq, c.Hkv, c.D, c.page, c.n_pages, c.bits_kv, c.kv_format) == (40, 8, 128, 64, 1000, bits, fmt)
    assert not any(getattr(c, n) for n in ("k", "v", "k_scale", "v_scale", "mass"))


@pytest.mark.parametrize("max_new", [1, 2, 4, 5, 100, 2048])
@pytest.mark.parametrize("B,Hq,Hkv", [(1, 1, 1), (1, 32, 8), (7, 40, 8), (64, 32, 8)])
def test_workspace_grows_with_the_batch(lib, B, Hq, Hkv, max_new):
    """A workspace for T token rows serves every smaller T, and one for a step
    with masses also one without."""
    c, _ = hyq.hyq_pcache_init(Hq, Hkv, 32, 1000)
    for max_len in (0, 1000, 32768):
        last = 0
        for T in (1, B, B * max_new // 2 + 1, B * max_new):
            b = hyq._PBatch(B, T, max_new, max_len, 1 << 16, None, None, None)
            n = [ctypes.c_size_t() for _ in range(2)]
            for m in range(2):
                assert lib.hyq_paged_ws_bytes(c, b, m, ctypes.byref(n[m])) == 0
            assert n[0].value <= n[1].value
            if T > 1:
                assert n[1].value >= last or T < B
            last = max(last, n[1].value) if T >= B else last


def test_workspace_of_a_mixed_batch(lib):
    """The splits of a single token do not multiply the rows of the chunk beside it:
    one KV head's partials of 16 rows in 256 splits, 520 bytes each."""
    c, _ = hyq.hyq_pcache_init(8, 1, 32, 1000)
    n = ctypes.c_size_t()
    b = hyq._PBatch(2, 4096, 4095, 1 << 17, 1 << 16, None, None, None)
    assert lib.hyq_paged_ws_bytes(c, b, 0, ctypes.byref(n)) == 0
    assert n.value <= 2 * 16 * 256 * 520 + 4096


def test_binding_checks():
    """The binding refuses tensors of other shapes, types and places."""
    import torch
    bf = torch.bfloat16
    x = torch.zeros((4, 12, 128), dtype=bf)
    with pytest.raises(ValueError):
        hyq._row_args(x[:, :8], "q", 4, 7, 128, x.device)
    with pytest.raises(TypeError):
        hyq._row_args(x[:, :8].float(), "q", 4, 8, 128, x.device)
    with pytest.raises(ValueError):
        hyq._row_args(x[:, ::2], "q", 4, 6, 128, x.device)
    with pytest.raises(ValueError):
        hyq._row_args(x[:, :8], "q", 4, 8, 128, torch.device("meta"))
    assert hyq._row_args(x[:, 8:], "k", 4, 4, 128, x.device) == (x.data_ptr() + 8 * 256, 12 * 128)
    assert hyq._row_args(x[:1, 8:], "k", 1, 4, 128, x.device)[1] == 4 * 128
    i32 = torch.int32
    with pytest.raises(ValueError):
        hyq.PagedBatch(torch.zeros(3, dtype=i32), torch.zeros(2, dtype=i32), torch.zeros(4, dtype=i32), 1, 1)
    with pytest.raises(ValueError):
        hyq.PagedBatch(torch.zeros(2, dtype=i32), torch.zeros(2, dtype=i32), torch.zeros((2, 4), dtype=i32), 1, 1)
    with pytest.raises(TypeError):
        hyq.PagedBatch(torch.zeros(3), torch.zeros(2, dtype=i32), torch.zeros((2, 4), dtype=i32), 1, 1)
    with pytest.raises(TypeError):
        hyq.Rope(q_weight=torch.ones(128), inv_freq=torch.ones(64))
    with pytest.raises(ValueError):
        hyq.Rope(rot_dim=64, inv_freq=torch.ones(31))
    with pytest.raises(ValueError):
        hyq.Rope(rot_dim=64)
    with pytest.raises(ValueError):   # buffers smaller than the pool
        hyq.PagedCache(8, 2, 16, 10, "cpu", bufs=dict(k=torch.zeros(5, dtype=bf), v=torch.zeros(5, dtype=bf)))
    with pytest.raises(ValueError):   # 8 bits without scales
        u = torch.zeros(10 * 2 * 16 * 128, dtype=torch.uint8)
        hyq.PagedCache(8, 2, 16, 10, "cpu", bits_kv=8, bufs=dict(k=u, v=u))
    with pytest.raises(hyq.HyqError) as e:
        hyq.PagedCache(8, 2, 17, 10, "cpu")
    assert e.value.code == EINVAL
    c = hyq.PagedCache(8, 2, 16, 10, "cpu", mass=True)
    b = hyq.PagedBatch(torch.zeros(3, dtype=i32), torch.zeros(2, dtype=i32), torch.zeros((2, 4), dtype=i32), 1, 1)
    q = torch.zeros((2, 8, 128), dtype=bf)
    with pytest.raises(ValueError):   # not on a GPU
        hyq.hyq_paged_attn(c, b, q, q.float())
    with pytest.raises(ValueError):
        hyq.hyq_paged_attn(c, b, q[:, :4], q[:, :4].float())
