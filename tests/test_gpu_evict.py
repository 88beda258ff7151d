"""hyq_evict on the GPU against the oracle: slots, rows, scales and masses are
moved, not computed, so everything is compared bit for bit."""
import numpy as np
import pytest

import paged_common as pc
import paper_2608_27875_amd as hyq
from oracle import paged_oracle as po

pytestmark = pytest.mark.gpu
D = 128

CASES = [
    # lens, Hkv, page, fmt, budget, recent, max_len beyond, kind of masses
    ([0], 1, 16, "bf16", 1, 0, 0, "normal"),
    ([1], 1, 16, "bf16", 1, 1, 0, "normal"),
    ([17, 3, 16], 2, 16, "bf16", 5, 2, 0, "normal"),
    ([200, 64, 65], 3, 64, "fp8", 64, 10, 0, "few values"),
    ([300], 2, 32, "int8", 100, 100, 5000, "normal"),       # only the recent ones
    ([1000, 999], 1, 128, "bf16", 333, 0, 0, "zero"),       # all equal: the lowest slots
    ([4096, 4097, 5000], 1, 256, "bf16", 1025, 7, 0, "wide"),
    ([9000, 200], 2, 64, "fp8", 500, 64, 0, "few values"),
    ([20000], 1, 16, "bf16", 4000, 128, 0, "odd"),
    ([40000, 33000], 1, 64, "int8", 2000, 100, 0, "wide"),  # keys read again for every pass
    ([5000], 1, 64, "bf16", 4999, 1, 40000, "few values"),
    ([400, 800], 2, 16, "bf16", 75, 0, 0, "classes"),       # three whole classes; one and a half
    ([33600, 400], 1, 16, "fp8", 4200, 0, 0, "classes"),    # two whole ones, keys read again
]


def masses(rng, kind, shape):
    if kind == "zero":
        return np.where(rng.random(shape) < 0.5, 0.0, -0.0).astype(np.float32)
    if kind == "few values":
        return rng.integers(0, 5, shape).astype(np.float32) / 4
    if kind == "classes":   # every 16 slots hold each of 16 powers of two once
        return np.broadcast_to(2.0 ** (np.arange(shape[-1]) % 16 - 8), shape).astype(np.float32)
    if kind == "odd":
        x = rng.standard_normal(shape).astype(np.float32)
        r = rng.random(shape)
        x[r < 0.1] = np.nan
        x[(r > 0.1) & (r < 0.2)] = np.inf
        x[(r > 0.2) & (r < 0.3)] = -np.inf
        return x
    if kind == "wide":
        return np.exp(20 * rng.standard_normal(shape)).astype(np.float32)
    return rng.random(shape).astype(np.float32)


@pytest.mark.parametrize("case", CASES, ids=str)
def test_against_oracle(case):
    import torch
    lens, Hkv, page, fmt, budget, recent, more, kind = case
    rng = np.random.default_rng(sum(lens) + budget)
    B, new_pages = len(lens), -(-budget // page)
    table, n_pages = pc.tables(rng, lens, page, extra_pages=B * new_pages + 1)
    used = set(table[(table >= 0) & (table < n_pages)].tolist())
    owned = set()
    for b, n in enumerate(lens):
        owned |= set(table[b, :-(-n // page)].tolist())
    free = [p for p in range(n_pages) if p not in owned]
    new_table = rng.permutation(free)[:B * new_pages].reshape(B, new_pages).astype(np.int32)
    small = n_pages * Hkv * page * D < 3e6
    if small:
        bufs, _ = pc.pool(rng, fmt, n_pages, Hkv, page)
    else:
        bufs = {n: rng.integers(0, 256, (n_pages, Hkv, page, D), dtype=np.uint8) if fmt != "bf16"
                else rng.integers(0, 1 << 15, (n_pages, Hkv, page, D), dtype=np.uint16) for n in "kv"}
        if fmt != "bf16":
            for n in "kv":
                bufs[n + "_scale"] = rng.random((n_pages, Hkv, page)).astype(np.float32)
    mass = masses(rng, kind, (n_pages, Hkv, page))
    cache = pc.cache_of(bufs, fmt, Hkv, mass)
    keep = torch.full((B, Hkv, budget), -9, dtype=torch.int32, device="cuda")
    new_lens = torch.full((B,), -9, dtype=torch.int32, device="cuda")
    hyq.hyq_evict(cache, pc.dev(np.array(lens, np.int32)), pc.dev(table), pc.dev(new_table), keep,
                  new_lens, max_len=max(lens) + more, budget=budget, recent=recent)
    torch.cuda.synchronize()
    want_keep, want_lens = po.evict(mass, lens, table, budget, recent)
    np.testing.assert_array_equal(new_lens.cpu().numpy(), want_lens)
    np.testing.assert_array_equal(keep.cpu().numpy(), want_keep)
    bufs["mass"] = mass
    for name, was in bufs.items():
        want = was.copy()
        for b in range(B):
            for j in range(Hkv):
                m = int(want_lens[b])
                src = want_keep[b, j, :m]
                dst = np.arange(m)
                want[new_table[b, dst // page], j, dst % page] = was[table[b, src // page], j, src % page]
        got = cache.bufs[name]
        got = got.view(torch.int16 if got.dtype == torch.bfloat16 else got.dtype).cpu().numpy()
        kind_ = {1: np.uint8, 2: np.uint16, 4: np.uint32}[got.dtype.itemsize]
        np.testing.assert_array_equal(np.ascontiguousarray(got).view(kind_),
                                      np.ascontiguousarray(want).view(kind_), err_msg=name)


def test_missing_pages():
    """A slot of a missing page counts as less than any mass; kept anyway (a
    recent one), it becomes a row of zeros.  A missing new page takes no rows."""
    import torch
    rng = np.random.default_rng(1)
    bufs, _ = pc.pool(rng, "bf16", 8, 1, 16)
    mass = rng.random((8, 1, 16)).astype(np.float32)
    table = np.array([[0, 99, 2, -1]], dtype=np.int32)
    new_table = np.array([[5, -1, 6]], dtype=np.int32)
    cache = pc.cache_of(bufs, "bf16", 1, mass)
    keep = torch.empty((1, 1, 40), dtype=torch.int32, device="cuda")
    new_lens = torch.empty((1,), dtype=torch.int32, device="cuda")
    hyq.hyq_evict(cache, pc.dev(np.array([60], np.int32)), pc.dev(table), pc.dev(new_table), keep,
                  new_lens, max_len=60, budget=40, recent=4)
    want, lens = po.evict(mass, [60], table, 40, 4)
    np.testing.assert_array_equal(keep.cpu().numpy(), want)
    k = pc.host(cache.bufs["k"])
    was = po.bf16(bufs["k"])
    for i, s in enumerate(want[0, 0]):
        at = po.place(table, 0, int(s), 16, 8)
        to = po.place(new_table, 0, i, 16, 8)
        if to is not None:
            row = was[at[0], 0, at[1]] if at else np.zeros(D)
            np.testing.assert_array_equal(k[to[0], 0, to[1]], row)
    assert np.array_equal(k[6, 0, 8:], was[6, 0, 8:])
    assert np.array_equal(k[[1, 3, 4, 7]], was[[1, 3, 4, 7]])


def test_shared_old_pages():
    """Two sequences with the same prompt pages, evicted in one call: the old
    pages are only read."""
    import torch
    rng = np.random.default_rng(2)
    bufs, _ = pc.pool(rng, "int8", 12, 2, 16)
    mass = rng.random((12, 2, 16)).astype(np.float32)
    table = np.array([[0, 1, 2], [0, 1, 3]], dtype=np.int32)
    new_table = np.array([[5, 6], [7, 8]], dtype=np.int32)
    cache = pc.cache_of(bufs, "int8", 2, mass)
    keep = torch.empty((2, 2, 20), dtype=torch.int32, device="cuda")
    new_lens = torch.empty((2,), dtype=torch.int32, device="cuda")
    hyq.hyq_evict(cache, pc.dev(np.array([48, 40], np.int32)), pc.dev(table), pc.dev(new_table), keep,
                  new_lens, max_len=48, budget=20, recent=3)
    want, _ = po.evict(mass, [48, 40], table, 20, 3)
    np.testing.assert_array_equal(keep.cpu().numpy(), want)
    k = cache.bufs["k"].cpu().numpy()
    for b in range(2):
        for j in range(2):
            for i, s in enumerate(want[b, j]):
                assert np.array_equal(k[new_table[b, i // 16], j, i % 16], bufs["k"][table[b, s // 16], j, s % 16])
    assert np.array_equal(k[:5], bufs["k"][:5]) and np.array_equal(k[9:], bufs["k"][9:])


def test_lengths_beyond_their_bound():
    """Device lengths outside [0, max_len] count as the nearest bound."""
    import torch
    rng = np.random.default_rng(3)
    bufs, _ = pc.pool(rng, "bf16", 16, 1, 16)
    mass = rng.random((16, 1, 16)).astype(np.float32)
    table = np.arange(8, dtype=np.int32).reshape(2, 4)
    new_table = np.array([[9], [10]], dtype=np.int32)
    cache = pc.cache_of(bufs, "bf16", 1, mass)
    keep = torch.empty((2, 1, 10), dtype=torch.int32, device="cuda")
    new_lens = torch.empty((2,), dtype=torch.int32, device="cuda")
    hyq.hyq_evict(cache, pc.dev(np.array([-5, 1 << 30], np.int32)), pc.dev(table), pc.dev(new_table), keep,
                  new_lens, max_len=50, budget=10, recent=2)
    want, lens = po.evict(mass, [0, 50], table, 10, 2)
    np.testing.assert_array_equal(keep.cpu().numpy(), want)
    np.testing.assert_array_equal(new_lens.cpu().numpy(), lens)
