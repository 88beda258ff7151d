"""The workspace that hyq_paged_ws_bytes gives without a number of token rows:
enough for every step the batch's bounds allow, never refused for rows that no
step could have."""
import pytest

import paper_2608_27875_amd as hyq
from test_paged_abi import lib   # noqa: F401 (a fixture)


def handles(B, Hq, Hkv, max_new, max_len):
    import torch
    i32 = torch.int32
    cache = hyq.PagedCache(Hq, Hkv, 16, 4, "cpu", mass=True)
    batch = hyq.PagedBatch(torch.zeros(B + 1, dtype=i32), torch.zeros(B, dtype=i32),
                           torch.zeros((B, 1 << 12), dtype=i32), max_new=max_new, max_len=max_len)
    return cache, batch


@pytest.mark.parametrize("mass", [False, True])
@pytest.mark.parametrize("B,Hq,Hkv,max_new,max_len", [
    (256, 32, 8, 2048, 32768),       # one prompt chunk beside single tokens
    (64, 32, 8, 8192, 4096),
    (1024, 40, 8, 1 << 15, 1000),
    (4096, 1, 1, 1 << 20, 1000),     # B * max_new beyond 32 bits
])
def test_batches_of_many_sequences(lib, B, Hq, Hkv, max_new, max_len, mass):   # noqa: F811
    cache, batch = handles(B, Hq, Hkv, max_new, max_len)
    n = hyq.hyq_paged_ws_bytes(cache, batch, mass)
    most = hyq.PAGED_MAX_ROWS // (Hq + 2 * Hkv)
    for T in (1, B, B + max_new, 4096, most):
        if T <= most:
            assert hyq.hyq_paged_ws_bytes(cache, batch, mass, T) <= n
    with pytest.raises(hyq.HyqError) as e:   # there is no such step
        hyq.hyq_paged_ws_bytes(cache, batch, mass, most + 1)
    assert e.value.code == hyq.HYQ_EUNSUPPORTED


def test_small_batches_need_what_they_have(lib):   # noqa: F811
    cache, batch = handles(3, 8, 2, 7, 500)
    assert hyq.hyq_paged_ws_bytes(cache, batch) == hyq.hyq_paged_ws_bytes(cache, batch, False, 21)


def test_limit_is_the_header_s():
    import os
    text = open(os.path.join(os.path.dirname(os.path.dirname(hyq.__file__)), "include", "hyq.h")).read()
    assert "#define HYQ_PAGED_MAX_ROWS (1 << 24)" in text and hyq.PAGED_MAX_ROWS == 1 << 24
