"""hyq_evict with the largest budget an int32 holds (it keeps everything): the
list's entries behind the kept slots are padding up to the last one, and nothing
before it or behind it is written."""
import numpy as np
import pytest

import paged_common as pc
import paper_2608_27875_amd as hyq

pytestmark = pytest.mark.gpu
BUDGET = (1 << 31) - 1


def test_largest_budget():
    import torch
    page, n, guard = 256, 300, 1 << 16
    bufs, _ = pc.pool(np.random.default_rng(1), "int8", 6, 1, page)
    cache = pc.cache_of(bufs, "int8", 1, np.random.default_rng(2).random((6, 1, page)).astype(np.float32))
    new_table = torch.full((1, -(-BUDGET // page)), -1, dtype=torch.int32, device="cuda")
    new_table[0, :2] = torch.tensor([4, 5], dtype=torch.int32)
    whole = torch.full((BUDGET + 2 * guard,), -9, dtype=torch.int32, device="cuda")
    keep = whole[guard:guard + BUDGET].view(1, 1, BUDGET)
    new_lens = torch.empty((1,), dtype=torch.int32, device="cuda")
    table = pc.dev(np.array([[2, 0]], np.int32))
    hyq.hyq_evict(cache, pc.dev(np.array([n], np.int32)), table, new_table, keep, new_lens, max_len=n,
                  budget=BUDGET, recent=7)
    torch.cuda.synchronize()
    assert new_lens.item() == n
    assert torch.equal(keep[0, 0, :n].cpu(), torch.arange(n, dtype=torch.int32))
    for at in range(n, BUDGET, 1 << 28):
        part = keep[0, 0, at:min(at + (1 << 28), BUDGET)]
        assert int(part.min()) == int(part.max()) == hyq.KQ_POS_PAD
    assert bool((whole[:guard] == -9).all()) and bool((whole[guard + BUDGET:] == -9).all())
    k = cache.bufs["k"].cpu().numpy()
    assert np.array_equal(k[4, 0], bufs["k"][2, 0]) and np.array_equal(k[5, 0, :n - page], bufs["k"][0, 0, :n - page])
    assert np.array_equal(k[5, 0, n - page:], bufs["k"][5, 0, n - page:])
    del whole, keep
    torch.cuda.empty_cache()
