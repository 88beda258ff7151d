"""hyq_evict above 32768 slots, where keys are read again group by group, with
more slots of the threshold's mass than are wanted: the lowest of them are kept,
and the count of those kept is carried from one group of 32768 to the next."""
import numpy as np
import pytest

import test_gpu_evict as te

GROUP = 32768

CASES = [
    # as in test_gpu_evict; the group in which the last kept slot of the threshold's mass lies
    (([70000], 1, 64, "fp8", 40000, 0, 0, "zero"), 1),
    (([70000], 1, 256, "int8", 69000, 500, 0, "zero"), 2),
    (([40000, 70001], 1, 16, "bf16", 33000, 128, 7, "zero"), 1),
    (([100000], 1, 128, "int8", 30000, 0, 0, "few values"), 1),
    (([100000], 1, 32, "fp8", 38000, 100, 0, "few values"), 2),
    (([66000], 2, 64, "int8", 20000, 64, 50000, "few values"), 1),
    (([70000], 1, 64, "fp8", 67500, 10, 0, "odd"), 1),        # among the NaNs
    (([70000], 1, 64, "int8", 69800, 0, 0, "odd"), 2),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", [c for c, _ in CASES], ids=str)
def test_against_oracle(case):
    te.test_against_oracle(case)


@pytest.mark.parametrize("case,group", CASES, ids=str)
def test_cases_have_ties_across_groups(case, group):
    """With masses of the same kind and number: the threshold is shared by more
    slots than are wanted, and the wanted ones end in the group given."""
    lens, Hkv, page, fmt, budget, recent, _, kind = case
    n = max(lens)
    m = te.masses(np.random.default_rng(sum(lens) + budget), kind, (-(-n // page), 1, page)).reshape(-1)[:n - recent]
    m = np.where(m == -np.inf, np.float32(-3e38), m)
    m = np.where(np.isnan(m), -np.inf, m)   # NaN is below every number
    t = np.sort(m)[::-1][budget - recent - 1]
    equal = np.flatnonzero(m == t)
    wanted = budget - recent - int((m > t).sum())
    assert wanted < equal.size
    assert equal[wanted - 1] // GROUP == group
    assert equal[0] < GROUP
