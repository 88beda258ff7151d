"""Which sizes hyq_norm_rope takes: read off the refusal that comes after the
one of sizes (an output on top of an input), so nothing is enqueued."""
import pytest

import paper_2608_27875_amd as hyq
from test_paged_abi import EINVAL, EUNSUP, FAKE, lib, norm_rope   # noqa: F401 (lib is a fixture)


@pytest.mark.parametrize("kw", [dict(B=4, Hq=40, Hkv=8, L=131072), dict(B=16, Hq=32, Hkv=8, L=1048575),
                                dict(B=1, Hq=8, Hkv=8, L=8388608)])
def test_large_calls_are_taken(lib, kw):   # noqa: F811
    assert norm_rope(lib, s=hyq.Shape(**kw), qs=kw["Hq"] * 128, ks=kw["Hkv"] * 128, vs=kw["Hkv"] * 128,
                     Q=FAKE) == EINVAL
    assert "overlap" in hyq.hyq_last_error()


@pytest.mark.parametrize("kw", [dict(B=16, Hq=8, Hkv=8, L=1048576), dict(B=1 << 30, Hq=8, Hkv=8, L=1 << 23),
                                dict(B=8, Hq=512, Hkv=64, L=1048576)])
def test_too_large_ones_are_refused(lib, kw):   # noqa: F811
    assert norm_rope(lib, s=hyq.Shape(**kw), qs=kw["Hq"] * 128, ks=kw["Hkv"] * 128, vs=kw["Hkv"] * 128) == EUNSUP
