"""Softmax scales of hyq_paged_attn: the kernels take log2(e) times them."""
import pytest

import test_paged_abi as pa
from test_paged_abi import EINVAL, lib   # noqa: F401 (lib is a fixture)


@pytest.mark.parametrize("scale,refused", [(3.4e38, True), (2.4e38, True), (2.3e38, False), (1e-45, False)])
def test_scales_stay_finite(lib, scale, refused):   # noqa: F811
    """Read off which refusal comes: that of the scale, or the later one of q."""
    import paper_2608_27875_amd as hyq
    assert pa.attn(lib, scale=scale, q=None) == EINVAL
    assert ("softmax_scale" in hyq.hyq_last_error()) == refused
