"""Sizes that the cross attention takes or refuses (CPU: workspace sizes alone)."""
import ctypes

import pytest

from paper_2506_20686_amd import binding as B
from test_more_abi import lib  # noqa: F401

OK, UNS = B.OK, B.ERR_UNSUPPORTED
EACH = (512, 768, 768)  # samples with a map each: 2^24 pieces of 16 keys and more


# (dtype, batch, queries, keys, heads, key heads, channels, bias maps)
@pytest.mark.parametrize("size,code", [
    ((B.BF16, *EACH, 8, 8, 32, 512), OK), ((B.F32, *EACH, 8, 8, 64, 512), OK),
    ((B.BF16, *EACH, 4, 4, 128, 512), OK),
    # no planes either of one map
    ((B.BF16, 2, 1 << 21, 65, 4, 4, 8, 1), OK), ((B.BF16, 2, 1 << 21, 65, 4, 4, 8, 2), OK),
    # planes: shared key heads, heads not in fours, wide fp32 rows
    ((B.BF16, *EACH, 8, 4, 32, 512), UNS), ((B.BF16, *EACH, 6, 6, 32, 512), UNS),
    ((B.F32, *EACH, 8, 8, 72, 512), UNS), ((B.BF16, 2, 1 << 21, 65, 6, 6, 8, 1), UNS),
    ((B.BF16, 300, 768, 768, 6, 6, 32, 300), OK),
])
def test_maps_of_many_samples(lib, size, code):  # noqa: F811
    r = ctypes.c_size_t(0)
    for name in ("fwd", "bwd"):
        f = getattr(lib, f"tri_cross_attn_{name}_workspace_bytes")
        assert f(*size, ctypes.byref(r)) == code
