"""CPU tests of the 8-bit cache's largest sizes: what would pass 32-bit positions in the kernels is refused."""

import ctypes as C

import pytest

from paper_2608_20397_amd import nexus as N
from test_kv8_abi import _cache, _pt, suffix

NPP = (1 << 27) - 1                                # the most pages a cache may have
END = 16 * NPP


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n_s", [1, 40])
def test_suffixes_near_the_last_position(D, n_s):
    """A split may end up to 32767 slots past a sequence's last key, a key tile 63 and a query block 31: their
    positions have to stay below 2^31 too."""
    c = _cache(n_phys_pages=NPP, n_kv_heads=1, head_dim=D)
    need = lambda past: N.lib().nexus_kv8_suffix_attn_workspace(n_s, 2, C.byref(c), past)
    last = (1 << 31) - 65536 - n_s
    for past in (END - n_s, last + 1):
        assert need(past) == (1 << 64) - 1
        assert suffix(c=c, pt=_pt(NPP), lens=(n_s,), pasts=(past,), hq=2) == N.ERANGE
        assert suffix(c=c, pt=_pt(NPP), starts=(0, n_s), lens=(n_s, n_s), pasts=(5, past), hq=2) == N.ERANGE
    assert 0 < need(last) < (1 << 64) - 1
    assert suffix(c=c, pt=_pt(NPP), lens=(n_s,), pasts=(last,), hq=2) == N.EWORKSPACE
