"""Sizes that packed attention refuses before any launch, without a GPU."""
import ctypes

import pytest

P = ctypes.c_void_p(4096)        # never dereferenced


@pytest.fixture(scope="module")
def hsa():
    from paper_2605_06892_gb300 import build as b
    b.build()
    import paper_2605_06892_gb300 as m
    m.lib()
    return m


@pytest.mark.parametrize("batch,Hkv", [((1 << 23) + 1, 1), ((1 << 22) + 1, 2), (1 << 20, 16), (2 ** 31 - 1, 1)])
def test_more_sequences_than_the_waits_allow_for(hsa, batch, Hkv):
    """A block that passes over that many sequences could outlast the other warps' waits."""
    c0 = hsa.hsa_launch_count()
    assert hsa.lib().hsa_packed_attention(P, Hkv * 64, P, Hkv * 64, P, Hkv * 64, P, P, batch, 10, 10, Hkv, Hkv, 64,
                                          1, 0.0, P, 0, None, 0, None) == -4
    assert hsa.hsa_launch_count() == c0
