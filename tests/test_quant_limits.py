"""Limits of the calls around the 8-bit cache, found on the host: made-up addresses that are never dereferenced."""
import ctypes as C

import pytest

import paper_2508_06526_amd as pk

UNSUPPORTED = -2
FAKE = C.c_void_p(0x1000)


@pytest.mark.parametrize("B,k,S,held", [(65535, 1, 128, True), (65536, 1, 128, False),           # 256 query rows, a block of 256 threads each
                                        (16384, 32, 128, True), (16384, 33, 128, False), (16383, 33, 128, True),     # ... of 1024
                                        (16384, 1, 32 << 10, True), (16384, 1, 33 << 10, False)])
def test_the_merge_stays_within_a_launch(B, k, S, held):
    d = pk.make_desc(B, 256, 1, 32, 64, S, dtype=1)
    size = pk.pikv_quant_attn_workspace_bytes(d, k)
    assert (size > 0) == held
    if not held:
        assert pk.load_library().pikv_quant_attn(C.byref(d), 0, 16, *[FAKE] * 7, None, k, 0, 0.0, FAKE, None, None, None, None, FAKE, 1 << 50,
                                                 None) == UNSUPPORTED
