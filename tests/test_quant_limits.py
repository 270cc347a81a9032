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


def test_nothing_to_do_needs_no_addresses():
    """Tensors without elements have none."""
    lib, d = pk.load_library(), C.byref(pk.make_desc(0, 8, 4, 64, 8, 100, dtype=1))
    n = None
    assert lib.pikv_norm_rope(n, 0, 12 * 64, 4, 4, 64, 1, FAKE, FAKE, 1e-6, n, FAKE, 64, 0, n, n, n, n) == 0
    assert lib.pikv_quant_pack(d, 0, 16, n, n, 6400, 64, n, n, n, n, n, n) == 0
    assert lib.pikv_quant_read(d, 0, 16, n, n, n, n, n, n, n, 6400, 64, n) == 0
    assert lib.pikv_quant_append(d, 0, 16, n, n, n, 2, n, n, 1, n, n, n, n, n, n, n) == 0
    assert lib.pikv_quant_attn(d, 0, 16, n, n, n, n, n, n, n, n, 2, 0, 0.0, n, n, n, n, n, n, 0, n) == 0


@pytest.mark.parametrize("tokens,kw", [(0, dict(D=96)), (0, dict(eps=-1.0)), (0, dict(rotary=8)), (0, dict(stride=64)), (0, dict(dtype=2)), (-1, {})])
def test_what_can_be_checked_without_addresses_is(tokens, kw):
    a = dict(dict(D=64, eps=1e-6, rotary=64, stride=12 * 64, dtype=1), **kw)
    assert pk.load_library().pikv_norm_rope(None, tokens, a["stride"], 4, 4, a["D"], a["dtype"], None, None, a["eps"], None, None, a["rotary"], 0, None, None,
                                            None, None) in (-1, -2)
    d = C.byref(pk.make_desc(0, 8, 4, 64, 8, 100, dtype=1))
    assert pk.load_library().pikv_quant_append(d, 0, 16, *[None] * 3, 9, None, None, 0, *[None] * 7) == -1


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("k", [1, 2, 3, 8])
def test_a_wave_of_the_short_form_has_two_stages_at_most(D, k):
    """One launch leaves one partial per row and shard to hold, a split pass one for each split."""
    def partials(S):
        return pk.pikv_quant_attn_workspace_bytes(pk.make_desc(1, 8, 8, D, 16, S, dtype=1), k) // (8 * k * (D + 2) * 4)
    stage = 32 * (8 // k)                                   # entries of a stage of a shard's waves
    most = stage * (1 if D == 128 else 2)
    assert partials(most) == 1
    assert partials(max(most, 128) + 1) > 1                 # (shards of up to 128 entries are not split)
