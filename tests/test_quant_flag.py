"""An 8-bit cache is told apart from dense shards: by PIKV_DESC_8BIT in its descriptor, and by the mark of its shard tables.  Everything
here is found on the host: the addresses are made up and never dereferenced."""
import ctypes as C

import pytest
import torch

import paper_2508_06526_amd as pk
from paper_2508_06526_amd import binding

INVALID = -1
FAKE = C.c_void_p(0x1000)


def desc(B=2, flags=2, **kw):
    return pk.make_desc(**dict(dict(B=B, Hq=8, Hkv=4, D=128, E=8, S=100, dtype=1, flags=flags), **kw))


def dense_calls(lib, d):
    """The calls that work on rows of the dense type; B == 0: nothing to do for any that takes the descriptor."""
    d, f, big = C.byref(d), FAKE, 1 << 30
    return dict(
        attn=lambda: lib.pikv_sharded_attn(d, f, f, f, None, None, f, f, None, 2, 0, 0.0, f, None, None, None, None, f, big, None),
        append=lambda: lib.pikv_append(d, f, f, f, 2, None, None, 0, f, f, f, f, None),
        compacting=lambda: lib.pikv_evict(d, f, f, 50, None, 0, f, f, 4, 1, f, f, None),
        step=lambda: lib.pikv_decode_step(d, f, f, None, f, f, f, f, None, None, f, f, 2, 0, 0.0, 1.0, f, f, f, f, f, f, f, f, f, f, big, None),
        policy_step=lambda: lib.pikv_decode_step_policy(d, f, f, None, f, f, f, f, None, None, f, f, 2, 0, 0.0, 1.0, f, f, f, f, f, f, f, f, f, f, big,
                                                        None, None, None))


def quant_calls(lib, d):
    d, f = C.byref(d), FAKE
    return dict(
        pack=lambda: lib.pikv_quant_pack(d, 0, 16, f, f, 12800, 128, f, f, f, f, f, None),
        read=lambda: lib.pikv_quant_read(d, 0, 16, f, f, f, f, f, f, f, 12800, 128, None),
        append=lambda: lib.pikv_quant_append(d, 0, 16, f, f, f, 2, None, None, 0, f, f, f, f, f, f, None),
        attn=lambda: lib.pikv_quant_attn(d, 0, 16, f, f, f, f, f, f, f, None, 2, 0, 0.0, f, None, None, None, None, f, 1 << 30, None),
        evict=lambda: lib.pikv_evict(d, f, f, 50, None, 0, f, f, 4, 0, None, None, None),
        utility=lambda: lib.pikv_update_utility(d, f, f, f, f, 2, 1.0, f, None),
        tracked=lambda: lib.pikv_update_utility_tracked(d, f, f, f, f, 2, 1.0, f, 0.1, 3, f, f, None),
        stamp=lambda: lib.pikv_policy_stamp(d, f, 2, None, None, 0, f, 3, f, f, f, None),
        policy=lambda: lib.pikv_policy_utility(d, pk.POLICY_H2O, f, 3, 0.0, 0, 0, f, f, f, f, f, None),
        stamps=lambda: lib.pikv_policy_compact(d, f, f, 4, f, f, f, f, None))


@pytest.fixture(scope="module")
def lib():
    return pk.load_library()


def test_calls_on_dense_rows_refuse_the_descriptor_of_an_8_bit_cache(lib):
    assert pk.DESC_8BIT == 2
    for B in (0, 2):
        for name, call in dense_calls(lib, desc(B)).items():
            assert call() == INVALID, name
    for name, call in dense_calls(lib, desc(0, flags=0)).items():
        assert call() == 0, name
    assert pk.pikv_attn_workspace_bytes(desc(), 2) == 0 and pk.pikv_attn_workspace_bytes(desc(flags=0), 2) > 0


@pytest.mark.parametrize("flags", [0, 2])
def test_calls_that_serve_an_8_bit_cache_take_it_with_the_flag_and_without(lib, flags):
    for name, call in quant_calls(lib, desc(0, flags)).items():
        assert call() == 0, name
    assert pk.pikv_quant_attn_workspace_bytes(desc(flags=flags), 2) > 0


def test_the_flag_stands_for_rows_of_bytes(lib):
    for bad in (desc(0, rank=32), desc(0, flags=3), desc(0, flags=6), desc(0, stride_s=120), desc(0, stride_s=136)):
        for name, call in quant_calls(lib, bad).items():
            assert call() == INVALID, name
    assert quant_calls(lib, desc(0, stride_s=144))["pack"]() == 0


@pytest.mark.parametrize("dtype", [torch.int8, torch.float8_e4m3fn])
def test_tables_of_8_bit_shards_are_refused_by_the_calls_on_dense_rows(dtype):
    shards = torch.zeros((1, 2, 1, 4, 64), dtype=torch.int8).view(dtype)
    d, f = pk.make_desc(1, 1, 1, 64, 2, 4, dtype=1), torch.zeros(64)
    for tab in (pk.shard_table(shards), pk.shard_table([shards[0, 0], shards[0, 1]])):
        for name, call in dict(
                pikv_sharded_attn=lambda: pk.pikv_sharded_attn(d, f, tab, tab, None, None, f, f, None, 1, 0, 0.0, f, None, None, None, None, f),
                pikv_sharded_attn_noalloc=lambda: pk.pikv_sharded_attn_noalloc(d, f, tab, tab, None, None, f, f, None, 1, 0, 0.0, f, None, None, None, None),
                pikv_append=lambda: pk.pikv_append(d, f, f, f, 1, None, None, 0, tab, tab, f, f),
                pikv_evict=lambda: pk.pikv_evict(d, f, f, 1, None, 0, f, f, 1, True, tab, tab),
                pikv_decode_step=lambda: pk.pikv_decode_step(d, *[f] * 5, tab, tab, None, None, f, f, 1, 0, 0.0, 1.0, *[f] * 10),
                pikv_decode_step_policy=lambda: pk.pikv_decode_step_policy(d, *[f] * 5, tab, tab, None, None, f, f, 1, 0, 0.0, 1.0, *[f] * 10, None),
                pikv_quant_pack=lambda: pk.pikv_quant_pack(d, 0, 16, tab, tab, 256, 64, f, tab, tab, f, f),
                pikv_quant_read=lambda: pk.pikv_quant_read(d, 0, 16, tab, tab, f, f, f, tab, tab, 256, 64)).items():
            with pytest.raises(TypeError, match="%s.*8-bit" % name):
                call()


def test_tables_of_other_shards_carry_no_mark():
    for dtype in (torch.bfloat16, torch.float32, torch.uint8):
        assert not hasattr(pk.shard_table(torch.zeros((1, 2, 1, 4, 64), dtype=dtype)), binding._MARK)
