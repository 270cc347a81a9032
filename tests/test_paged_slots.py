"""Calls that go by slots and counts take the descriptor of a paged cache with as many query rows as its own calls do."""
import ctypes as C

import pytest

import paper_2508_06526_amd as pk
from test_paged_abi import FAKE, INVALID, UNSUPPORTED, desc


@pytest.fixture(scope="module")
def lib():
    return pk.load_library()


def evict(lib, d, compact=0):
    return lib.pikv_evict(C.byref(d), FAKE, FAKE, 10, None, 0, FAKE, FAKE, 4, compact, FAKE, FAKE, None)


CALLS = {
    "evict": evict,
    "compact": lambda lib, d: lib.pikv_policy_compact(C.byref(d), FAKE, FAKE, 4, FAKE, FAKE, FAKE, FAKE, None),
    "stamp": lambda lib, d: lib.pikv_policy_stamp(C.byref(d), FAKE, 2, FAKE, FAKE, 1, FAKE, 5, FAKE, FAKE, FAKE, None),
    "policy": lambda lib, d: lib.pikv_policy_utility(C.byref(d), pk.POLICY_H2O, FAKE, 5, 0.0, 0, 0, FAKE, FAKE, FAKE, FAKE, FAKE, None),
    "utility": lambda lib, d: lib.pikv_update_utility(C.byref(d), FAKE, FAKE, FAKE, FAKE, 2, 1.0, FAKE, None),
    "tracked": lambda lib, d: lib.pikv_update_utility_tracked(C.byref(d), FAKE, FAKE, FAKE, FAKE, 2, 1.0, None, 0.1, 5, FAKE, FAKE, None)}


@pytest.mark.parametrize("name", CALLS)
def test_query_rows_of_drafts(lib, name):
    limited = name in ("utility", "tracked")             # a thread a query row
    for kw in (dict(Hq=320, Hkv=8, tq=5), dict(Hq=1024, Hkv=8), dict(Hq=1024, Hkv=256)):
        assert CALLS[name](lib, desc(B=0, **kw)) == (UNSUPPORTED if limited else 0)
    assert CALLS[name](lib, desc(B=0, Hq=256)) == 0
    assert CALLS[name](lib, desc(B=0, Hq=320, stride_s=60)) == (UNSUPPORTED if limited else INVALID)
    assert CALLS[name](lib, desc(B=0, Hq=1028)) == UNSUPPORTED and CALLS[name](lib, desc(Hq=322)) == INVALID


def test_an_eviction_that_moves_rows_is_of_whole_shards(lib):
    assert evict(lib, desc(B=0, Hq=320), 1) == UNSUPPORTED and evict(lib, desc(B=0, Hq=320, route_rows_per_seq=320)) == 0
    assert evict(lib, desc(B=0), 1) == 0
