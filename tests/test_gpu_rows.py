"""A row's bits are its own: neither the rows that share its wave nor keys that only those see have a part in them."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

import paged_reference as ref  # noqa: E402
from test_gpu_paged import Attention  # noqa: E402
from test_gpu_prompt import Device, host  # noqa: E402


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("slopes", [False, True], ids=["", "slopes"])
@pytest.mark.parametrize("lens,Hq,D", [([150], 4, 64), ([700], 4, 128), ([400] * 20, 16, 128), ([150] + [2] * 600, 4, 64)],
                         ids=["split", "eight", "whole", "ragged"])
def test_rows_of_a_prompt(lens, Hq, D, slopes, dtype):
    make = lambda: ref.Prompts(lens, Hq, Hq // 2, D, dtype, seed=3, std=4.0, slopes=slopes, window=60)
    want = Device(make())
    want.attend()
    token = np.arange(want.p.tokens)
    # queries that take every maximum with them, one in a wave
    p = make()
    p.q[::40] = ref.stored(p.q[::40] * 50.0, dtype)
    d = Device(p)
    d.attend()
    same = token % 40 != 0
    for a, b in ((d.out, want.out), (d.row_max, want.row_max), (d.row_norm, want.row_norm)):
        np.testing.assert_array_equal(host(a)[same], host(b)[same])
    # a key
    for large in (50.0, 1e30):
        p = make()
        p.k[70] = ref.stored(p.k[70] * large, dtype)
        d = Device(p)
        d.attend()
        same = (token < 70) | (token >= 130)
        for a, b in ((d.out, want.out), (d.row_max, want.row_max), (d.row_norm, want.row_norm)):
            np.testing.assert_array_equal(host(a)[same], host(b)[same])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G,D,S", [(4, 64, 100), (16, 128, 700), (33, 32, 300), (4, 64, 6000)])
def test_rows_of_a_step(G, D, S, dtype):
    make = lambda: Attention(2, 3, 2, G, S, D, dtype, 16, 2, seed=4, std=4.0, window=S)
    a = make()
    a.run()
    want = [host(x) for x in (a.y, a.row_max, a.row_norm)]
    b = make()
    b.q[:, ::G] = ref.stored(b.q[:, ::G] * 50.0, dtype)
    b.run()
    same = np.arange(a.Hq) % G != 0
    for got, w in zip((b.y, b.row_max, b.row_norm), want):
        np.testing.assert_array_equal(host(got)[:, same], w[:, same])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G,D,S", [(4, 64, 100), (16, 128, 700), (33, 32, 300), (4, 64, 6000)])
def test_a_query_that_is_no_number(G, D, S, dtype):
    """NaN in its own row of y, nothing of it in row_norm and slot_coef, and no other row any different - in one launch and in two."""
    make = lambda: Attention(2, 3, 2, G, S, D, dtype, 16, 2, seed=4, full=True)
    a, b = make(), make()
    a.run()
    b.q[1, G - 1, 3] = np.nan
    b.run()
    other = np.ones(a.y.shape[:2], bool)
    other[1, G - 1] = False
    for got, w in zip((b.y, b.row_max, b.row_norm, b.coef), (a.y, a.row_max, a.row_norm, a.coef)):
        np.testing.assert_array_equal(host(got)[other], host(w)[other])
    assert np.isnan(host(b.y)[~other]).all() and (host(b.row_norm)[~other] == 0).all() and (host(b.coef)[~other][..., 1] == 0).all()
