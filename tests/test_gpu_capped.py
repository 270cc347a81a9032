"""Capped scores, each in the form that its own size asks for: what a row does not see, and the rows beside it, have no part in its bits.

Errors, beside those of tests/paged_reference.py.  x = s / cap comes from the product by a factor that is rounded twice (scale / cap) and a rounding of
its own: 3 * 2^-24 of it, which the tanh passes on at most whole.  Its small form is off by 1.04 * 2^-24 of the value, its large form by
3.6 * 2^-24, at most 7.8 * 2^-24 of a value of 0.46 and more; times the cap: 2^-24.  In all at most 12 * 2^-24 of the score."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

import paged_reference as ref  # noqa: E402
from test_gpu_paged import Attention  # noqa: E402
from test_gpu_prompt import Device, host  # noqa: E402

BAD = [np.nan, np.inf, -np.inf, 3e38, 1e30]


def error_of(A, D, n, bias=0.0):
    """(absolute error of a score, relative error of a weight and of sums of n of them) of scores of up to A."""
    ds = (D + 8 + 12) * 2.0 ** -24 * A + 2.0 ** -24 * (A + bias)
    return ds, 2 * ds + 2.0 ** -22 * (2 * A + 1) + n * 2.0 ** -24


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("slopes", [False, True], ids=["", "slopes"])
@pytest.mark.parametrize("lens,D", [([150], 64), ([150] + [2] * 600, 128), ([700], 32)], ids=["few", "many", "runs"])
def test_keys_that_a_row_does_not_see(lens, D, slopes, dtype):
    make = lambda: ref.Prompts(lens, 4, 2, D, dtype, seed=7, window=60, prefix=[4] + [0] * (len(lens) - 1), cap=40.0, std=2.0, slopes=slopes)
    clean = Device(make())
    assert clean.p.magnitude() > 2
    clean.attend(), clean.weigh()
    token = np.arange(clean.p.tokens)
    sees = (token >= 70) & (token - 70 < 60)
    for bad in BAD:
        p = make()
        p.k[70] = ref.stored(np.full(p.k[70].shape, bad), dtype)
        d = Device(p)
        d.attend()
        for got, want in ((d.out, clean.out), (d.row_max, clean.row_max), (d.row_norm, clean.row_norm)):
            np.testing.assert_array_equal(host(got)[~sees], host(want)[~sees])
        # utilities: an entry's scores are its own, whatever its neighbours hold
        d.row_max, d.row_norm = clean.row_max, clean.row_norm
        d.weigh()
        np.testing.assert_array_equal(np.delete(host(d.mass), 70), np.delete(host(clean.mass), 70))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tq,D,S", [(1, 64, 100), (1, 128, 700), (3, 32, 90), (1, 64, 6000)])
def test_entries_that_a_step_does_not_see(tq, D, S, dtype):
    make = lambda: Attention(1, 2, 1, 2, S, D, dtype, 16, 2, tq=tq, seed=5, window=S // 2, full=True, cap=60.0, std=2.0)
    a = make()
    a.run()
    want = [host(x) for x in (a.y, a.row_max, a.row_norm, a.scores)]
    hidden = (a.pos[0, 0] > a.q_pos.max()) | (a.pos[0, 0] <= a.q_pos.min() - S // 2)
    at = np.flatnonzero(hidden)[::2]
    assert len(at) > 8
    for bad in BAD:
        a = make()
        a.K[0, 0, 0, at] = ref.stored(np.full(D, bad), dtype)
        a.run()
        for got, w in zip((a.y, a.row_max, a.row_norm, a.scores), want):
            np.testing.assert_array_equal(host(got), w)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap", [1e4, 1e6, 1e30])
@pytest.mark.parametrize("lens,Hq,Hkv,D", [([130], 4, 2, 64), ([300] * 20, 16, 8, 128)], ids=["split", "whole"])
def test_a_row_beside_one_with_huge_scores(lens, Hq, Hkv, D, cap, dtype):
    """Rows of ordinary scores under a large cap keep the bits of their scores where a wave also holds rows that reach the cap."""
    p = ref.Prompts(lens, Hq, Hkv, D, dtype, seed=9, cap=cap)
    A = p.magnitude()
    huge = np.zeros((p.tokens, Hq), bool)
    huge[::9, 0] = True
    p.q[huge] = ref.stored(p.q[huge] * cap, dtype)
    d = Device(p)
    d.attend()
    d_norm, d_max, d_out = host(d.row_norm), host(d.row_max), host(d.out)
    out, top, norm, weight, _ = p.attend()
    ds, e = error_of(A, D, max(lens))
    keep = ~huge
    assert (np.abs(d_max - top)[keep] <= ds + 2.0 ** -23 * np.abs(top[keep])).all(), float(np.abs(d_max - top)[keep].max() / ds)
    assert (np.abs(d_norm - norm)[keep] <= e * norm[keep]).all(), float((np.abs(d_norm - norm)[keep] / norm[keep]).max() / e)
    bar = 2 * e * weight + 2.0 ** -24 * np.abs(out)
    if dtype == "bf16":
        bar += 2.0 ** -8 * weight + (1 + 2.0 ** -8) * 2.0 ** -8 * (np.abs(out) + bar) + 2.0 ** -133
    assert (np.abs(d_out - out)[keep] <= bar[keep]).all()
    # the utilities that those rows give: the others' sums are left out
    d.row_norm[torch.from_numpy(huge).to(d.row_norm.device)] = 0.0
    d.weigh()
    want = p.mass(host(d.row_max), host(d.row_norm))
    assert (np.abs(host(d.mass) - want) <= (e + (Hq + 4) * 2.0 ** -24) * want + 2.0 ** -120).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap", [1e4, 1e6])
@pytest.mark.parametrize("G,D,S,slopes", [(4, 64, 100, False), (16, 128, 700, True), (33, 32, 300, False)])
def test_a_head_beside_one_with_huge_scores(G, D, S, slopes, cap, dtype):
    a = Attention(2, 3, 2, G, S, D, dtype, 16, 2, seed=4, cap=cap, slopes=slopes)
    a.run()
    A = a.reference()[5]
    huge = np.zeros((2, a.Hq), bool)
    huge[:, ::G] = True
    a.q[huge] = ref.stored(a.q[huge] * cap, dtype)
    a.run()
    y, top, norm, weight, raw, _ = a.reference()
    ds, e = error_of(A, D, 300, 40.0 if slopes else 0.0)
    fine = ~huge & np.isfinite(top)
    assert (np.abs(host(a.row_max) - top)[fine] <= ds + 2.0 ** -23 * np.abs(top[fine])).all()
    assert (np.abs(host(a.row_norm) - norm)[fine] <= e * norm[fine]).all()
    assert (np.abs(host(a.y) - y) <= 2 * e * weight + 2.0 ** -23 * np.abs(y) + 2.0 ** -120)[fine].all()
    s = host(a.scores)
    seen = np.isfinite(raw) & ~huge[:, :, None, None]
    assert (np.abs(s - raw)[seen] <= ds + 2.0 ** -23 * np.abs(raw[seen])).all()
