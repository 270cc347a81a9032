"""Norms of queries and keys with the position rotation, against the plain 64-bit form.

Bars.  bf16: the 64-bit value rounded once is off by at most half a step, 2^-8 of it relative; what the kernel holds in fp32 before it
rounds is off by at most e = 16 * 2^-24 * (|z_a| + |z_b|) (sum of up to 128 squares joined in a tree of 7 + 7 additions and halved by the
root: 8 roundings; root, division, two products: 4; cosine or sine, product, sum: 4) - so |d| <= 2^-8 |ref| + e (1 + 2^-8).  fp32: e
and the last rounding, 2^-24 |ref|."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

import paper_2508_06526_amd as pk  # noqa: E402
import quant_reference as ref  # noqa: E402

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def up(a, dtype):
    return torch.from_numpy(np.asarray(a, np.float32)).to(DEV).to(DTYPES[dtype])


def make(tokens, Hq, Hkv, D, R, dtype, norm=True, value=True, reach=5000, pad=0, seed=0):
    rng = np.random.default_rng(seed)
    heads = Hq + Hkv * (2 if value else 1)
    c = dict(tokens=tokens, Hq=Hq, Hkv=Hkv, D=D, R=R, dtype=dtype, stride=heads * D + pad)
    c["x"] = ref.rounded(rng.normal(0, 2, (tokens, heads, D)) * np.exp(rng.normal(0, 1, (tokens, heads, 1))), dtype)
    c["w"] = [ref.rounded(1 + 0.2 * rng.normal(size=D), dtype) if norm else None for _ in range(2)]
    c["positions"] = rng.integers(0, reach, tokens).astype(np.int32)
    c["inv_freq"] = (10000.0 ** (-np.arange(0, R, 2) / max(R, 1))).astype(np.float32)
    return c


def run(c, interleaved, eps=1e-6, x=None, value=True):
    t, n, Hq, Hkv, D = DTYPES[c["dtype"]], c["tokens"], c["Hq"], c["Hkv"], c["D"]
    if x is None:
        wide = torch.full((n, c["stride"]), float("nan"), device=DEV, dtype=t)
        x = wide[:, :c["x"].shape[1] * D]
        x.copy_(up(c["x"].reshape(n, -1), c["dtype"]))
    w = [None if a is None else up(a, c["dtype"]) for a in c["w"]]
    out = [torch.full((n + 1, h, D), 7.0, device=DEV, dtype=t) for h in (Hq, Hkv, Hkv)]         # a row behind the last
    pos = torch.from_numpy(c["positions"]).to(DEV)
    freq = torch.from_numpy(c["inv_freq"]).to(DEV) if c["R"] else None
    pk.pikv_norm_rope(x, n, c["stride"], Hq, Hkv, D, w[0], w[1], eps, pos if c["R"] else None, freq, c["R"], interleaved,
                      out[0] if Hq else None, out[1] if Hkv else None, out[2] if value and Hkv else None)
    torch.cuda.synchronize()
    assert all((o[n] == 7.0).all() for o in out)
    return [o[:n].float().cpu().numpy().astype(np.float64) for o in out]


def check(c, got, interleaved, eps=1e-6, value=True):
    Hq, Hkv, R = c["Hq"], c["Hkv"], c["R"]
    x = c["x"].astype(np.float64)
    step = 2.0 ** -8 if c["dtype"] == "bf16" else 2.0 ** -24
    for out, rows, w in ((got[0], x[:, :Hq], c["w"][0]), (got[1], x[:, Hq:Hq + Hkv], c["w"][1])):
        w = None if w is None else w.astype(np.float64)
        want = ref.norm_rope(rows, w, eps, c["positions"], c["inv_freq"], R, interleaved)
        z = np.abs(ref.norm_rope(rows, w, eps, 0 * c["positions"], c["inv_freq"], 0, interleaved))
        i = np.arange(R // 2)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
        both = z.copy()
        both[..., a] = both[..., b] = z[..., a] + z[..., b]
        e = 16 * 2.0 ** -24 * both
        err = np.abs(out - want)
        assert (err <= step * np.abs(want) + e * (1 + step) + 1e-40).all(), (err / (np.abs(want) + both + 1e-30)).max()
    if value:
        np.testing.assert_array_equal(got[2], x[:, Hq + Hkv:])


SHAPES = [  # tokens, Hq, Hkv, D, R
    (1, 32, 8, 128, 128), (1, 1, 1, 16, 16), (3, 7, 1, 64, 32), (37, 6, 2, 64, 64), (5, 4, 4, 32, 16), (2, 17, 5, 128, 96), (130, 3, 3, 16, 0),
    (1, 128, 8, 128, 64), (700, 32, 8, 128, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "T%d_%d_%d_D%d_R%d" % s)
def test_norm_rope(shape, interleaved, dtype):
    c = make(*shape, dtype)
    check(c, run(c, interleaved), interleaved)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_without_norm_without_values_and_rows_of_a_wider_projection(dtype):
    c = make(9, 4, 2, 64, 64, dtype, norm=False, value=False, pad=48)
    check(c, run(c, False, value=False), False, value=False)
    c = make(9, 4, 2, 64, 32, dtype, pad=64, seed=4)
    c["w"][1] = None                                   # queries are normed, keys are not
    check(c, run(c, True), True)


@pytest.mark.parametrize("side", ["queries", "keys"])
def test_queries_or_keys_alone(side):
    c = make(11, 5 if side == "queries" else 0, 0 if side == "queries" else 3, 128, 128, "bf16")
    check(c, run(c, False), False)


@pytest.mark.parametrize("reach", [1 << 20, (1 << 31) - 1])
def test_far_positions_keep_their_angles(reach):
    c = make(64, 2, 1, 128, 128, "f32", reach=reach)
    c["positions"][:3] = [0, reach - 1, -5]
    check(c, run(c, False), False)


def test_zero_rows_and_non_finite_rows_stay_where_they_are():
    c = make(4, 2, 1, 64, 64, "f32")
    c["x"][1, 0] = 0.0
    c["x"][2, 1, 5] = np.nan
    c["x"][3, 2, 7] = np.inf
    got = run(c, False)
    assert (got[0][1, 0] == 0).all()
    assert np.isnan(got[0][2, 1]).all() and np.isfinite(got[0][2, 0]).all() and np.isfinite(got[1][2]).all()
    # an infinite key: its norm is infinite, the others of its head are x / inf, it and its partner in the rotation inf / inf
    pair = np.isin(np.arange(64), [7, 39])
    assert np.isfinite(got[0][3]).all() and np.isnan(got[1][3, 0, pair]).all() and (got[1][3, 0, ~pair] == 0).all()


def test_no_tokens_is_a_no_op():
    z = torch.zeros(4096, device=DEV, dtype=torch.bfloat16)
    i, f = torch.zeros(1, device=DEV, dtype=torch.int32), torch.zeros(32, device=DEV)
    out = torch.ones(4096, device=DEV, dtype=torch.bfloat16)
    pk.pikv_norm_rope(z, 0, 512, 4, 2, 64, None, None, 1e-6, i, f, 64, False, out, out, out)
    torch.cuda.synchronize()
    assert (out == 1).all()
