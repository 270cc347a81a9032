"""Scores and outputs of the 8-bit attention to the bits that fp32 queries and weights have: quant_precision.py derives inputs and bars."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

import quant_precision as prec  # noqa: E402
import quant_reference as ref  # noqa: E402
from test_gpu_quant import E4M3, INT8, Attn  # noqa: E402

SHAPES = [dict(B=2, Hq=4, Hkv=2, E=3, S=100, k=2), dict(B=1, Hq=32, Hkv=4, E=2, S=700, k=1), dict(B=1, Hq=2, Hkv=1, E=2, S=5000, k=2)]


def place(a, codes, scales):
    """Codes (their values) and scales of K and V."""
    fmt = a.cache.fmt
    coded = [ref.encode(c, fmt).view(np.uint8) for c in codes]
    full = [np.full(a.cache.scales[0].shape, s, np.float32) for s in scales]
    a.cache.set(coded, full)
    a.K, a.V = (ref.values(c, s, fmt, a.cache.block) for c, s in zip(coded, full))


@pytest.mark.parametrize("fmt", [INT8, E4M3], ids=["int8", "e4m3"])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("spec", SHAPES, ids=lambda s: "S%d" % s["S"])
def test_scores_have_all_bits_of_fp32_queries(spec, D, fmt):
    rng = np.random.default_rng(D + spec["S"])
    a = Attn(**spec, D=D, dtype="f32", fmt=fmt, n=spec["S"], seed=51)
    shape = (spec["B"], spec["E"], spec["Hkv"], spec["S"], D)
    place(a, [prec.sparse_codes(rng, shape, fmt), prec.sparse_codes(rng, shape, fmt)], [2.0 ** -9, 1.0])
    a.q = prec.queries(rng, a.q.shape)
    a.buffers()
    a.run(scale=0.25)
    torch.cuda.synchronize()
    want = a.reference(scale=0.25)["scores"]
    assert (np.abs(a.scores.cpu().numpy() - want) <= prec.SCORE_BAR * want).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", [INT8, E4M3], ids=["int8", "e4m3"])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("spec", SHAPES, ids=lambda s: "S%d" % s["S"])
def test_outputs_have_all_bits_of_the_weights(spec, D, fmt, dtype):
    rng = np.random.default_rng(D + spec["S"])
    a = Attn(**spec, D=D, dtype=dtype, fmt=fmt, n=spec["S"], seed=52, gates=False)
    B, E, Hkv, S = (spec[x] for x in ("B", "E", "Hkv", "S"))
    top = 127.0 if fmt == INT8 else 448.0
    K, V = np.zeros((B, E, Hkv, S, D)), prec.sparse_codes(rng, (B, E, Hkv, S, D), fmt)
    K[..., 1] = -top
    for b in range(B):
        for h in range(Hkv):
            v = rng.choice(prec.weight_codes(fmt))                   # (the same in every shard: what is lost adds up)
            for e in range(E):
                one, two = rng.choice(S, 2, replace=False)
                K[b, e, h, [one, two], 1] = 0
                K[b, e, h, two, 0] = -v
                V[b, e, h, one] = 0
                V[b, e, h, two] = ref.decode(rng.integers(1, 127, D).astype(np.uint8), fmt)
    place(a, [K, V], [prec.KEY_STEP[fmt], 0.5])
    a.q = np.zeros(a.q.shape, np.float32)
    a.q[..., 0], a.q[..., 1] = 1.0, 1024.0
    a.buffers()
    a.run(scale=1.0)
    torch.cuda.synchronize()
    want = a.reference(scale=1.0)["y"]
    assert (want > 0).all() and (np.abs(a.y.cpu().numpy() - want) <= prec.Y_BAR * want).all()
