"""Long streams through full 8-bit shards, bit for bit against the plain form: what an entry leaves behind when it goes."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

import paper_2508_06526_amd as pk  # noqa: E402
import quant_recovery as rec  # noqa: E402
import quant_reference as ref  # noqa: E402
from test_gpu_quant import E4M3, INT8, Cache, i32, make_values, same_codes, up  # noqa: E402


class Stream:
    """Full shards whose entries are replaced one by one, here and in the plain form."""

    def __init__(self, S, D, Hkv, dtype, fmt, block, seed, values=None):
        self.shape = B, E, _, _, _ = (2, 3, Hkv, S, D)
        self.rng, self.dtype, self.fmt, self.block = np.random.default_rng(seed), dtype, fmt, block
        self.cache = Cache(*self.shape, dtype, fmt, block, pad=16, gap=1)
        self.cache.pack(make_values(self.rng, self.shape, dtype, spread=0.3) if values is None else values, np.full((B, E), S))
        self.codes, self.scales = self.cache.host()
        self.utility = torch.ones((B, E, S), device="cuda:0")
        self.topk = np.array([[0, 2], [2, 1]])

    def row(self, size=1.0):
        B, _, Hkv, _, D = self.shape
        return [ref.rounded(self.rng.normal(size=(B, Hkv, D)) * size, self.dtype) for _ in range(2)]

    def replace(self, slot, rows):
        B, E, _, S, _ = self.shape
        freed, cnt, n = np.full((B, E, 1), slot), np.ones((B, E), int), i32(np.full((B, E), S - 1))
        pk.pikv_quant_append(self.cache.desc, self.fmt, self.block, up(rows[0], self.dtype), up(rows[1], self.dtype), i32(self.topk), 2, i32(freed),
                             i32(cnt), 1, *self.cache.tabs, *self.cache.scales, self.utility, n)
        for b in range(B):
            for e in self.topk[b]:
                for x, c, s in zip(rows, self.codes, self.scales):
                    rec.append(x[b].astype(np.float64), slot, S - 1, 1, self.fmt, self.block, c[b, e], s[b, e], S)

    def check(self):
        codes, scales = self.cache.host()
        for got, want, gs, ws in zip(codes, self.codes, scales, self.scales):
            np.testing.assert_array_equal(gs.view(np.uint32), ws.view(np.uint32))
            same_codes(got, want, self.fmt)
        self.cache.padding_is_untouched()
        return scales


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", [INT8, E4M3], ids=["int8", "e4m3"])
@pytest.mark.parametrize("S,D,Hkv,block", [(70, 64, 3, 32), (130, 128, 20, 128), (33, 32, 2, 16)])
def test_scales_come_down_after_a_large_entry(S, D, Hkv, block, fmt, dtype):
    s = Stream(S, D, Hkv, dtype, fmt, block, seed=21)
    large = S // 2
    s.replace(large, s.row(1000.0))
    s.replace(S - 1, s.row(1e-3))                        # a last block of few slots: a small entry beside small ones
    held = s.check()[0][0, 0, :, large // block].copy()
    for slot in s.rng.permutation(S):
        s.replace(slot, s.row())
    after = s.check()[0][0, 0, :, large // block]
    assert (after <= held / 32).all()                    # 2^-10 of the large entry's values, four times that at most, a power of two each
    assert (s.utility[0, 0] == 0).all()
