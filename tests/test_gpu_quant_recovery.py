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
from test_gpu_quant import E4M3, INT8, Attn, Cache, i32, make_values, same_codes, up  # noqa: E402


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
@pytest.mark.parametrize("S,D,Hkv,block", [(70, 64, 3, 32), (130, 128, 2, 128), (24, 128, 40, 16), (33, 32, 2, 16)])
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


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", [INT8, E4M3], ids=["int8", "e4m3"])
@pytest.mark.parametrize("S,D,Hkv,block", [(70, 64, 3, 32), (130, 128, 2, 128), (40, 128, 40, 16), (40, 32, 2, 16)])
def test_entries_that_are_not_finite_are_forgotten_with_their_slots(S, D, Hkv, block, fmt, dtype):
    s = Stream(S, D, Hkv, dtype, fmt, block, seed=22)
    at = [S // 2, S // 2 + 1, 0]
    for slot, bad in zip(at, (np.nan, np.inf, -np.inf)):
        rows = s.row()
        rows[0][0, 1, D - 1] = rows[1][1, 0, 3] = bad
        s.replace(slot, rows)
    scales = s.check()
    assert np.isnan(scales[0][0, [0, 2], 1, at[0] // block]).all() and np.isfinite(scales[0][0, :, 0]).all() and np.isfinite(scales[0][0, 1]).all()
    n = np.full(s.shape[:2], S)
    K = s.cache.read(n)[0].float()
    lo = at[0] // block * block
    assert torch.isnan(K[0, 0, 1, lo:min(lo + block, S), :D]).all() and torch.isfinite(K[0, 0, 0, :S, :D]).all()
    for slot in (at[0] - 1, at[1] + 1):                  # beside them, a large and a small one
        s.replace(slot, s.row(30.0 if slot < at[0] else 0.01))
    s.check()
    for i, slot in enumerate(at):
        s.replace(slot, s.row())
        s.check()
    got = s.check()
    assert all(np.isfinite(a).all() for a in got)
    for slot in s.rng.permutation(S)[:20]:
        s.replace(slot, s.row())
    s.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", [INT8, E4M3], ids=["int8", "e4m3"])
@pytest.mark.parametrize("S,D,block", [(100, 64, 16), (333, 128, 128), (70, 32, 64), (129, 128, 32)])
def test_packed_rows_that_are_not_finite(S, D, block, fmt, dtype):
    shape = B, E, Hkv = 2, 3, 2
    rng = np.random.default_rng(23)
    values = make_values(rng, shape + (S, D), dtype, spread=0.3)
    n = np.array([[S, S - 3, 0], [1, S // 2, S]])
    for v in values:
        for _ in range(12):
            v[rng.integers(B), rng.integers(E), rng.integers(Hkv), rng.integers(S), rng.integers(D)] = rng.choice([np.nan, np.inf, -np.inf])
        v[1, 0, 0, 0, 5] = np.nan                        # a shard's only entry
        v[0, 0, 1, :block] = np.inf                      # all entries of a block
    cache = Cache(*shape, S, D, dtype, fmt, block, pad=16, gap=3)
    want = cache.host()
    for v, c, a in zip(values, *want):
        rec.pack(v.astype(np.float64), n, fmt, block, c, a)
    cache.pack(values, n)
    codes, scales = cache.host()
    for got, c, gs, a in zip(codes, want[0], scales, want[1]):
        written = ~np.isnan(a) | (rec.bits(a) != 0x7fc00000)
        np.testing.assert_array_equal(gs.view(np.uint32)[written], rec.bits(a)[written])
        assert np.isnan(gs[~written]).all()
        same_codes(got, c, fmt)
    cache.padding_is_untouched()
    K = cache.read(n)[0].float().cpu().numpy()[..., :S, :D]
    live = np.broadcast_to((np.arange(S) < n[..., None])[:, :, None, :, None], K.shape)
    assert np.isnan(K[~np.isfinite(values[0]) & live]).all()


def test_shards_filled_past_a_row_that_is_not_finite_and_streamed_through():
    """Appended behind the last entry such a row costs its block all codes; they are whole again when every slot is rewritten."""
    B, E, Hkv, S, D, block = 1, 1, 2, 40, 64, 16
    cache = Cache(B, E, Hkv, S, D, "f32", INT8, block)
    n, u = i32([[0]]), torch.zeros((B, E, S), device="cuda:0")
    rng = np.random.default_rng(24)
    codes, scales = cache.host()
    for i in range(S + 40):
        x = rng.normal(size=(2, 1, Hkv, D)).astype(np.float32)
        if i == 18:
            x[0, 0, 1, 3] = np.nan
        full, slot = i >= S, i if i < S else (7 * i) % S
        n.fill_(min(i, S - 1))
        pk.pikv_quant_append(cache.desc, INT8, block, up(x[0]), up(x[1]), i32([[0]]), 1, i32([[[slot]]]) if full else None, i32([[1]]) if full else None,
                             1 if full else 0, *cache.tabs, *cache.scales, u, n)
        for r, c, s in zip(x, codes, scales):
            rec.append(r[0].astype(np.float64), slot, min(i, S - 1), int(full), INT8, block, c[0, 0], s[0, 0], S)
        if i in (20, S, S + 10, S + 39):
            for got, want, gs, ws in zip(cache.host()[0], codes, cache.host()[1], scales):
                live = ~np.isnan(gs) | (gs.view(np.uint32) != 0x7fc00000)
                np.testing.assert_array_equal(np.isnan(gs), np.isnan(ws))
                np.testing.assert_array_equal(gs.view(np.uint32)[live], ws.view(np.uint32)[live])
                np.testing.assert_array_equal(got, want)
            assert np.isnan(cache.host()[1][0][0, 0, 1, 1]) == (i < S + 39)


@pytest.mark.parametrize("S", [100, 700], ids=["merged", "split"])
def test_attention_sees_a_poisoned_block_until_its_row_is_gone(S):
    a = Attn(1, 4, 2, 64, 2, S, 2, n=S, seed=25, dtype="f32")
    one, cnt = i32([[[40], [40]]]), i32([[1, 1]])

    def put(x):
        n = i32([[S - 1, S - 1]])
        pk.pikv_quant_append(a.cache.desc, INT8, a.cache.block, up(x[0]), up(x[1]), i32([[1, 0]]), 2, one, cnt, 1, *a.cache.tabs, *a.cache.scales,
                             torch.zeros((1, 2, S), device="cuda:0"), n)

    x = np.random.default_rng(26).normal(size=(2, 1, 2, 64)).astype(np.float32)
    x[1, 0, 1, 0] = np.inf
    put(x)
    a.run()
    torch.cuda.synchronize()
    assert torch.isfinite(a.y[0, :2]).all() and torch.isnan(a.y[0, 2:]).all()
    x[1, 0, 1, 0] = 0.5
    put(x)
    codes, scales = a.cache.host()
    a.K, a.V = (ref.values(c, s, a.cache.fmt, a.cache.block) for c, s in zip(codes, scales))
    a.buffers()
    a.run()
    a.check()
