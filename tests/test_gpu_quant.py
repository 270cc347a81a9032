"""The cache held in 8 bits: written from dense shards, by new entries, read back, attended over - against the plain 64-bit forms.

Codes and scales are compared bit for bit (scales are powers of two; a code is one rounding).  Attention: with A the largest
sum of |q_d K_d| * scale over entries, a score is off by at most ds = (D + 8) 2^-24 A (D products summed in fp32), a weight exp(s - M) by
2 ds + 2^-22 |s - M| relative, the sums by another 2^-24 per addition of a chain: chains are at most 300 long here (128 of a
wave, splits and shards joined).  |s - M| <= 2 A.  So |dy| <= 2 (2 ds + 2^-21 A + 300 2^-24) max|V|, row_max within ds, row_norm
within the weights' relative error.  Errors of thousands of weights being independent, the bound on the norm of dy is a tenth of that."""
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
INT8, E4M3 = pk.QUANT_INT8, pk.QUANT_E4M3


def up(a, dtype="f32"):
    return torch.from_numpy(np.array(a, np.float32)).to(DEV).to(DTYPES[dtype])


def i32(a):
    return torch.from_numpy(np.array(a, np.int32)).to(DEV)


class Cache:
    """Shards of codes (bytes full of `fill`, scales NaN) with their dense side, rows `pad` elements apart beyond D."""

    def __init__(self, B, E, Hkv, S, D, dtype, fmt, block, pad=0, gap=0, fill=0xA5, dense_pad=None, **desc):
        self.shape, self.dtype, self.fmt, self.block = (B, E, Hkv, S, D), dtype, fmt, block
        self.pad, self.rows = pad // 2 if dense_pad is None else dense_pad, S + gap
        self.codes = [torch.full((B, E, Hkv, self.rows, D + pad), fill, device=DEV, dtype=torch.uint8) for _ in range(2)]
        self.scales = [torch.full((B, E, Hkv, -(-S // block)), float("nan"), device=DEV) for _ in range(2)]
        self.tabs = [pk.shard_table([t[b, e] for b in range(B) for e in range(E)]) for t in self.codes]
        self.desc = pk.make_desc(**dict(dict(B=B, Hq=Hkv, Hkv=Hkv, D=D, E=E, S=S, dtype=int(dtype == "bf16"), stride_s=D + pad,
                                             stride_h=self.rows * (D + pad)), **desc))

    def dense(self, values=None):
        """Two dense shards (K, V) of the cache's type with their tables and strides."""
        B, E, Hkv, S, D = self.shape
        pad = self.pad
        bufs = [torch.full((B, E, Hkv, self.rows, D + pad), 3.0, device=DEV, dtype=DTYPES[self.dtype]) for _ in range(2)]
        if values is not None:
            for t, v in zip(bufs, values):
                t[..., :S, :D] = up(v, self.dtype)
        return bufs, [pk.shard_table([t[b, e] for b in range(B) for e in range(E)]) for t in bufs], (self.rows * (D + pad), D + pad)

    def host(self):
        """Codes [B, E, Hkv, S, D] (bytes) and scales of K and V."""
        S, D = self.shape[3:]
        torch.cuda.synchronize()
        return [t[..., :S, :D].cpu().numpy().copy() for t in self.codes], [t.cpu().numpy().copy() for t in self.scales]

    def set(self, codes, scales):
        S, D = self.shape[3:]
        for t, a in zip(self.codes, codes):
            t[..., :S, :D] = torch.from_numpy(a).to(DEV)
        for t, a in zip(self.scales, scales):
            t.copy_(torch.from_numpy(np.asarray(a, np.float32)))

    def pack(self, values, n_valid):
        _, tabs, strides = self.dense(values)
        pk.pikv_quant_pack(self.desc, self.fmt, self.block, *tabs, *strides, i32(n_valid), *self.tabs, *self.scales)

    def read(self, n_valid):
        bufs, tabs, strides = self.dense()
        pk.pikv_quant_read(self.desc, self.fmt, self.block, *self.tabs, *self.scales, i32(n_valid), *tabs, *strides)
        torch.cuda.synchronize()
        return bufs

    def padding_is_untouched(self, fill=0xA5):
        S, D = self.shape[3:]
        assert all((t[..., D:] == fill).all() and (t[..., S:, :] == fill).all() for t in self.codes)


def same_codes(got, want, fmt):
    np.testing.assert_array_equal(ref.decode(got, fmt), ref.decode(want, fmt))       # (a negative zero is a zero)


def make_values(rng, shape, dtype, spread=1.0):
    B, E, Hkv, S, D = shape
    return [ref.rounded(rng.normal(size=shape) * np.exp(rng.normal(0, spread, (B, E, Hkv, S, 1))), dtype) for _ in range(2)]


def expected_pack(values, n_valid, fmt, block, fill=0xA5):
    out = []
    for v in values:
        codes = np.full(v.shape, fill, np.uint8)
        scales = np.full(v.shape[:3] + (-(-v.shape[3] // block),), np.nan)
        ref.pack(v.astype(np.float64), n_valid, fmt, block, codes, scales)
        out.append((codes, scales))
    return out


def check_pack(cache, values, n_valid):
    cache.pack(values, n_valid)
    codes, scales = cache.host()
    for got_c, got_s, (want_c, want_s) in zip(codes, scales, expected_pack(values, n_valid, cache.fmt, cache.block)):
        np.testing.assert_array_equal(got_s, want_s.astype(np.float32))
        live = np.arange(cache.shape[3]) < np.asarray(n_valid)[..., None]
        live = np.broadcast_to(live[:, :, None, :, None], got_c.shape)
        same_codes(got_c[live], want_c[live], cache.fmt)
        assert (got_c[~live] == 0xA5).all()
    cache.padding_is_untouched()


def check_read(cache, n_valid):
    codes, scales = cache.host()
    S, D = cache.shape[3:]
    live = np.broadcast_to((np.arange(S) < np.asarray(n_valid)[..., None])[:, :, None, :, None], cache.shape)
    for got, c, s in zip(cache.read(n_valid), codes, scales):
        with np.errstate(over="ignore", under="ignore"):
            want = ref.rounded(np.float32(ref.values(c, s, cache.fmt, cache.block)), cache.dtype)
        out = got.float().cpu().numpy()
        np.testing.assert_array_equal(out[..., :S, :D][live], want[live])
        assert (out[..., :S, :D][~live] == 3.0).all() and (out[..., D:] == 3.0).all() and (out[..., S:, :] == 3.0).all()


GEOMETRIES = [  # B, E, Hkv, S, D, pad, gap
    (1, 1, 1, 1, 128, 0, 0), (2, 3, 2, 100, 64, 0, 0), (1, 2, 3, 333, 32, 16, 5), (2, 2, 2, 129, 128, 32, 1), (1, 4, 1, 64, 64, 0, 0)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", [INT8, E4M3], ids=["int8", "e4m3"])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("geo", GEOMETRIES, ids=lambda g: "B%d_E%d_H%d_S%d_D%d" % g[:5])
def test_pack_and_read_back(geo, block, fmt, dtype):
    shape = geo[:5]
    rng = np.random.default_rng(5)
    cache = Cache(*shape, dtype, fmt, block, pad=geo[5], gap=geo[6])
    n = rng.integers(0, shape[3] + 1, shape[:2])
    n[0, 0] = shape[3]
    if shape[1] > 1:
        n[0, 1] = 0
    if shape[1] > 2:
        n[0, 2] = 1
    check_pack(cache, make_values(rng, shape, dtype), n)
    check_read(cache, n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", [INT8, E4M3], ids=["int8", "e4m3"])
def test_values_at_the_borders_of_the_formats(fmt, dtype):
    """Zeros, ties, the ends of the range, subnormal magnitudes, infinities and NaN; entries behind the last are not read."""
    S, D = 64, 32
    rng = np.random.default_rng(6)
    v = np.zeros((1, 1, 1, S, D), np.float32)
    v[0, 0, 0, :16] = rng.integers(-127, 128, (16, D)) + 0.5 * rng.integers(0, 2, (16, D))      # int8: ties under scale 1
    v[0, 0, 0, 0, 0] = 127.0
    top = 127.0 if fmt == INT8 else 448.0
    v[0, 0, 0, 16, :4] = [top, -top, np.nextafter(np.float32(top), np.float32(1e9)) if dtype == "f32" else top * 1.0078125, 3.0]
    v[0, 0, 0, 32, :5] = [1e-39, -3e-40, 2.0 ** -133, 2.0 ** -126, 0.0]
    v[0, 0, 0, 48:] = ref.rounded(rng.normal(size=(16, D)) * 1e37, dtype)
    v = ref.rounded(v, dtype)
    values = [v, -v]
    n = np.array([[60]])
    values[0][0, 0, 0, 60:] = np.nan
    values[1][0, 0, 0, 60:] = np.inf
    cache = Cache(1, 1, 1, S, D, dtype, fmt, 16)
    check_pack(cache, values, n)
    check_read(cache, n)
    for bad in (np.nan, np.inf, -np.inf):
        poisoned = [values[0].copy(), values[1].copy()]
        poisoned[0][0, 0, 0, 20, 3] = bad
        cache = Cache(1, 1, 1, S, D, dtype, fmt, 16)
        cache.pack(poisoned, n)
        scales = cache.host()[1]
        assert np.isnan(scales[0][0, 0, 0, 1]) and np.isfinite(scales[0][0, 0, 0, [0, 2, 3]]).all() and np.isfinite(scales[1]).all()
        K = cache.read(n)[0].float()
        assert torch.isnan(K[0, 0, 0, 16:32]).all() and torch.isfinite(K[0, 0, 0, :16]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", [INT8, E4M3], ids=["int8", "e4m3"])
@pytest.mark.parametrize("block,D,Hkv", [(16, 128, 3), (32, 64, 40), (64, 32, 2), (128, 128, 40)])
def test_appended_entries(block, D, Hkv, fmt, dtype):
    """Shards that are empty, inside a block, at a block's start, full, with a freed slot, with several; rows of growing size."""
    B, E, S, k = 2, 5, 2 * block + 3, 4
    rng = np.random.default_rng(7)
    cache = Cache(B, E, Hkv, S, D, dtype, fmt, block, pad=16, gap=2)
    values = make_values(rng, (B, E, Hkv, S, D), dtype, spread=0.3)
    n = np.array([[0, block, S, S - 1, block - 3], [2 * block, 5, S - 4, S - 1, 1]])
    cnt = np.array([[0, 0, 0, 1, 0], [0, 0, 4, 1, 0]])                     # [1, 2]: four slots freed, [., 3]: one
    held = np.minimum(n + cnt, S)
    cache.pack(values, held)
    topk = np.array([[3, 0, 2, 1], [4, 2, 3, 0]])
    freed = np.zeros((B, E, 4), np.int32)
    freed[0, 3], freed[1, 2], freed[1, 3] = S - 1, [1, block + 2, 2 * block, 2 * block + 1], block + 1
    utility = torch.full((B, E, S), 5.0, device=DEV)
    nd = i32(n)
    for step in range(3):
        new = [ref.rounded(rng.normal(size=(B, Hkv, D)) * 4.0 ** step * np.exp(rng.normal(0, 1, (B, Hkv, 1))), dtype) for _ in range(2)]
        codes, scales = cache.host()
        n_before = nd.cpu().numpy()
        pk.pikv_quant_append(cache.desc, fmt, block, up(new[0], dtype), up(new[1], dtype), i32(topk), k, i32(freed), i32(cnt), 4,
                             *cache.tabs, *cache.scales, utility, nd)
        got_codes, got_scales = cache.host()
        n_after = nd.cpu().numpy()
        u = utility.cpu().numpy()
        for b in range(B):
            for e in range(E):
                m, c = int(n_before[b, e]), int(cnt[b, e])
                if e not in topk[b] or m >= S:
                    assert n_after[b, e] == m
                    continue
                slot = int(freed[b, e, 0]) if c > 0 else m
                assert n_after[b, e] == m + 1 and u[b, e, slot] == 0.0
                for x, cc, ss in zip(new, codes, scales):
                    ref.append(x[b].astype(np.float64), slot, m, c, fmt, block, cc[b, e], ss[b, e], S)
        for got, want, gs, ws in zip(got_codes, codes, got_scales, scales):
            np.testing.assert_array_equal(gs, ws.astype(np.float32))
            same_codes(got, want, fmt)
        cnt = np.where(np.isin(np.arange(E), topk) & (cnt > 0), cnt - 1, cnt)          # the caller moves on to the next freed slot
        freed = np.roll(freed, -1, -1)
    cache.padding_is_untouched()


def test_append_without_freed_slots_and_a_poisoned_block():
    B, E, Hkv, S, D, block = 1, 1, 2, 40, 64, 16
    cache = Cache(B, E, Hkv, S, D, "f32", INT8, block)
    n, u = i32([[0]]), torch.zeros((B, E, S), device=DEV)
    rng = np.random.default_rng(8)
    rows = rng.normal(size=(S + 1, 1, Hkv, D)).astype(np.float32)
    rows[18, 0, 1, 3] = np.nan
    for s in range(S + 1):                               # the last one finds the shard full
        pk.pikv_quant_append(cache.desc, INT8, block, up(rows[s]), up(rows[s]), i32([[0]]), 1, None, None, 0, *cache.tabs,
                             *cache.scales, u, n)
    codes, scales = cache.host()
    assert n.item() == S
    want_c, want_s = np.full(cache.shape, 0xA5, np.uint8), np.full((1, 1, Hkv, 3), np.nan)
    for s in range(S):
        ref.append(rows[s, 0].astype(np.float64), s, s, 0, INT8, block, want_c[0, 0], want_s[0, 0], S)
    for got_c, got_s in zip(codes, scales):
        np.testing.assert_array_equal(got_s, want_s.astype(np.float32))
        np.testing.assert_array_equal(got_c, want_c)
    assert np.isnan(scales[0][0, 0, 1, 1]) and np.isfinite(scales[0][0, 0, 1, [0, 2]]).all() and np.isfinite(scales[0][0, 0, 0]).all()


def test_append_into_a_block_of_zeros_that_was_never_written():
    cache = Cache(1, 1, 2, 32, 64, "f32", E4M3, 16, fill=0x3C)          # (bytes that stand for nothing: their scale is 0)
    for s in cache.scales:
        s.zero_()
    n, u, rows = i32([[5]]), torch.zeros((1, 1, 32), device=DEV), up(np.random.default_rng(2).normal(size=(1, 2, 64)))
    assert all((t[0, 0, :, :5] == 0).all() for t in cache.read([[5]]))
    pk.pikv_quant_append(cache.desc, E4M3, 16, rows, rows, i32([[0]]), 1, None, None, 0, *cache.tabs, *cache.scales, u, n)
    after = cache.read([[6]])
    assert all((t[0, 0, :, :5] == 0).all() and (t[0, 0, :, 5] != 0).any() for t in after)


def test_offsets_beyond_32_bits():
    """Rows 4 MiB apart: a kv head's codes span 4.6 GiB, the second head starts behind them."""
    B, E, Hkv, S, D, block = 1, 1, 2, 1150, 32, 64
    cache = Cache(B, E, Hkv, S, D, "bf16", INT8, block, pad=(1 << 22) - D, dense_pad=0, Hq=4)
    rng = np.random.default_rng(17)
    values = make_values(rng, (B, E, Hkv, S, D), "bf16", spread=0.3)
    n = i32([[S - 1]])
    cache.pack(values, [[S - 1]])
    new = [ref.rounded(rng.normal(size=(1, Hkv, D)) * 9, "bf16") for _ in range(2)]
    u = torch.zeros((B, E, S), device=DEV)
    pk.pikv_quant_append(cache.desc, INT8, block, up(new[0], "bf16"), up(new[1], "bf16"), i32([[0]]), 1, None, None, 0, *cache.tabs, *cache.scales, u, n)
    check_read(cache, [[S]])
    got, scales = cache.host()
    want = expected_pack(values, np.array([[S - 1]]), INT8, block)
    for g, s, (wc, ws), x in zip(got, scales, want, new):
        ref.append(x[0].astype(np.float64), S - 1, S - 1, 0, INT8, block, wc[0, 0], ws[0, 0], S)
        np.testing.assert_array_equal(s, ws.astype(np.float32))
        same_codes(g, wc, INT8)
    a = Attn(B, 4, Hkv, D, E, 8, 1)                      # (its geometry is replaced by the cache's)
    a.geo, a.cache, a.n, a.topk, a.gates = (B, 4, Hkv, D, E, S, 1), cache, np.array([[S]]), np.array([[0]]), None
    a.K, a.V = (ref.values(c, s, INT8, block) for c, s in zip(got, scales))
    a.buffers()
    a.run()
    a.check()


# ------------------------------------------------------------------------------ attention
class Attn:
    def __init__(self, B, Hq, Hkv, D, E, S, k, dtype="bf16", fmt=INT8, block=32, per_head=False, tq=1, n=None, seed=0, pad=0, gap=0, gates=True,
                 boost=1.0):
        rng = np.random.default_rng(seed)
        self.geo, self.per_head, self.tq, self.dtype = (B, Hq, Hkv, D, E, S, k), per_head, tq, dtype
        self.cache = Cache(B, E, Hkv, S, D, dtype, fmt, block, pad=pad, gap=gap, Hq=Hq, route_rows_per_seq=Hq if per_head else 1, tq=tq)
        self.n = rng.integers(0, S + 1, (B, E)) if n is None else np.broadcast_to(np.asarray(n), (B, E)).copy()
        self.cache.pack(make_values(rng, (B, E, Hkv, S, D), dtype, spread=0.5), self.n)
        codes, scales = self.cache.host()
        self.K, self.V = (np.nan_to_num(ref.values(c, s, fmt, block)) for c, s in zip(codes, scales))     # (NaN: blocks without entries)
        rows = B * (Hq if per_head else 1)
        self.topk = np.stack([rng.permutation(E)[:k] for _ in range(rows)])
        g = rng.random((rows, k)) + 0.05
        self.gates = (g / g.sum(1, keepdims=True)).astype(np.float32) if gates else None
        self.q = ref.rounded(rng.normal(size=(B, Hq, D)) * boost, dtype)
        self.buffers()

    def buffers(self):
        B, Hq, _, D, _, S, k = self.geo
        nan = float("nan")
        self.y, self.scores = torch.full((B, Hq, D), nan, device=DEV), torch.full((B, Hq, k, S), nan, device=DEV)
        self.row_max, self.row_norm = (torch.full((B, Hq), nan, device=DEV) for _ in range(2))
        self.coef = torch.full((B, Hq, k, 2), nan, device=DEV)
        self.ws = torch.full((pk.pikv_quant_attn_workspace_bytes(self.cache.desc, k),), 0xFF, device=DEV, dtype=torch.uint8)
        self.d = dict(q=up(self.q, self.dtype), n=i32(self.n), topk=i32(self.topk), gates=None if self.gates is None else up(self.gates))

    def run(self, combine=pk.COMBINE_LSE, scale=0.0, scores=True, stats=True, q=None):
        c, d = self.cache, self.d
        pk.pikv_quant_attn(c.desc, c.fmt, c.block, d["q"] if q is None else q, *c.tabs, *c.scales, d["n"], d["topk"], d["gates"], self.geo[6], combine, scale,
                           self.y, self.row_max if stats else None, self.row_norm if stats else None, self.scores if scores else None,
                           self.coef if stats else None, self.ws)

    def reference(self, combine=pk.COMBINE_LSE, scale=None):
        return ref.attend(self.q.astype(np.float64), self.K, self.V, self.n, self.topk, self.gates, self.geo[2],
                          local=combine == pk.COMBINE_LOCAL, tq=self.tq, per_head=self.per_head, scale=scale)

    def bounds(self, scale=None):
        D = self.geo[3]
        scale = D ** -0.5 if scale is None else scale
        A = np.abs(self.q).astype(np.float64).max(axis=(0, 1)) @ np.abs(self.K).max(axis=(0, 1, 2, 3)) * scale     # (no smaller than any entry's)
        most = max(np.linalg.norm(self.q.astype(np.float64), axis=-1).max() * np.linalg.norm(self.K, axis=-1).max() * scale, 1e-30)
        A = min(A, most)
        ds = (D + 8) * 2.0 ** -24 * A
        w = 2 * ds + 2.0 ** -21 * A + 300 * 2.0 ** -24
        return ds, w

    def check(self, combine=pk.COMBINE_LSE, scale=None, scores=True):
        torch.cuda.synchronize()
        want = self.reference(combine, scale)
        ds, w = self.bounds(scale)
        y = self.y.cpu().numpy().astype(np.float64)
        vmax = np.abs(self.V).max() if self.V.size else 0.0
        err = np.abs(y - want["y"])
        assert err.max() <= 2 * w * vmax + 1e-37, (err.max(), 2 * w * vmax)
        assert np.linalg.norm(y - want["y"]) <= 0.1 * 2 * w * np.linalg.norm(want["y"]) + 1e-37
        rm, rn = self.row_max.cpu().numpy(), self.row_norm.cpu().numpy()
        empty = want["row_max"] == -np.inf
        assert (rm[empty] == -np.inf).all() and (rn[empty] == 0).all() and (y[empty] == 0).all()
        assert (np.abs(rm[~empty] - want["row_max"][~empty]) <= ds).all()
        assert (np.abs(rn[~empty] - want["row_norm"][~empty]) <= (w + 2.0 ** -20) * want["row_norm"][~empty]).all()
        if scores:
            got = self.scores.cpu().numpy()
            live = ~np.isnan(want["scores"])
            assert (np.isnan(got) == ~live).all()                    # nothing is written behind a shard's entries
            assert (np.abs(got - want["scores"])[live] <= ds).all()
        return want


ATTN = [
    dict(B=1, Hq=1, Hkv=1, D=128, E=1, S=1, k=1),
    dict(B=2, Hq=8, Hkv=2, D=128, E=4, S=333, k=2),
    dict(B=1, Hq=32, Hkv=8, D=128, E=4, S=1500, k=3),
    dict(B=2, Hq=4, Hkv=4, D=64, E=3, S=200, k=3),
    dict(B=1, Hq=6, Hkv=2, D=32, E=5, S=97, k=2),
    dict(B=1, Hq=48, Hkv=2, D=64, E=2, S=130, k=1),
    dict(B=1, Hq=100, Hkv=1, D=128, E=2, S=70, k=2),
    dict(B=1, Hq=256, Hkv=1, D=32, E=2, S=40, k=2),
    dict(B=3, Hq=7, Hkv=7, D=128, E=64, S=17, k=20),
    dict(B=1, Hq=2, Hkv=1, D=64, E=2, S=5000, k=2),
]


@pytest.mark.parametrize("combine", [pk.COMBINE_LSE, pk.COMBINE_LOCAL], ids=["lse", "local"])
@pytest.mark.parametrize("fmt", [INT8, E4M3], ids=["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("spec", ATTN, ids=lambda s: "_".join("%s%s" % i for i in s.items()))
def test_attention(spec, dtype, fmt, combine):
    a = Attn(**spec, dtype=dtype, fmt=fmt, block=[16, 32, 64, 128][spec["S"] % 4], gates=spec["S"] % 3 != 0)
    a.run(combine)
    a.check(combine)


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("fmt", [INT8, E4M3], ids=["int8", "e4m3"])
@pytest.mark.parametrize("n", [[0, 0, 0, 0], [1, 0, 0, 0], [16, 17, 15, 1], [31, 32, 33, 0], [63, 64, 65, 66], [127, 128, 129, 255], [300, 299, 257, 2]],
                         ids=lambda n: "n" + "_".join(map(str, n)))
def test_counts_around_tiles_and_blocks(n, fmt, block):
    a = Attn(2, 8, 2, 128, 4, 300, 3, fmt=fmt, block=block, n=[n, n[::-1]], seed=3)
    for combine in (pk.COMBINE_LSE, pk.COMBINE_LOCAL):
        a.run(combine)
        a.check(combine)


@pytest.mark.parametrize("spec", [dict(B=2, Hq=8, Hkv=4, D=64, E=5, S=150, k=2, dtype="f32"), dict(B=1, Hq=32, Hkv=4, D=128, E=4, S=260, k=4),
                                  dict(B=1, Hq=4, Hkv=4, D=32, E=4, S=64, k=1, fmt=E4M3)], ids=["f32", "gqa8", "d32"])
def test_routing_per_head(spec):
    a = Attn(**spec, per_head=True, seed=5)
    for combine in (pk.COMBINE_LSE, pk.COMBINE_LOCAL):
        a.run(combine)
        a.check(combine)


@pytest.mark.parametrize("spec", [dict(Hq=32, Hkv=2, tq=4, D=128), dict(Hq=48, Hkv=4, tq=3, D=64, dtype="f32"), dict(Hq=64, Hkv=1, tq=8, D=128, fmt=E4M3),
                                  dict(Hq=10, Hkv=1, tq=5, D=32), dict(Hq=160, Hkv=2, tq=16, D=128), dict(Hq=128, Hkv=4, tq=16, D=64, fmt=E4M3)],
                         ids=lambda s: "tq%d_%d_%d_D%d" % (s["tq"], s["Hq"], s["Hkv"], s["D"]))
def test_draft_queries_in_the_tokens_layout(spec):
    a = Attn(B=2, E=4, S=210, k=2, seed=6, **spec)
    a.run()
    a.check()


@pytest.mark.parametrize("dtype,fmt", [("bf16", INT8), ("f32", E4M3)], ids=["bf16_int8", "f32_e4m3"])
@pytest.mark.parametrize("k", [1, 2, 3, 4, 5, 6, 7, 8, 9, 16, 17])
def test_short_shards_whose_waves_share_a_block(k, dtype, fmt):
    """8 waves over up to 8 shards: a power of two each, some left over; shards without entries, rows without any."""
    E = max(9, k)
    n = np.random.default_rng(k).integers(0, 41, (3, E)) * (np.random.default_rng(k + 50).random((3, E)) < 0.7)
    n[2] = 0
    a = Attn(3, 12, 4, [128, 64][k % 2], E, 40, k, dtype=dtype, fmt=fmt, block=16, n=n, seed=k, gates=k != 4)
    for combine in (pk.COMBINE_LSE, pk.COMBINE_LOCAL):
        a.run(combine)
        want = a.check(combine)
        u = torch.rand((3, E, 40), device=DEV)
        after = u.clone()
        pk.pikv_update_utility(a.cache.desc, a.scores, a.coef, a.d["n"], a.d["topk"], k, 0.5, after)
        visited = np.zeros((3, E, 1), bool)
        for b in range(3):
            visited[b, a.topk[b]] = True
        live = (np.arange(40) < n[..., None]) & visited
        u = u.cpu().numpy().astype(np.float64)
        np.testing.assert_allclose(after.cpu().numpy(), np.where(live, 0.5 * u + want["mass"], u), rtol=1e-4, atol=1e-9)


@pytest.mark.parametrize("spec", [dict(B=48, Hq=8, Hkv=4, D=64, E=3, S=300, k=3), dict(B=47, Hq=8, Hkv=4, D=64, E=3, S=300, k=3),
                                  dict(B=100, Hq=2, Hkv=2, D=128, E=2, S=130, k=2, dtype="f32"), dict(B=25, Hq=8, Hkv=8, D=32, E=4, S=150, k=1, per_head=True),
                                  dict(B=40, Hq=60, Hkv=5, D=64, E=2, S=90, k=2, tq=4, fmt=E4M3), dict(B=161, Hq=4, Hkv=4, D=32, E=2, S=33, k=1),
                                  dict(B=96, Hq=32, Hkv=2, D=128, E=2, S=100, k=2), dict(B=99, Hq=32, Hkv=2, D=128, E=3, S=60, k=3, dtype="f32", fmt=E4M3),
                                  dict(B=3, Hq=32, Hkv=2, D=128, E=2, S=200, k=2), dict(B=1, Hq=32, Hkv=2, D=64, E=20, S=40, k=16, dtype="f32")],
                         ids=lambda s: "B%d_Hkv%d_S%d" % (s["B"], s["Hkv"], s["S"]))
def test_many_sequences(spec):
    """Enough (sequence, kv head) pairs for a block each, and one fewer."""
    a = Attn(**spec, seed=12)
    a.run()
    a.check()


def test_strided_rows_a_given_scale_and_a_query_that_is_not_aligned():
    a = Attn(2, 12, 3, 64, 3, 170, 2, pad=48, gap=7, seed=7)
    q = torch.zeros(a.d["q"].numel() + 1, device=DEV, dtype=torch.bfloat16)[1:].view(a.d["q"].shape)
    q.copy_(a.d["q"])
    a.run(scale=0.3, q=q)
    a.check(scale=0.3)
    f = Attn(2, 12, 3, 64, 3, 170, 2, dtype="f32", seed=7)
    q = torch.zeros(f.d["q"].numel() + 1, device=DEV)[1:].view(f.d["q"].shape)
    q.copy_(f.d["q"])
    f.run(q=q)
    f.check()


def test_large_scores_and_scales_far_apart():
    """Scores of several hundred, and value blocks whose scales are 2^40 apart: the weights of the small ones keep their bits."""
    a = Attn(1, 4, 1, 128, 2, 256, 2, dtype="f32", boost=30.0, n=256, seed=8)
    codes, scales = a.cache.host()
    for s in scales[1][0, 0, 0, ::2], scales[1][0, 1, 0, 1::2]:
        s *= 2.0 ** -40
    a.cache.set(codes, scales)
    a.V = ref.values(codes[1], scales[1], a.cache.fmt, a.cache.block)
    a.run()
    a.check()
    only = a.V[0, :, 0][np.abs(a.V[0, :, 0]).max(-1) < 1e-6]
    assert len(only) == 256
    a.n[:] = 32                                          # of shard 0 only a small block, of shard 1 a large one
    a.topk[:] = [[0, 1]]
    a.gates = np.array([[1.0, 0.0]], np.float32)
    a.buffers()
    a.run()
    torch.cuda.synchronize()
    want = a.reference()["y"]
    assert np.abs(want).max() < 1e-6
    assert np.linalg.norm(a.y.cpu().numpy() - want) <= 0.2 * a.bounds()[1] * np.linalg.norm(want)


def test_a_poisoned_block_shows_in_the_rows_that_read_it_alone():
    a = Attn(1, 4, 2, 64, 3, 100, 2, n=100, seed=9)
    a.topk[:] = [[0, 1]]
    a.buffers()
    a.cache.scales[1][0, 0, 1, 2] = float("nan")        # kv head 1 of a selected shard
    a.cache.scales[0][0, 2] = float("nan")              # a shard nobody selected
    a.run()
    torch.cuda.synchronize()
    assert torch.isfinite(a.y[0, :2]).all() and torch.isnan(a.y[0, 2:]).all()


@pytest.mark.parametrize("S", [100, 700], ids=["merged", "split"])
def test_a_poisoned_key_block_shows_too(S):
    a = Attn(1, 4, 2, 64, 3, S, 2, n=S, seed=9, fmt=E4M3)
    a.topk[:] = [[0, 1]]
    a.buffers()
    a.cache.scales[0][0, 1, 0, 1] = float("nan")        # kv head 0 of a selected shard
    a.run()
    torch.cuda.synchronize()
    assert torch.isnan(a.y[0, :2]).all() and torch.isfinite(a.y[0, 2:]).all()


@pytest.mark.parametrize("S", [100, 700], ids=["merged", "split"])
def test_selections_of_no_shard_count_as_empty(S):
    a = Attn(2, 8, 2, 64, 3, S, 3, seed=14)
    a.topk[:] = [[2, 0, 1], [1, 2, 0]]
    a.buffers()
    a.d["topk"][0, 1], a.d["topk"][1, 2] = -1, 3
    n = a.n.copy()
    a.n[0, 0] = a.n[1, 0] = 0                            # the plain form: these shards are empty
    a.run()
    a.check()
    a.n = n


def test_a_shard_listed_twice_takes_a_new_entry_once():
    caches = [Cache(1, 3, 2, 40, 64, "f32", INT8, 16) for _ in range(2)]
    rng = np.random.default_rng(15)
    values = make_values(rng, (1, 3, 2, 40, 64), "f32")
    new = up(rng.normal(size=(1, 2, 64)) * 50)
    counts = []
    for cache, topk in zip(caches, ([[2, 0, 2]], [[2, 0, 1]])):
        n, u = i32([[20, 20, 20]]), torch.ones((1, 3, 40), device=DEV)
        cache.pack(values, n.cpu().numpy())
        pk.pikv_quant_append(cache.desc, INT8, 16, new, new, i32(topk), 3, None, None, 0, *cache.tabs, *cache.scales, u, n)
        torch.cuda.synchronize()
        counts.append(n.tolist())
    assert counts == [[[21, 20, 21]], [[21, 21, 21]]]
    for a, b in zip(caches[0].codes + caches[0].scales, caches[1].codes + caches[1].scales):
        a, b = a[0, [0, 2]], b[0, [0, 2]]
        assert ((a == b) | (a != a)).all()


def test_codes_behind_the_last_entry_and_their_scales_are_not_read():
    """Unwritten bytes are NaN codes (e4m3 0xFF), unwritten scales NaN."""
    a = Attn(2, 8, 2, 128, 3, 200, 2, fmt=E4M3, block=16, n=[[33, 0, 200], [1, 16, 48]], seed=10)
    S, D = 200, 128
    live = torch.arange(S, device=DEV) < a.d["n"][..., None]
    for t in a.cache.codes:
        t[~live[:, :, None].expand(2, 3, 2, S)] = 0xFF
    a.run()
    a.check()


def test_optional_outputs_do_not_change_the_others():
    a = Attn(2, 8, 2, 64, 4, 400, 3, seed=11)
    a.run()
    torch.cuda.synchronize()
    y = a.y.clone()
    a.y.fill_(float("nan"))
    a.scores.fill_(7.0)
    a.row_max.fill_(7.0)
    a.run(scores=False, stats=False)
    torch.cuda.synchronize()
    assert torch.equal(a.y, y) and (a.scores == 7.0).all() and (a.row_max == 7.0).all()


def test_device_tensors_of_another_kind_are_refused():
    """By both paths of the binding, before anything is launched."""
    a = Attn(1, 4, 2, 64, 3, 40, 2, seed=16)
    c, d = a.cache, a.d
    other, host = d["q"].float(), d["q"].cpu()
    bf, i = torch.zeros(4096, device=DEV, dtype=torch.bfloat16), d["n"]
    f = torch.zeros(4096, device=DEV)

    def attn(q=d["q"], tab=c.tabs[0], n=d["n"], y=a.y):
        pk.pikv_quant_attn(c.desc, c.fmt, c.block, q, tab, c.tabs[1], *c.scales, n, d["topk"], d["gates"], 2, pk.COMBINE_LSE, 0.0, y, None, None, None,
                           None, a.ws)

    def append(K_new=bf):
        pk.pikv_quant_append(c.desc, c.fmt, c.block, K_new, bf, d["topk"], 2, None, None, 0, *c.tabs, *c.scales, f, d["n"])

    def rope(w=bf, freq=f, positions=i):
        pk.pikv_norm_rope(bf, 1, 512, 4, 2, 64, w, bf, 1e-6, positions, freq, 64, False, bf, bf, bf)

    before = [t.clone() for t in c.codes + c.scales + [d["n"]]]
    for call in (lambda: attn(q=other), lambda: attn(tab=c.codes[0]), lambda: attn(n=d["n"].long()), lambda: attn(y=a.y.double()), lambda: append(f),
                 lambda: rope(w=f), lambda: rope(freq=f.double()), lambda: rope(positions=i.long())):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: attn(q=host), lambda: attn(tab=c.tabs[0].cpu()), lambda: attn(y=a.y.cpu()), lambda: attn(q=d["q"].transpose(1, 2))):
        with pytest.raises(ValueError):
            call()
    torch.cuda.synchronize()
    assert torch.isnan(a.y).all() and all(torch.equal(x.nan_to_num(), y.nan_to_num()) for x, y in zip(before, c.codes + c.scales + [d["n"]]))


def test_no_sequences_is_a_no_op():
    d = pk.make_desc(0, 4, 4, 64, 2, 32, dtype=1)
    z, i, f = torch.zeros(64, device=DEV, dtype=torch.bfloat16), torch.zeros(4, device=DEV, dtype=torch.int32), torch.ones(64, device=DEV)
    t = torch.zeros(4, device=DEV, dtype=torch.int64)
    pk.pikv_quant_pack(d, INT8, 16, t, t, 32 * 64, 64, i, t, t, f, f)
    pk.pikv_quant_read(d, INT8, 16, t, t, f, f, i, t, t, 32 * 64, 64)
    pk.pikv_quant_append(d, INT8, 16, z, z, i, 1, None, None, 0, t, t, f, f, f, i)
    pk.pikv_quant_attn(d, INT8, 16, z, t, t, f, f, i, i, None, 1, 0, 0.0, f, None, None, None, None, f)
    torch.cuda.synchronize()
    assert (f == 1).all()
