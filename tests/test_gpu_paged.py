"""The paged cache: written by prompts and by single tokens, attended over - against the plain 64-bit forms; bars from
tests/paged_reference.py."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

import paged_reference as ref  # noqa: E402
import paper_2508_06526_amd as pk  # noqa: E402

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def up(a, dtype="f32"):
    return torch.from_numpy(np.array(a, np.float32)).to(DEV).to(DTYPES[dtype])


def i32(a):
    return None if a is None else torch.from_numpy(np.array(a, np.int32)).to(DEV)


def host(t):
    torch.cuda.synchronize()
    return t.float().cpu().numpy().astype(np.float64) if t.is_floating_point() else t.cpu().numpy()


class Cache:
    """Pages in random places of pools that hold `fill` elsewhere.  layout: "heads" [page, head, slot, D], "slots" [page, slot, head, D], or
    "both" (one pool [page, K or V, head, slot, D]); pad: elements between rows."""

    def __init__(self, B, E, Hkv, S, D, dtype, page, layout="heads", pad=0, fill=5.0, seed=0, **desc):
        self.shape, self.dtype, self.page, self.fill = (B, E, Hkv, S, D), dtype, page, fill
        rng = np.random.default_rng(seed)
        self.per = -(-S // page)
        self.n_pages = B * E * self.per + 4
        self.table = rng.permutation(self.n_pages)[:B * E * self.per].reshape(B, E, self.per).astype(np.int32)
        w = D + pad
        full = lambda *s: torch.full(s, fill, device=DEV, dtype=DTYPES[dtype])
        if layout == "heads":
            views = [full(self.n_pages, Hkv, page, w)[..., :D] for _ in range(2)]
        elif layout == "slots":
            views = [full(self.n_pages, page, Hkv, w)[..., :D].transpose(1, 2) for _ in range(2)]
        else:
            whole = full(self.n_pages, 2, Hkv, page, w)
            views = [whole[:, i, :, :, :D] for i in range(2)]
        self.views = views                       # [n_pages, Hkv, page, D]
        self.pages = pk.make_pages(self.n_pages, page, Hkv, D, *views[0].stride()[:3])
        self.entry_pos = torch.full((B, E, S), -7, device=DEV, dtype=torch.int32)
        self.utility = torch.full((B, E, S), -3.0, device=DEV)
        self.desc = pk.make_desc(**dict(dict(B=B, Hq=Hkv, Hkv=Hkv, D=D, E=E, S=S, dtype=int(dtype == "bf16")), **desc))

    def pools(self):
        return (*self.views, i32(self.table))

    def rows(self, which):
        """[B, E, Hkv, S, D] of the pool as float64; pages that are missing read as `fill`."""
        B, E, Hkv, S, D = self.shape
        pool = host(self.views[which])
        out = np.full((B, E, Hkv, S, D), self.fill)
        for s in range(S):
            at = self.table[:, :, s // self.page]
            good = (at >= 0) & (at < self.n_pages)
            out[good, :, s] = pool[at[good], :, s % self.page]
        return out

    def set(self, K, V):
        B, E, Hkv, S, D = self.shape
        for view, rows in zip(self.views, (K, V)):
            a = host(view)
            for s in range(S):
                at = self.table[:, :, s // self.page]
                good = (at >= 0) & (at < self.n_pages)
                a[at[good], :, s % self.page] = rows[good, :, s]
            view.copy_(up(a, self.dtype))

    def untouched_elsewhere(self, written):
        """Everything in both pools but the slots written[B, E, S] holds `fill`."""
        for view in self.views:
            a = host(view)
            for (b, e, s) in np.argwhere(written):
                a[self.table[b, e, s // self.page], :, s % self.page] = self.fill
            assert (a == self.fill).all()


def check_fill(c, lens, k, seed=0, weight=True, n0=None, positions=True, lead=0, tail=0, twice=False, stream=None, weights=None):
    B, E, Hkv, S, D = c.shape
    rng = np.random.default_rng(seed)
    cu = lead + np.concatenate([[0], np.cumsum(lens)])
    T = int(cu[-1]) + tail
    K, V = (ref.stored(rng.normal(size=(T, Hkv, D)), c.dtype) for _ in range(2))
    topk = np.argsort(rng.random((T, E)), 1)[:, :k].astype(np.int32)
    if twice:
        topk[::3, -1] = topk[::3, 0]
        topk[1::4, 0] = rng.choice([-1, E, 1 << 30], topk[1::4, 0].shape)
    w = None
    if weight:
        w = (np.round(np.exp(rng.normal(size=T)) * 8) / 8).astype(np.float32) if weights is None else weights(rng, T)
    pos = rng.integers(0, 1 << 20, T)
    n0 = np.zeros((B, E), np.int32) if n0 is None else np.asarray(n0, np.int32)

    def room_of(b, e):
        missing = np.flatnonzero((c.table[b, e] < 0) | (c.table[b, e] >= c.n_pages))
        missing = missing[missing >= n0[b, e] // c.page]
        return missing[0] * c.page if len(missing) else S
    want, counts = ref.fill(cu, topk, w, room_of, n0, S)
    n = i32(n0)
    slots = torch.full((T, k), -9, device=DEV, dtype=torch.int32)
    pk.pikv_paged_fill(c.desc, c.pages, up(K, c.dtype), up(V, c.dtype), T, i32(cu), i32(topk), k, None if w is None else up(w),
                       i32(pos) if positions else None, *c.pools(), c.entry_pos if positions else None, c.utility, n, slots, stream)
    got = host(slots)
    inside = (np.arange(T) >= cu[0]) & (np.arange(T) < cu[-1])
    assert (got[~inside] == -9).all()
    np.testing.assert_array_equal(got[inside], want[inside])
    np.testing.assert_array_equal(host(n), counts)
    utility, entry, written = np.full((B, E, S), -3.0), np.full((B, E, S), -7), np.zeros((B, E, S), bool)
    rows = [c.rows(0), c.rows(1)]
    for t in range(cu[0], cu[-1]):
        b = int(np.searchsorted(cu[1:], t, side="right"))
        for j in range(k):
            if want[t, j] >= 0:
                at = (b, topk[t, j], want[t, j])
                written[at] = True
                utility[at], entry[at] = (0.0 if w is None else w[t]), pos[t] if positions else -7
                np.testing.assert_array_equal(rows[0][at[0], at[1], :, at[2]], K[t])
                np.testing.assert_array_equal(rows[1][at[0], at[1], :, at[2]], V[t])
    np.testing.assert_array_equal(host(c.utility), utility)
    np.testing.assert_array_equal(host(c.entry_pos), entry)
    c.untouched_elsewhere(written)
    return want


FILLS = [  # B, E, Hkv, S, D, page, lens, k
    (1, 1, 1, 1, 64, 16, [1], 1), (2, 3, 2, 40, 32, 16, [50, 9], 2), (3, 4, 3, 33, 128, 32, [0, 100, 1], 3), (1, 8, 8, 300, 64, 64, [700], 2),
    (2, 64, 1, 20, 32, 16, [129, 64], 5), (1, 2, 1, 5000, 32, 256, [4500], 1), (4, 2, 16, 70, 128, 128, [64, 65, 63, 2], 2)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("weight", [True, False], ids=["weights", "first"])
@pytest.mark.parametrize("layout", ["heads", "slots", "both"])
@pytest.mark.parametrize("geo", FILLS, ids=lambda g: "B%d_E%d_H%d_S%d_D%d_p%d" % g[:6])
def test_prompts_go_into_pages(geo, layout, weight, dtype):
    B, E, Hkv, S, D, page, lens, k = geo
    check_fill(Cache(B, E, Hkv, S, D, dtype, page, layout, pad=8 if layout != "both" else 0), lens, k, weight=weight)


def test_what_is_there_stays_and_counts_against_the_room():
    c = Cache(2, 3, 2, 40, 32, "bf16", 16)
    check_fill(c, [60, 25], 2, n0=[[5, 40, 39], [0, -1, 16]])
    c = Cache(2, 3, 2, 40, 32, "bf16", 16)
    check_fill(c, [60, 25], 2, n0=[[5, 40, 39], [41, 1000, 16]], positions=False, weight=False)


def test_missing_pages_end_a_shard():
    c = Cache(2, 3, 2, 100, 64, "f32", 16)
    c.table[0, 0, 2] = -1
    c.table[0, 1, 0] = c.n_pages
    c.table[1, 2, 6] = 1 << 30
    c.table[1, 0, 0] = -5                    # behind what it holds already
    check_fill(c, [150, 140], 2, n0=[[0, 0, 0], [20, 0, 0]])


def test_tokens_outside_the_sequences_shards_listed_twice_and_shards_that_are_none():
    check_fill(Cache(2, 4, 2, 60, 64, "bf16", 16), [70, 90], 3, lead=11, tail=5, twice=True)


@pytest.mark.parametrize("weights", [
    lambda rng, T: np.where(rng.random(T) < 0.3, np.nan, np.where(rng.random(T) < 0.3, -np.inf, rng.normal(size=T))).astype(np.float32),
    lambda rng, T: np.where(rng.random(T) < 0.5, np.float32(0.0), np.float32(-0.0)).astype(np.float32),
    lambda rng, T: rng.choice([1e-45, -1e-45, 3e38, np.inf, 1e-38], T).astype(np.float32),
    lambda rng, T: np.float32(1.0) + np.arange(T, dtype=np.float32) * np.float32(2.0 ** -23)], ids=["nan", "zeros", "ends", "neighbours"])
def test_weights_at_the_ends_of_their_type(weights):
    check_fill(Cache(1, 2, 1, 37, 32, "f32", 16), [200], 1, weights=weights)
    check_fill(Cache(1, 2, 1, 1, 32, "f32", 16), [200], 1, weights=weights)


def test_a_long_prompt_over_few_slots():
    check_fill(Cache(1, 4, 1, 301, 32, "bf16", 64), [20000], 2)


def test_append_follows_the_dense_call():
    """The same slots, counts and utilities as pikv_append; rows and positions in their pages."""
    B, E, Hkv, S, D, k = 3, 4, 2, 37, 64, 2
    rng = np.random.default_rng(3)
    c = Cache(B, E, Hkv, S, D, "bf16", 16)
    n0 = rng.integers(0, S + 1, (B, E)).astype(np.int32)
    n0[0, 0], n0[1, 1], n0[2, 2] = S, 0, S - 1
    topk = np.argsort(rng.random((B, E)), 1)[:, :k].astype(np.int32)
    cnt = rng.integers(0, 2, (B, E)).astype(np.int32)
    n0[cnt > 0] = np.minimum(n0[cnt > 0], S - 1)
    idx = rng.integers(0, S, (B, E, 1)).astype(np.int32)
    new = [ref.stored(rng.normal(size=(B, Hkv, D)), "bf16") for _ in range(2)]
    for reuse in (True, False):
        c = Cache(B, E, Hkv, S, D, "bf16", 16)
        dense = [torch.full((B, E, Hkv, S, D), 5.0, device=DEV, dtype=torch.bfloat16) for _ in range(2)]
        n, m, util = i32(n0), i32(n0), torch.full((B, E, S), -3.0, device=DEV)
        freed = (i32(idx), i32(cnt), 1) if reuse else (None, None, 0)
        pk.pikv_append(c.desc, up(new[0], "bf16"), up(new[1], "bf16"), i32(topk), k, *freed, *(pk.shard_table(d) for d in dense), util, m)
        pk.pikv_paged_append(c.desc, c.pages, up(new[0], "bf16"), up(new[1], "bf16"), i32(topk), k, *freed, i32([11, 12, 13]), *c.pools(), c.entry_pos,
                             c.utility, n)
        assert torch.equal(n, m) and torch.equal(c.utility, util)
        for which in range(2):
            np.testing.assert_array_equal(c.rows(which), host(dense[which]))
        pos = host(c.entry_pos)
        written = host(util) == 0.0
        assert (pos[~written] == -7).all() and all((pos[b][written[b]] == 11 + b).all() for b in range(B))


def test_append_without_a_page_without_a_shard_and_twice():
    c = Cache(1, 4, 2, 40, 32, "f32", 16)
    c.table[0, 1, 0], c.table[0, 2, 1] = -1, c.n_pages
    n = i32([[3, 3, 16, -1]])
    new = up(np.ones((1, 2, 32)))
    pk.pikv_paged_append(c.desc, c.pages, new, new, i32([[1, 2, 3, 0]]), 4, None, None, 0, None, *c.pools(), None, c.utility, n)
    assert host(n).tolist() == [[4, 3, 16, -1]]
    pk.pikv_paged_append(c.desc, c.pages, new, new, i32([[0, 0, -1, 4]]), 4, None, None, 0, None, *c.pools(), None, c.utility, n)
    assert host(n).tolist() == [[5, 3, 16, -1]]
    written = np.zeros((1, 4, 40), bool)
    written[0, 0, 3:5] = True
    c.untouched_elsewhere(written)
    assert (host(c.entry_pos) == -7).all()


class Attention:
    """A call over a cache of random rows, with its 64-bit reference."""

    def __init__(self, B, E, Hkv, G, S, D, dtype, page, k, tq=1, per_head=False, layout="heads", pad=0, seed=0, std=1.5, cap=0.0, slopes=False, window=0,
                 prefix=False, positions=False, local=False, gates=True, scale=0.0, full=False):
        rng = np.random.default_rng(seed)
        self.geo = (B, E, Hkv, S, D)
        self.Hq, self.tq, self.k, self.per_head, self.local, self.scale = Hkv * G * tq, tq, k, per_head, local, scale
        self.cap, self.window = cap, window
        self.c = Cache(B, E, Hkv, S, D, dtype, page, layout, pad, fill=float("nan"), seed=seed, Hq=self.Hq, tq=tq, route_rows_per_seq=self.Hq if per_head else 1)
        self.n = rng.integers(0, S + 1, (B, E)).astype(np.int32)
        self.n[0, 0] = S
        if full:
            self.n[:] = S
        elif E > 1:
            self.n[0, 1] = 0
            self.n[-1, 0] = min(1, S)
        self.K, self.V = (ref.stored(rng.normal(size=(B, E, Hkv, S, D)), dtype) for _ in range(2))
        live = np.arange(S) < self.n[..., None]
        for a in (self.K, self.V):               # what lies behind the last entry is not read
            a[~np.broadcast_to(live[:, :, None, :], a.shape[:4])] = np.nan
        self.q = ref.stored(rng.normal(size=(B, self.Hq, D)) * std, dtype)
        rows = B * (self.Hq if per_head else 1)
        self.topk = np.argsort(rng.random((rows, E)), 1)[:, :k].astype(np.int32)
        self.gates = np.exp(rng.normal(size=(rows, k))).astype(np.float32) if gates else None
        self.positioned = positions or slopes or window > 0 or prefix
        self.pos = rng.integers(0, 2 * S + 3, (B, E, S)).astype(np.int32)
        self.q_pos = (rng.integers(S, 2 * S + 2, (B, 1)) + np.arange(tq)).astype(np.int32)
        self.slopes = np.exp2(-4.0 * np.arange(1, self.Hq // tq + 1) / (self.Hq // tq)).astype(np.float32) if slopes else None
        self.prefix = np.array([S // 2 if b % 3 == 0 else -1 if b % 3 == 1 else 2 * S for b in range(B)], np.int32) if prefix else None

    def run(self, scores=True, stream=None, mark=7.0):
        c, (B, E, Hkv, S, D), k = self.c, self.geo, self.k
        c.set(self.K, self.V)
        full = lambda *s: torch.full(s, mark, device=DEV)
        self.y, self.row_max, self.row_norm = full(B, self.Hq, D), full(B, self.Hq), full(B, self.Hq)
        self.scores = full(B, self.Hq, k, S) if scores else None
        self.coef = full(B, self.Hq, k, 2)
        self.ws = torch.full((pk.pikv_paged_attn_workspace_bytes(c.desc, k),), 0xff, device=DEV, dtype=torch.uint8)
        self.args = (c.desc, c.pages, up(self.q, c.dtype), *c.pools(), i32(self.n), i32(self.topk), None if self.gates is None else up(self.gates), k,
                     pk.COMBINE_LOCAL if self.local else pk.COMBINE_LSE, self.scale, self.cap, None if self.slopes is None else up(self.slopes), self.window,
                     i32(self.prefix), i32(self.pos) if self.positioned else None, i32(self.q_pos) if self.positioned else None, self.y, self.row_max,
                     self.row_norm, self.scores, self.coef, self.ws)
        pk.pikv_paged_attn(*self.args, stream=stream)

    def reference(self):
        B, E, Hkv, S, D = self.geo
        heads, c = self.Hq // self.tq, self.c
        scale = self.scale if self.scale > 0 else D ** -0.5
        y, top, norm, weight = np.zeros((B, self.Hq, D)), np.full((B, self.Hq), -np.inf), np.zeros((B, self.Hq)), np.zeros((B, self.Hq, D))
        raw = np.full((B, self.Hq, self.k, S), np.nan)
        A = 0.0
        for b in range(B):
            for row in range(self.Hq):
                t, h = divmod(row, heads)
                hk = h // (heads // Hkv)
                r = b * self.Hq + row if self.per_head else b
                parts = []
                for j, e in enumerate(self.topk[r]):
                    m = min(max(int(self.n[b, e]), 0), S) if 0 <= e < E else 0
                    if m == 0:
                        continue
                    there = np.repeat((c.table[b, e] >= 0) & (c.table[b, e] < c.n_pages), c.page)[:m]
                    k = np.where(there[:, None], self.K[b, e, hk, :m], 0.0)
                    v = np.where(there[:, None], self.V[b, e, hk, :m], 0.0)
                    s, seen = ref.scores(self.q[b, row:row + 1], k, self.q_pos[b, t:t + 1], self.pos[b, e, :m], scale, self.cap,
                                         0.0 if self.slopes is None else self.slopes[h], self.window, 0 if self.prefix is None else int(self.prefix[b]),
                                         self.positioned)
                    s, seen = np.where(there, s[0], -np.inf), there & seen[0]
                    A = max(A, float((np.abs(self.q[b, row]) @ np.abs(k[np.isfinite(k).all(1)]).T).max(initial=0.0)) * scale)
                    raw[b, row, j, :m] = s
                    if seen.any():
                        parts.append((1.0 if self.gates is None else float(self.gates[r, j]), s, np.where(seen[:, None], v, 0.0)))
                if not parts:
                    continue
                top[b, row] = max(s.max() for _, s, _ in parts)
                if self.local:
                    norm[b, row] = sum(g for g, _, _ in parts)
                    w = [g / norm[b, row] * np.exp(s - s.max()) / np.exp(s - s.max()).sum() for g, s, _ in parts]
                else:
                    w = [g * np.exp(s - top[b, row]) for g, s, _ in parts]
                    norm[b, row] = sum(x.sum() for x in w)
                    w = [x / norm[b, row] for x in w]
                with np.errstate(invalid="ignore"):
                    for x, (_, _, v) in zip(w, parts):
                        y[b, row] += x @ v
                        weight[b, row] += x @ np.abs(v)
        return y, top, norm, weight, raw, A

    def check(self):
        B, E, Hkv, S, D = self.geo
        y, top, norm, weight, raw, A = self.reference()
        bias = 0.0 if self.slopes is None else min(40.0, float(self.slopes.max()) * 3 * S)
        ds, e = ref.error_of(A, D, 300, self.cap, bias)
        got = host(self.y)
        assert (np.abs(got - y) <= 2 * e * weight + 2.0 ** -23 * np.abs(y) + 2.0 ** -120).all(), float((np.abs(got - y) / (2 * e * weight + 1e-30)).max())
        fine = np.isfinite(top)
        np.testing.assert_array_equal(host(self.row_max)[~fine], top[~fine])
        assert (np.abs(host(self.row_max) - top)[fine] <= ds + 2.0 ** -23 * np.abs(top[fine])).all()
        assert (np.abs(host(self.row_norm) - norm) <= e * norm).all()
        if self.scores is not None and self.tq == 1:
            s = host(self.scores)
            live = ~np.isnan(raw)
            assert (s[~live] == 7.0).all()
            hidden = live & np.isneginf(raw)
            assert np.isneginf(s[hidden]).all()
            seen = live & ~hidden
            assert (np.abs(s - raw)[seen] <= ds + 2.0 ** -23 * np.abs(raw[seen])).all()
            # and the probabilities that the utility update makes of them
            coef = host(self.coef)
            with np.errstate(invalid="ignore"):
                p = np.where(live, coef[..., 1:] * np.exp(s - coef[..., :1]), 0.0)
            total = p.sum((2, 3))
            assert (np.abs(total[norm > 0] - 1.0) <= 3 * e + 2.0 ** -20).all() and (total[norm == 0] == 0).all()


GEOMETRIES = [  # B, E, Hkv, G, S, D, page, k
    (1, 1, 1, 1, 1, 64, 16, 1), (2, 3, 2, 4, 100, 128, 16, 2), (1, 4, 2, 3, 333, 32, 32, 3), (3, 2, 4, 1, 129, 64, 64, 1), (1, 4, 1, 16, 700, 128, 256, 4),
    (2, 2, 1, 20, 300, 64, 128, 2), (1, 2, 2, 33, 1100, 128, 16, 2), (1, 16, 8, 2, 40, 32, 16, 10), (30, 2, 8, 1, 500, 32, 64, 2)]
CHANGES = [dict(), dict(cap=10.0, std=5.0), dict(slopes=True), dict(window=60), dict(prefix=True, window=9), dict(cap=3.0, std=6.0, slopes=True, prefix=True),
           dict(positions=True)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("change", CHANGES, ids=lambda m: "_".join(m) or "plain")
@pytest.mark.parametrize("geo", GEOMETRIES, ids=lambda g: "B%d_E%d_H%d_G%d_S%d_D%d_p%d_k%d" % g)
def test_attention_over_pages(geo, change, dtype):
    B, E, Hkv, G, S, D, page, k = geo
    a = Attention(B, E, Hkv, G, S, D, dtype, page, k, seed=S, local=bool(G % 2), **change)
    a.run()
    a.check()
    y = a.y.clone()
    a.run(scores=False)
    assert torch.equal(y, a.y)


@pytest.mark.parametrize("layout,pad", [("slots", 0), ("slots", 8), ("both", 0), ("heads", 16)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layouts(layout, pad, dtype):
    a = Attention(2, 3, 2, 4, 150, 64, dtype, 32, 2, layout=layout, pad=pad, seed=1, window=100)
    a.run()
    a.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("change", [dict(), dict(slopes=True, window=50), dict(cap=4.0, std=5.0, prefix=True)], ids=lambda m: "_".join(m) or "plain")
@pytest.mark.parametrize("Hkv,G,tq,D,S", [(2, 2, 3, 64, 90), (1, 4, 8, 128, 400), (2, 1, 2, 32, 33), (1, 8, 5, 64, 260)])
def test_draft_queries(Hkv, G, tq, D, S, change, dtype):
    a = Attention(2, 4, Hkv, G, S, D, dtype, 16, 2, tq=tq, seed=2, **change)
    a.run()
    a.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("change", [dict(), dict(slopes=True, window=50)], ids=["plain", "positions"])
def test_routing_per_head(change, dtype):
    for G, S, D in ((3, 120, 64), (1, 1000, 128)):
        a = Attention(2, 5, 2, G, S, D, dtype, 32, 3, per_head=True, seed=3, **change)
        a.run()
        a.check()


def test_indices_that_are_no_shard_missing_pages_no_gates_and_a_scale():
    a = Attention(2, 4, 2, 4, 200, 128, "bf16", 16, 3, seed=4, gates=False, scale=0.4)
    a.topk[0, 1], a.topk[1, 0] = 77, -3
    a.c.table[0, a.topk[0, 0], 2], a.c.table[1, a.topk[1, 1], 0] = -1, a.c.n_pages
    a.n[0, a.topk[0, 0]] = 190
    a.n[1, a.topk[1, 1]] = 100
    for x in (a.K, a.V):
        x[np.isnan(x)] = 1.0
    a.run()
    a.check()
    for x in (a.n,):
        x[0, 0], x[1, 2] = 100000, -4            # counts beyond the shard
    a.run()
    a.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tq,D,S", [(1, 64, 100), (1, 128, 700), (3, 32, 90), (2, 128, 600)])
def test_what_is_not_seen_may_hold_anything(tq, D, S, dtype):
    for bad in (np.nan, np.inf, -np.inf):
        make = lambda: Attention(1, 2, 1, 2, S, D, dtype, 16, 2, tq=tq, seed=5, window=S // 2, full=True)
        a = make()
        a.run()
        want = a.y.clone()
        a = make()
        hidden = (a.pos[0, 0] > a.q_pos.max()) | (a.pos[0, 0] <= a.q_pos.min() - S // 2)
        at = np.flatnonzero(hidden)[:3]
        a.K[0, 0, 0, at], a.V[0, 0, 0, at] = bad, bad
        a.run()
        assert torch.equal(a.y, want)
        # seen by the last query alone, if there are several
        a = make()
        a.pos[0, 1, 7] = a.q_pos.max()
        a.run()
        want = host(a.y)
        a.V[0, 1, 0, 7, 5] = bad
        a.run()
        got = host(a.y)
        last = slice(2 * (tq - 1), 2 * tq)
        changed = got[0, last, 5].copy()
        assert (np.isnan(changed) if np.isnan(bad) else changed == bad).all()
        got[0, last, 5] = want[0, last, 5]
        np.testing.assert_array_equal(got, want)


def test_rows_that_see_nothing():
    a = Attention(2, 3, 2, 2, 80, 64, "bf16", 16, 2, seed=6, positions=True)
    a.pos[0] = -1
    a.q_pos[1] = -4
    a.run()
    assert (host(a.y) == 0).all() and np.isneginf(host(a.row_max)).all() and (host(a.row_norm) == 0).all() and (host(a.coef)[..., 1] == 0).all()
    a.check()
    a = Attention(1, 3, 2, 2, 80, 64, "f32", 16, 3, seed=6, positions=True, local=True)
    a.pos[0, 1:] = 2 ** 31 - 1
    a.n[:] = 80
    a.K[np.isnan(a.K)] = a.V[np.isnan(a.V)] = 1.0
    a.run()
    a.check()


def test_pages_far_apart():
    """Offsets beyond 32 bits, in elements and in bytes."""
    Hkv, D, page, S, n_pages = 2, 128, 16, 60, 4
    stride = (1 << 30) + 64
    pool = torch.zeros((3 * stride + Hkv * page * D + 8,), device=DEV, dtype=torch.bfloat16)
    rng = np.random.default_rng(7)
    pages_all = pk.make_pages(3, page, Hkv, D, stride_page=stride)
    desc = pk.make_desc(1, Hkv, Hkv, D, 1, 48, dtype=pk.BF16)
    K, V = (ref.stored(rng.normal(size=(40, Hkv, D)), "bf16") for _ in range(2))
    n, util, slots = i32([[0]]), torch.zeros((1, 1, 48), device=DEV), torch.zeros((40, 1), device=DEV, dtype=torch.int32)
    table = i32([[[2, 0, 1]]])
    pool2 = torch.zeros_like(pool)
    pk.pikv_paged_fill(desc, pages_all, up(K, "bf16"), up(V, "bf16"), 40, i32([0, 40]), torch.zeros((40, 1), device=DEV, dtype=torch.int32), 1, None, None,
                       pool, pool2, table, None, util, n, slots)
    at = lambda p, s: p[[2, 0, 1][s // 16] * stride:][:Hkv * page * D].view(Hkv, page, D)[:, s % 16]
    for s in (0, 15, 16, 39):
        np.testing.assert_array_equal(host(at(pool, s)), K[s])
        np.testing.assert_array_equal(host(at(pool2, s)), V[s])
    q = ref.stored(rng.normal(size=(1, Hkv, D)), "bf16")
    y = torch.zeros((1, Hkv, D), device=DEV)
    ws = torch.zeros(pk.pikv_paged_attn_workspace_bytes(desc, 1), device=DEV, dtype=torch.uint8)
    pk.pikv_paged_attn(desc, pages_all, up(q, "bf16"), pool, pool2, table, n, i32([[0]]), None, 1, pk.COMBINE_LSE, 0.0, 0.0, None, 0, None, None, None, y, None,
                       None, None, None, ws)
    got = host(y)
    for h in range(Hkv):
        s, _ = ref.scores(q[0, h:h + 1], K[:, h], [0], np.zeros(40), D ** -0.5, positioned=False)
        want, _, _, weight = ref.attention(s, V[:, h])
        _, e = ref.error_of(float((np.abs(q[0, h]) @ np.abs(K[:, h]).T).max()) * D ** -0.5, D, 100)
        assert (np.abs(got[0, h] - want[0]) <= 2 * e * weight[0] + 2.0 ** -23 * np.abs(want[0])).all()


def test_extension_and_ctypes_make_the_same_calls(monkeypatch):
    def all_of(layout):
        c = Cache(2, 4, 2, 60, 64, "bf16", 16, layout)
        check_fill(c, [70, 90], 3)
        a = Attention(2, 3, 2, 4, 100, 128, "bf16", 16, 2, seed=8, cap=5.0, slopes=True, window=30, prefix=True, layout=layout)
        a.run()
        return a.y
    native = all_of("heads")
    assert torch.equal(native, all_of("both"))   # (pools that are parts of another take the general path)
    monkeypatch.setattr(pk.binding, "_native", pk.binding._NoExtension())
    assert torch.equal(native, all_of("heads"))


def test_on_a_stream_and_replayed_from_a_graph():
    a = Attention(2, 4, 2, 4, 900, 128, "bf16", 32, 3, seed=9, slopes=True)
    a.run()
    want = a.y.clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    a.y.zero_()
    side.wait_stream(torch.cuda.current_stream())
    pk.pikv_paged_attn(*a.args, stream=side)
    side.synchronize()
    assert torch.equal(a.y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pk.pikv_paged_attn(*a.args)
    for seed in (10, 11, 12):
        q = up(ref.stored(np.random.default_rng(seed).normal(size=a.q.shape), "bf16"), "bf16")
        a.args[2].copy_(q)
        graph.replay()
        torch.cuda.synchronize()
        replayed = a.y.clone()
        a.y.zero_()
        pk.pikv_paged_attn(*a.args)
        torch.cuda.synchronize()
        assert torch.equal(a.y, replayed)


def test_the_binding_refuses_what_is_too_small():
    a = Attention(2, 3, 2, 4, 100, 64, "bf16", 16, 2, seed=13, window=40)
    a.run()
    args = list(a.args)
    for at in (2, 5, 6, 7, 8, 15, 16, 17, 18, 19, 21):
        if args[at] is None:
            continue
        short = list(args)
        short[at] = args[at].flatten()[:1]
        with pytest.raises(ValueError, match="needed"):
            pk.pikv_paged_attn(*short)
    short = list(args)
    short[3] = args[3].contiguous()[:2]
    with pytest.raises(ValueError, match="pages take"):
        pk.pikv_paged_attn(*short)
    short = list(args)
    short[4] = args[4].float()
    with pytest.raises(TypeError):
        pk.pikv_paged_attn(*short)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("change", [dict(), dict(prefix=True, local=True)], ids=["plain", "prefix"])
@pytest.mark.parametrize("Hkv,G,tq,S,D", [(8, 8, 5, 13, 128), (8, 8, 5, 300, 64), (4, 16, 16, 90, 32)])
def test_more_query_rows_than_whole_shards_take(Hkv, G, tq, S, D, change, dtype):
    a = Attention(2, 3, Hkv, G, S, D, dtype, 16, 2, tq=tq, seed=S, **change)
    assert a.Hq > 256
    a.run()
    a.check()


def test_routing_of_more_heads_than_whole_shards_take():
    a = Attention(1, 4, 4, 80, 200, 64, "bf16", 16, 2, per_head=True, seed=3)
    a.run()
    a.check()
