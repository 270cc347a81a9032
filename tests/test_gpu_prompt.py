"""Attention of packed prompts and the utilities of their entries, against the plain 64-bit forms; bars from tests/paged_reference.py."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

import paper_2508_06526_amd as pk  # noqa: E402
from paged_reference import Prompts  # noqa: E402

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
MARK = 7.0           # what outputs hold before a call


def up(a, dtype="f32"):
    return torch.from_numpy(np.array(a, np.float32)).to(DEV).to(DTYPES[dtype])


def i32(a):
    return None if a is None else torch.from_numpy(np.array(a, np.int32)).to(DEV)


class Device:
    def __init__(self, p, pad=(0, 0, 0), max_len=None, stats=True):
        self.p = p
        self.max_len = max(p.lens) if max_len is None else max_len
        self.rows = []
        for x, extra in zip((p.q, p.k, p.v), pad):
            wide = torch.full((p.tokens, x.shape[1] * p.D + extra), float("nan"), device=DEV, dtype=DTYPES[p.dtype])
            wide[:, :x.shape[1] * p.D] = up(x, p.dtype).flatten(1)
            self.rows.append((wide, wide[:, :x.shape[1] * p.D], wide.shape[1]))
        self.cu, self.prefix = i32(p.cu), i32(p.prefix)
        self.slopes = None if p.slopes is None else up(p.slopes)
        self.out = torch.full((p.tokens, p.Hq, p.D), MARK, device=DEV, dtype=DTYPES[p.dtype])
        self.row_max, self.row_norm = (torch.full((p.tokens, p.Hq), MARK, device=DEV) if stats else None for _ in range(2))
        self.mass = torch.full((p.tokens,), MARK, device=DEV)
        self.ws = torch.full((pk.pikv_prompt_mass_workspace_bytes(p.tokens, p.Hkv, len(p.lens), self.max_len),), 0xff, device=DEV, dtype=torch.uint8)

    def masks(self):
        p = self.p
        return self.cu, len(p.lens), self.max_len, self.prefix, p.scale, p.cap, self.slopes, p.window

    def attend(self, stream=None):
        p, (q, k, v) = self.p, self.rows
        pk.pikv_prompt_attn(q[1], k[1], v[1], p.tokens, q[2], k[2], v[2], p.Hq, p.Hkv, p.D, *self.masks(), self.out, self.row_max, self.row_norm, stream)

    def weigh(self, stream=None):
        p, (q, k, _) = self.p, self.rows
        pk.pikv_prompt_mass(q[1], k[1], p.tokens, q[2], k[2], p.Hq, p.Hkv, p.D, *self.masks(), self.row_max, self.row_norm, self.mass, self.ws, stream)


def host(t):
    torch.cuda.synchronize()
    return t.float().cpu().numpy().astype(np.float64)


def check_attention(d, upto=None, rows=None):
    p = d.p
    out, top, norm, weight, inside = p.attend(upto)
    ds, e = p.errors()
    bar = 2 * e * weight + 2.0 ** -24 * np.abs(out)
    if p.dtype == "bf16":
        bar += 2.0 ** -8 * weight + (1 + 2.0 ** -8) * 2.0 ** -8 * (np.abs(out) + bar) + 2.0 ** -133
    got = host(d.out)
    assert (got[~inside] == MARK).all()
    keep = inside if rows is None else inside & rows
    assert (np.abs(got - out)[keep] <= bar[keep]).all(), float((np.abs(got - out) / np.maximum(bar, 1e-300))[keep].max())
    if d.row_max is not None:
        got_max, got_norm = host(d.row_max), host(d.row_norm)
        assert (got_max[~inside] == MARK).all() and (got_norm[~inside] == MARK).all()
        assert (np.abs(got_max - top)[keep] <= ds + 2.0 ** -23 * np.abs(top[keep])).all()
        assert (np.abs(got_norm - norm)[keep] <= e * norm[keep]).all()


def check_mass(d, entries=None):
    p = d.p
    want = p.mass(host(d.row_max), host(d.row_norm))
    _, e = p.errors()
    inside = np.zeros(p.tokens, bool)
    for b, n in enumerate(p.lens):
        inside[p.cu[b]:p.cu[b] + n] = True
    got = host(d.mass)
    assert (got[~inside] == MARK).all()
    keep = inside if entries is None else inside & entries
    # (given maxima and sums: only the scores, the exponentials and sums of up to Hq n terms are the kernel's, a term is a product more)
    bar = (e + (p.Hq + 4) * 2.0 ** -24) * want + 2.0 ** -120
    assert (np.abs(got - want)[keep] <= bar[keep]).all(), float((np.abs(got - want) / bar)[keep].max())


SHAPES = [  # lens, Hq, Hkv, D
    ([1], 1, 1, 64), ([5], 4, 2, 32), ([129], 2, 2, 128), ([40, 0, 1, 77, 200], 6, 2, 64), ([257, 3], 8, 1, 128), ([64, 128], 12, 4, 32), ([300], 7, 7, 64)]
MASKS = [dict(), dict(cap=20.0, std=6.0), dict(slopes=True), dict(window=33), dict(prefix=1), dict(cap=5.0, std=8.0, slopes=True, window=70, prefix=1)]


def with_prefix(kw, lens):
    kw = dict(kw)
    if "prefix" in kw:               # none, a part, more than there is, a negative one
        kw["prefix"] = [(n // 3, 0, n + 9, -2, 2 * n // 3)[b % 5] for b, n in enumerate(lens)]
    return kw


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask", MASKS, ids=lambda m: "_".join(m) or "causal")
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "n%s_H%d_%d_D%d" % ("x".join(map(str, s[0])), *s[1:]))
def test_prompts_and_their_utilities(shape, mask, dtype):
    d = Device(Prompts(*shape, dtype, seed=3, **with_prefix(mask, shape[0])))
    d.attend()
    check_attention(d)
    d.weigh()
    check_mass(d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask", MASKS, ids=lambda m: "_".join(m) or "causal")
@pytest.mark.parametrize("shape", [([70] * 30 + [300, 129], 16, 16, 128), ([70] * 30 + [133], 24, 24, 64), ([40] * 30 + [133], 40, 40, 32), ([20, 32, 1], 6, 2, 64)],
                         ids=lambda s: "x%d_H%d_%d_D%d" % (len(s[0]), *s[1:]))
def test_enough_prompts_for_blocks_of_many_rows_and_prompts_of_a_tile(shape, mask, dtype):
    d = Device(Prompts(*shape, dtype, seed=21, **with_prefix(mask, shape[0])))
    d.attend()
    check_attention(d)
    d.weigh()
    check_mass(d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_token_gives_each_head_one_unit_of_attention(dtype):
    p = Prompts([333, 90], 8, 4, 64, dtype, seed=4)
    d = Device(p)
    d.attend()
    d.weigh()
    mass = host(d.mass)
    _, e = p.errors()
    for b, n in enumerate(p.lens):
        assert abs(mass[p.cu[b]:p.cu[b + 1]].sum() - p.Hq * n) <= 2 * e * p.Hq * n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_rows_rows_outside_the_sequences_and_a_short_max_len(dtype):
    p = Prompts([50, 140], 4, 2, 64, dtype, seed=5, lead=7, tail=9)
    outside = np.ones(p.tokens, bool)
    outside[p.cu[0]:p.cu[-1]] = False
    for x in (p.q, p.k, p.v):
        x[outside] = np.nan
    d = Device(p, pad=(16, 32, 8))
    d.attend()
    check_attention(d)
    d.weigh()
    check_mass(d)
    p.lens = [50, 140]
    short = Device(p, max_len=100)
    short.attend()
    out, top, norm, weight, inside = p.attend(100)
    assert inside.sum() == 150
    got = host(short.out)
    assert (got[~inside] == MARK).all() and np.isfinite(got[inside]).all()
    check_attention(short, 100)


def test_counts_that_leave_the_arrays_are_cut_off():
    p = Prompts([60, 30], 2, 2, 32, "bf16", seed=6)
    want = Device(p)
    want.attend()
    d = Device(p)
    d.cu = i32([0, 60, 2 ** 30])
    d.attend()
    assert torch.equal(d.out, want.out)
    d.cu = i32([-5, 60, 90])                 # the first sequence starts at row 0
    d.attend()
    assert torch.equal(d.out, want.out)
    d = Device(p)
    d.cu = i32([0, 60, 10])                  # ends before it starts: empty
    d.attend()
    torch.cuda.synchronize()
    assert torch.equal(d.out[:60], want.out[:60]) and (d.out[60:] == MARK).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("others", [0, 600], ids=["few", "many"])
def test_what_is_not_seen_may_hold_anything(others, D, dtype):
    """A token that holds NaN or infinities changes the rows that see it, and no other.  (With many short prompts beside: blocks of many rows.)"""
    fresh = lambda: Prompts([150] + [2] * others, 4, 2, D, dtype, seed=7, window=60, prefix=[4] + [0] * others)
    clean = fresh()
    ref = Device(clean)
    ref.attend()
    for bad in (np.nan, np.inf, -np.inf):
        p = fresh()
        p.v[70, 0, 3] = bad
        d = Device(p)
        d.attend()
        token = np.arange(clean.tokens)
        sees = (token >= 70) & (token - 70 < 60)
        got, want = host(d.out), host(ref.out)
        touched = np.zeros(got.shape, bool)
        touched[sees, :2, 3] = True
        np.testing.assert_array_equal(got[~touched], want[~touched])
        assert (np.isnan(got[touched]) if np.isnan(bad) else got[touched] == bad).all()
        p = fresh()
        p.k[70, 1] = bad
        d = Device(p)
        d.attend()
        got = host(d.out)
        touched = np.zeros(got.shape, bool)
        touched[sees, 2:] = True
        np.testing.assert_array_equal(got[~touched], want[~touched])
    # a query: its own rows only, and the entries it sees
    p = fresh()
    p.q[100, 1] = np.nan
    d = Device(p)
    d.attend()
    got = host(d.out)
    assert np.isnan(got[100, 1]).all()
    got[100, 1] = want[100, 1]
    np.testing.assert_array_equal(got, want)
    d.weigh()
    token = np.arange(clean.tokens)
    assert np.isnan(host(d.mass)[(token > 40) & (token <= 100)]).all()
    ref.weigh()
    rest = ~(((token > 40) & (token <= 100)) | (token < 4))
    np.testing.assert_array_equal(host(d.mass)[rest], host(ref.mass)[rest])


def test_scores_beyond_the_range_of_their_cap():
    p = Prompts([130], 4, 2, 64, "bf16", seed=8, std=60.0, cap=3.0)
    assert p.magnitude() > 100
    d = Device(p)
    d.attend()
    check_attention(d)


def test_rows_whose_sum_is_zero_give_nothing():
    p = Prompts([90], 4, 2, 64, "f32", seed=9)
    d = Device(p)
    d.attend()
    d.row_norm[10:20] = 0.0
    d.row_max[10:20] = -float("inf")
    d.weigh()
    check_mass(d)


@pytest.mark.parametrize("lens,Hq,Hkv,D", [([700], 2, 1, 64), ([1500, 40], 4, 1, 32)])
def test_few_long_prompts_are_cut_into_runs(lens, Hq, Hkv, D):
    for mask in (dict(), dict(window=100), dict(prefix=[30, 50][:len(lens)])):
        d = Device(Prompts(lens, Hq, Hkv, D, "bf16", seed=10, **mask))
        d.attend()
        check_attention(d)
        d.weigh()
        check_mass(d)
        first = d.mass.clone()
        d.weigh()
        assert torch.equal(first, d.mass)


def test_without_statistics_and_with_a_scale():
    p = Prompts([100, 20], 4, 4, 64, "bf16", seed=11, scale=0.3)
    d, plain = Device(p), Device(p, stats=False)
    d.attend()
    check_attention(d)
    plain.attend()
    assert torch.equal(d.out, plain.out)


def test_extension_and_ctypes_make_the_same_calls(monkeypatch):
    p = Prompts([77, 130], 6, 2, 64, "bf16", seed=12, cap=10.0, slopes=True, window=50, prefix=[5, 0])
    a, b = Device(p), Device(p)
    a.attend(), a.weigh()
    monkeypatch.setattr(pk.binding, "_native", pk.binding._NoExtension())
    b.attend(), b.weigh()
    assert torch.equal(a.out, b.out) and torch.equal(a.mass, b.mass) and torch.equal(a.row_norm, b.row_norm)


def test_on_a_stream_and_replayed_from_a_graph():
    p = Prompts([200, 60], 8, 2, 128, "bf16", seed=13)
    want = Device(p)
    want.attend(), want.weigh()
    torch.cuda.synchronize()
    d = Device(p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    d.attend(side), d.weigh(side)
    side.synchronize()
    assert torch.equal(d.out, want.out) and torch.equal(d.mass, want.mass)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        d.attend(), d.weigh()
    fresh = [Prompts([200, 60], 8, 2, 128, "bf16", seed=s) for s in (14, 15, 16)]
    for q in fresh:
        for x, (wide, _, _) in zip((q.q, q.k, q.v), d.rows):
            wide.copy_(up(x, "bf16").flatten(1))
        graph.replay()
        torch.cuda.synchronize()
        eager = Device(q)
        eager.attend(), eager.weigh()
        torch.cuda.synchronize()
        assert torch.equal(d.out, eager.out) and torch.equal(d.mass, eager.mass) and torch.equal(d.row_max, eager.row_max)


def test_the_binding_refuses_what_is_too_small():
    p = Prompts([40], 4, 2, 64, "bf16", seed=17)
    d = Device(p)
    for name, short in (("out", d.out[:30]), ("row_max", d.row_max[:30]), ("cu", d.cu[:1])):
        kept = getattr(d, name)
        setattr(d, name, short.contiguous())
        with pytest.raises(ValueError, match="needed"):
            d.attend()
        setattr(d, name, kept)
    d.mass = d.mass[:30]
    with pytest.raises(ValueError, match="mass"):
        d.weigh()
    d = Device(p)
    d.out = d.out.float()
    with pytest.raises(TypeError):
        d.attend()
    d = Device(p)
    d.ws = d.ws[:256]
    with pytest.raises(pk.PikvError) as e:
        d.weigh()
    assert e.value.status == -3


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_as_far_apart_as_they_may_be(dtype):
    """The largest stride, 2^25 bytes: offsets beyond 32 bits within a tile of 128 rows.  The same bits as packed rows."""
    t = DTYPES[dtype]
    Hq, Hkv, D, lens, stride = 2, 2, 64, [3, 140], (1 << 25) // (2 if dtype == "bf16" else 4)
    T = sum(lens)
    wide = torch.empty((T, stride), device=DEV, dtype=t)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(3)
    packed = [torch.randn((T, Hq * D), generator=gen, device=DEV).to(t) for _ in range(3)]
    views = [wide[:, i * 1024:i * 1024 + Hq * D] for i in range(3)]
    for v, p in zip(views, packed):
        v.copy_(p)
    cu = i32([0, 3, T])
    results = []
    for (q, k, v), step in ((packed, Hq * D), (views, stride)):
        out, mass = torch.zeros((T, Hq, D), device=DEV, dtype=t), torch.zeros(T, device=DEV)
        stats = [torch.zeros((T, Hq), device=DEV) for _ in range(2)]
        ws = torch.zeros(pk.pikv_prompt_mass_workspace_bytes(T, Hkv, 2, max(lens)), device=DEV, dtype=torch.uint8)
        masks = (cu, 2, max(lens), None, 0.0, 0.0, None, 0)
        pk.pikv_prompt_attn(q, k, v, T, step, step, step, Hq, Hkv, D, *masks, out, *stats)
        pk.pikv_prompt_mass(q, k, T, step, step, Hq, Hkv, D, *masks, *stats, mass, ws)
        torch.cuda.synchronize()
        results.append([out, mass, *stats])
    assert all(torch.equal(a, b) for a, b in zip(*results)) and float(results[0][1].min()) > 0


@pytest.mark.parametrize("lens,Hq", [([200], 2), ([300] * 12, 16)], ids=["split", "whole"])
def test_a_scale_that_leaves_nothing_of_the_scores(lens, Hq):
    d = Device(Prompts(lens, Hq, Hq, 128, "bf16", seed=4, scale=1e-38))
    d.attend()
    check_attention(d)
    assert (host(d.row_norm) >= 1).all()
    d.weigh()
    check_mass(d)
