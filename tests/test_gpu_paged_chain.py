"""The operators between a prompt and a paged cache together, as a program uses them.  A prompt: norm and rotation -> route -> attention ->
utilities -> pages.  A step: norm and rotation -> route -> evict -> append -> attention over the pages -> utility.  Eager, on another stream,
and captured and replayed."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

import paged_reference as ref  # noqa: E402
import paper_2508_06526_amd as pk  # noqa: E402
from test_gpu_paged import Attention, Cache, check_fill, host, i32, up  # noqa: E402
from test_gpu_prompt import MARK, check_attention, check_mass  # noqa: E402

DEV = "cuda:0"
LENS, HQ, HKV, D, E, S, K, PAGE = [90, 41], 4, 2, 64, 4, 20, 2, 16
B, T = len(LENS), sum(LENS)
CAP, WINDOW, EPS, DECAY = 12.0, 70, 1e-6, 0.9


class Model:
    """One layer's state.  The projections' rows are drawn; everything after them is the library's."""

    def __init__(self, seed=0, dtype="bf16"):
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        t = torch.bfloat16 if dtype == "bf16" else torch.float32
        normal = lambda *s, std=1.0: (torch.randn(s, generator=gen, device=DEV) * std).to(t)
        width = (HQ + 2 * HKV) * D
        self.x, self.steps, self.x1 = normal(T, width), [normal(B, width) for _ in range(5)], torch.zeros((B, width), device=DEV, dtype=t)
        self.w = [normal(D, std=0.1) + 1 for _ in range(2)]
        self.inv_freq = (10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).float().to(DEV)
        self.W_r = normal(HQ * D, E, std=0.05)
        self.slopes = up(np.exp2(-4.0 * np.arange(1, HQ + 1) / HQ))
        zeros = lambda *s, **kw: torch.zeros(s, device=DEV, **kw)
        self.cu, self.positions = i32(np.concatenate([[0], np.cumsum(LENS)])), i32(np.concatenate([np.arange(n) for n in LENS]))
        self.q, self.k, self.v = (zeros(T, h, D, dtype=t) for h in (HQ, HKV, HKV))
        self.out, self.row_max, self.row_norm = torch.full((T, HQ, D), MARK, device=DEV, dtype=t), zeros(T, HQ), zeros(T, HQ)
        self.mass = torch.full((T,), MARK, device=DEV)
        self.mass_ws = zeros(pk.pikv_prompt_mass_workspace_bytes(T, HKV, B, max(LENS)), dtype=torch.uint8)
        self.topk, self.gates, self.slots = zeros(T, K, dtype=torch.int32), zeros(T, K), zeros(T, K, dtype=torch.int32)
        self.c = Cache(B, E, HKV, S, D, dtype, PAGE, "slots", seed=seed, Hq=HQ)
        self.n, self.table = zeros(B, E, dtype=torch.int32), i32(self.c.table)
        self.position = i32(LENS)
        self.q1, self.k1, self.v1 = (zeros(B, h, D, dtype=t) for h in (HQ, HKV, HKV))
        self.topk1, self.gates1 = zeros(B, K, dtype=torch.int32), zeros(B, K)
        self.eidx, self.ecnt = zeros(B, E, 1, dtype=torch.int32), zeros(B, E, dtype=torch.int32)
        self.y, self.max1, self.norm1 = zeros(B, HQ, D), zeros(B, HQ), zeros(B, HQ)
        self.scores, self.coef = zeros(B, HQ, K, S), zeros(B, HQ, K, 2)
        self.ws = zeros(pk.pikv_paged_attn_workspace_bytes(self.c.desc, K), dtype=torch.uint8)
        torch.cuda.synchronize()

    def prompt(self, stream=None):
        c, masks = self.c, (self.cu, B, max(LENS), None, 0.0, CAP, self.slopes, WINDOW)
        rows = (T, HQ * D, HKV * D)
        pk.pikv_norm_rope(self.x, T, (HQ + 2 * HKV) * D, HQ, HKV, D, *self.w, EPS, self.positions, self.inv_freq, D, False, self.q, self.k, self.v,
                          stream=stream)
        pk.pikv_route(self.q, self.W_r, None, T, HQ * D, E, K, self.topk, self.gates, stream=stream)
        pk.pikv_prompt_attn(self.q, self.k, self.v, *rows, HKV * D, HQ, HKV, D, *masks, self.out, self.row_max, self.row_norm, stream)
        pk.pikv_prompt_mass(self.q, self.k, *rows, HQ, HKV, D, *masks, self.row_max, self.row_norm, self.mass, self.mass_ws, stream)
        pk.pikv_paged_fill(c.desc, c.pages, self.k, self.v, T, self.cu, self.topk, K, self.mass, self.positions, *c.views, self.table, c.entry_pos,
                           c.utility, self.n, self.slots, stream)

    def step(self, stream=None):
        c, d = self.c, self.c.desc
        pk.pikv_norm_rope(self.x1, B, (HQ + 2 * HKV) * D, HQ, HKV, D, *self.w, EPS, self.position, self.inv_freq, D, False, self.q1, self.k1, self.v1,
                          stream=stream)
        pk.pikv_route(self.q1, self.W_r, None, B, HQ * D, E, K, self.topk1, self.gates1, stream=stream)
        pk.pikv_evict(d, c.utility, self.n, S - 1, self.topk1, K, self.eidx, self.ecnt, 1, False, None, None, stream=stream)
        pk.pikv_paged_append(d, c.pages, self.k1, self.v1, self.topk1, K, self.eidx, self.ecnt, 1, self.position, *c.views, self.table, c.entry_pos,
                             c.utility, self.n, stream)
        pk.pikv_paged_attn(d, c.pages, self.q1, *c.views, self.table, self.n, self.topk1, self.gates1, K, pk.COMBINE_LSE, 0.0, CAP, self.slopes, WINDOW,
                           None, c.entry_pos, self.position, self.y, self.max1, self.norm1, self.scores, self.coef, self.ws, stream)
        pk.pikv_update_utility(d, self.scores, self.coef, self.n, self.topk1, K, DECAY, c.utility, stream=stream)

    def tensors(self):
        c = self.c
        return [self.q, self.k, self.v, self.topk, self.gates, self.out, self.row_max, self.row_norm, self.mass, self.slots, *c.views, c.entry_pos, c.utility,
                self.n, self.topk1, self.gates1, self.ecnt, self.y, self.max1, self.norm1]

    def state(self):
        torch.cuda.synchronize()
        return [t.clone() for t in self.tensors()]

    def restore(self, saved):
        for t, s in zip(self.tensors(), saved):
            t.copy_(s)

    def same(self, other):
        return all(torch.equal(a, b) for a, b in zip(self.state(), other.state()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_prompt_and_steps_against_the_plain_forms(dtype):
    m = Model(dtype=dtype)
    m.prompt()
    p = m.p = ref.Prompts(LENS, HQ, HKV, D, dtype, cap=CAP, window=WINDOW)
    p.q, p.k, p.v, p.slopes = host(m.q), host(m.k), host(m.v), host(m.slopes)
    check_attention(m)
    check_mass(m)
    topk, mass = host(m.topk), host(m.mass).astype(np.float32)
    slots, n = ref.fill(host(m.cu), topk, mass, lambda b, e: S, np.zeros((B, E), np.int64), S)
    np.testing.assert_array_equal(host(m.slots), slots)
    np.testing.assert_array_equal(host(m.n), n)
    rows, pos, u = [np.zeros((B, E, HKV, S, D)) for _ in range(2)], np.zeros((B, E, S), np.int64), np.zeros((B, E, S))
    for b, t in ((b, t) for b in range(B) for t in range(int(m.cu[b]), int(m.cu[b + 1]))):
        for e, s in zip(topk[t], slots[t]):
            if s >= 0:
                rows[0][b, e, :, s], rows[1][b, e, :, s], pos[b, e, s], u[b, e, s] = p.k[t], p.v[t], t - int(m.cu[b]), mass[t]
    assert (n == S).any()                        # (else the prompt's utilities chose nothing, and no step evicts)
    for i, x in enumerate(m.steps):
        m.x1.copy_(x)
        m.step()
        topk, gates, q = host(m.topk1), host(m.gates1), host(m.q1)
        for b in range(B):
            for e in topk[b]:
                full = n[b, e] == S
                assert host(m.ecnt)[b, e] == int(full)
                s = int(np.flatnonzero(u[b, e] == u[b, e].min())[-1]) if full else int(n[b, e])
                rows[0][b, e, :, s], rows[1][b, e, :, s], pos[b, e, s], u[b, e, s] = host(m.k1)[b], host(m.v1)[b], LENS[b] + i, 0.0
                n[b, e] += not full
        np.testing.assert_array_equal(host(m.n), n)
        live = np.arange(S) < n[..., None]
        np.testing.assert_array_equal(host(m.c.entry_pos)[live], pos[live])
        for which in (0, 1):
            at = np.broadcast_to(live[:, :, None, :], (B, E, HKV, S))
            np.testing.assert_array_equal(m.c.rows(which)[at], rows[which][at])
        y, weight, got_mass = np.zeros((B, HQ, D)), np.zeros((B, HQ, D)), np.zeros((B, E, S))
        A = 0.0
        for b in range(B):
            for h in range(HQ):
                parts = []
                for g, e in zip(gates[b], topk[b]):
                    k = rows[0][b, e, h // (HQ // HKV), :n[b, e]]
                    s, _ = ref.scores(q[b, h:h + 1], k, [LENS[b] + i], pos[b, e, :n[b, e]], D ** -0.5, CAP, p.slopes[h], WINDOW)
                    A = max(A, float((np.abs(q[b, h]) @ np.abs(k).T).max()) * D ** -0.5)
                    parts.append((e, g, s[0]))
                top = max(s.max() for _, _, s in parts)
                norm = sum(g * np.exp(s - top).sum() for _, g, s in parts)
                for e, g, s in parts:
                    w, v = g * np.exp(s - top) / norm, rows[1][b, e, h // (HQ // HKV), :n[b, e]]
                    y[b, h] += w @ v
                    weight[b, h] += w @ np.abs(v)
                    got_mass[b, e, :n[b, e]] += w
        _, err = ref.error_of(A, D, 300, CAP, 40.0)
        assert (np.abs(host(m.y) - y) <= 2 * err * weight + 2.0 ** -23 * np.abs(y)).all()
        visited = np.zeros((B, E, 1), bool)
        for b in range(B):
            visited[b, topk[b]] = True
        want = np.where(live & visited, np.float32(DECAY) * u + got_mass, u)
        # (a probability has the errors of its weight, of the sum and of their quotient; HQ of them and the decayed value are added)
        bar = (3 * err + (HQ + 20) * 2.0 ** -24) * got_mass + 2.0 ** -22 * want
        got = host(m.c.utility)
        assert (np.abs(got - want)[live] <= bar[live]).all()
        u = np.where(live, got, u)               # (the next step's order is of these)
        m.position += 1


def test_on_another_stream_than_the_current_one():
    a, b = Model(seed=1), Model(seed=1)
    side = torch.cuda.Stream()
    for run in ("prompt", "step", "step"):
        for m in (a, b):
            m.x1.copy_(a.steps[0])
        getattr(a, run)()
        torch.cuda.synchronize()
        getattr(b, run)(stream=side)
        side.synchronize()
        assert a.same(b)


def test_calls_of_two_states_on_two_streams_at_once():
    a, b, want = Model(seed=2), Model(seed=3), [Model(seed=2), Model(seed=3)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for m in want:
        m.x1.copy_(m.steps[0])
        m.prompt()
        m.step()
    for m in (a, b):
        m.x1.copy_(m.steps[0])
    torch.cuda.synchronize()
    for run in ("prompt", "step"):
        for m, stream in zip((a, b), streams):
            getattr(m, run)(stream=stream)
    for stream in streams:
        stream.synchronize()
    assert a.same(want[0]) and b.same(want[1])


def test_captured_prompts_and_steps_replay_to_the_eager_bits():
    """Graphs of two states, each with its own workspaces, replayed in turn with the eager calls of twins between them."""
    states, twins, graphs = [Model(seed=4), Model(seed=5)], [Model(seed=4), Model(seed=5)], []
    for m in states:
        start = m.state()
        m.prompt()                               # (the library and its kernels are loaded)
        m.step()
        torch.cuda.synchronize()
        m.restore(start)
        pair = []
        for run in (m.prompt, m.step):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                run()
            pair.append(graph)
        graphs.append(pair)
    for m in states + twins:
        m.c.utility.fill_(-3.0)
    for at in range(3):                          # new prompts into the shards that were emptied, and steps behind each
        for m in states + twins:
            m.n.zero_()
            m.x.copy_(m.x * (1.0 + 0.5 * at))
            m.position.copy_(i32(LENS))
        for (graph, _), twin in zip(graphs, twins):
            graph.replay()
            twin.prompt()
        for x in range(3):
            for m in states + twins:
                m.x1.copy_(m.steps[x + at])
            for (_, graph), twin in zip(graphs, twins):
                graph.replay()
                twin.step()
            for m, twin in zip(states, twins):
                assert m.same(twin)
            for m in states + twins:
                m.position += 1


@pytest.mark.parametrize("weight", [True, False], ids=["weights", "first"])
def test_a_prompt_longer_than_a_block_holds(weight):
    """More than 16 tokens for every thread of a shard's block, which it then reads again in every step of its plan."""
    check_fill(Cache(1, 3, 1, 150, 32, "bf16", 16, seed=8), [17001], 2, weight=weight)


def test_calls_without_tokens_or_sequences():
    t = dict(device=DEV, dtype=torch.bfloat16)
    none = lambda *s, dtype=torch.float32: torch.zeros(s, device=DEV, dtype=dtype)
    out, mass = torch.zeros((0, HQ, D), **t), none(0)
    q, kv = torch.zeros((0, HQ * D), **t), torch.zeros((0, HKV * D), **t)
    rows = (0, HQ * D, HKV * D)
    for cu, b in ((i32([0, 0, 0]), 2), (i32([0]), 0)):
        masks = (cu, b, 5, None, 0.0, 0.0, None, 0)
        pk.pikv_prompt_attn(q, kv, kv, *rows, HKV * D, HQ, HKV, D, *masks, out)
        pk.pikv_prompt_mass(q, kv, *rows, HQ, HKV, D, *masks, none(0, HQ), none(0, HQ), mass,
                            none(max(pk.pikv_prompt_mass_workspace_bytes(0, HKV, b, 5), 1), dtype=torch.uint8))
    c = Cache(2, E, HKV, S, D, "bf16", PAGE, Hq=HQ)
    n = i32(np.full((2, E), 3))
    pk.pikv_paged_fill(c.desc, c.pages, torch.zeros((0, HKV, D), **t), torch.zeros((0, HKV, D), **t), 0, i32([0, 0, 0]), none(0, K, dtype=torch.int32), K, None,
                       None, *c.pools(), None, c.utility, n, none(0, K, dtype=torch.int32))
    assert (host(n) == 3).all() and (host(c.utility) == -3).all()
    c.untouched_elsewhere(np.zeros((2, E, S), bool))
    # sequences of a batch that have no tokens
    check_fill(Cache(4, E, HKV, S, D, "bf16", PAGE), [0, 7, 0, 0], K)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("change", [dict(), dict(slopes=True, window=50)], ids=["plain", "positions"])
@pytest.mark.parametrize("Hkv,G,tq,D,S", [(2, 2, 3, 64, 90), (1, 4, 8, 128, 400), (2, 4, 2, 32, 1100)])
def test_utilities_of_draft_queries(Hkv, G, tq, D, S, change, dtype):
    """The raw scores and slot_coef of a call with drafts, through pikv_update_utility: the attention that all rows gave."""
    a = Attention(2, 3, Hkv, G, S, D, dtype, 16, 2, tq=tq, seed=S + tq, **change)
    a.run()
    a.check()
    u = torch.full((2, 3, S), 0.5, device=DEV)
    pk.pikv_update_utility(a.c.desc, a.scores, a.coef, i32(a.n), i32(a.topk), 2, 0.25, u)
    y, top, norm, weight, raw, A = a.reference()
    _, err = ref.error_of(A, D, 300, 0.0, 40.0)
    want, got = np.full((2, 3, S), 0.5), host(u)
    for b in range(2):
        for j, e in enumerate(a.topk[b]):
            m = int(a.n[b, e])
            with np.errstate(divide="ignore", invalid="ignore"):
                p = np.where(norm[b, :, None] > 0, a.gates[b, j] * np.exp(raw[b, :, j, :m] - np.where(norm[b] > 0, top[b], 0.0)[:, None]) / norm[b, :, None], 0.0)
            want[b, e, :m] = 0.125 + p.sum(0)
    bar = (3 * err + (a.Hq + 20) * 2.0 ** -24) * np.maximum(want - 0.125, 0.0) + 2.0 ** -22 * want
    assert (np.abs(got - want) <= bar).all(), float((np.abs(got - want) / bar).max())
