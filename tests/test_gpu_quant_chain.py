"""The operators of an 8-bit cache together, as a decode step uses them: projection -> norm and rotation -> route -> evict -> insert
as codes -> attention -> utility; eager, on another stream, and captured and replayed."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

import paper_2508_06526_amd as pk  # noqa: E402
import quant_reference as ref  # noqa: E402

DEV = "cuda:0"
B, HQ, HKV, D, E, S, K, BLOCK = 3, 8, 2, 64, 4, 50, 2, 16
EPS = 1e-6


class Step:
    def __init__(self, fmt=pk.QUANT_INT8, seed=0):
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        t = torch.bfloat16
        normal = lambda *s, std=1.0: (torch.randn(s, generator=gen, device=DEV) * std).to(t)
        self.fmt = fmt
        self.steps = [normal(B, (HQ + 2 * HKV) * D) for _ in range(6)]
        self.x = torch.zeros_like(self.steps[0])
        self.w = [normal(D, std=0.1) + 1 for _ in range(2)]
        self.inv_freq = (10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).float().to(DEV)
        self.position = torch.tensor([3, 700, 90000], device=DEV, dtype=torch.int32)
        self.W_r = normal(HQ * D, E, std=0.05)
        self.q, self.k_new, self.v_new = (torch.zeros((B, h, D), device=DEV, dtype=t) for h in (HQ, HKV, HKV))
        i32 = dict(device=DEV, dtype=torch.int32)
        self.topk, self.gates = torch.zeros((B, K), **i32), torch.zeros((B, K), device=DEV)
        self.eidx, self.ecnt = torch.zeros((B, E, 1), **i32), torch.zeros((B, E), **i32)
        self.codes = [torch.zeros((B, E, HKV, S, D), device=DEV, dtype=torch.uint8) for _ in range(2)]
        self.tabs = [pk.shard_table(c) for c in self.codes]
        self.scales = [torch.zeros((B, E, HKV, -(-S // BLOCK)), device=DEV) for _ in range(2)]
        self.n = torch.tensor([[S, S - 2, 7, S], [0, S, S, S - 1], [16, 15, S, 31]], **i32)
        self.utility = torch.rand((B, E, S), generator=gen, device=DEV) + 0.1
        self.desc = pk.make_desc(B, HQ, HKV, D, E, S, dtype=pk.BF16)
        dense = [normal(B, E, HKV, S, D) for _ in range(2)]
        pk.pikv_quant_pack(self.desc, fmt, BLOCK, *[pk.shard_table(d) for d in dense], S * D, D, self.n, *self.tabs, *self.scales)
        self.y, self.row_max, self.row_norm = torch.zeros((B, HQ, D), device=DEV), torch.zeros((B, HQ), device=DEV), torch.zeros((B, HQ), device=DEV)
        self.scores, self.coef = torch.zeros((B, HQ, K, S), device=DEV), torch.zeros((B, HQ, K, 2), device=DEV)
        self.ws = torch.zeros(pk.pikv_quant_attn_workspace_bytes(self.desc, K), device=DEV, dtype=torch.uint8)
        torch.cuda.synchronize()

    def calls(self, stream=None):
        d = self.desc
        pk.pikv_norm_rope(self.x, B, (HQ + 2 * HKV) * D, HQ, HKV, D, *self.w, EPS, self.position, self.inv_freq, D, False, self.q, self.k_new,
                          self.v_new, stream=stream)
        pk.pikv_route(self.q, self.W_r, None, B, HQ * D, E, K, self.topk, self.gates, stream=stream)
        pk.pikv_evict(d, self.utility, self.n, S - 1, self.topk, K, self.eidx, self.ecnt, 1, False, None, None, stream=stream)
        pk.pikv_quant_append(d, self.fmt, BLOCK, self.k_new, self.v_new, self.topk, K, self.eidx, self.ecnt, 1, *self.tabs, *self.scales,
                             self.utility, self.n, stream=stream)
        pk.pikv_quant_attn(d, self.fmt, BLOCK, self.q, *self.tabs, *self.scales, self.n, self.topk, self.gates, K, pk.COMBINE_LSE, 0.0, self.y,
                           self.row_max, self.row_norm, self.scores, self.coef, self.ws, stream=stream)
        pk.pikv_update_utility(d, self.scores, self.coef, self.n, self.topk, K, 0.9, self.utility, stream=stream)

    def state(self):
        torch.cuda.synchronize()
        return [t.clone() for t in [self.q, self.k_new, self.v_new, self.topk, self.gates, self.ecnt, *self.codes, *self.scales, self.n, self.utility,
                                    self.y, self.row_max, self.row_norm]]

    def restore(self, saved):
        for t, s in zip([self.q, self.k_new, self.v_new, self.topk, self.gates, self.ecnt, *self.codes, *self.scales, self.n, self.utility, self.y,
                         self.row_max, self.row_norm], saved):
            t.copy_(s)


@pytest.mark.parametrize("fmt", [pk.QUANT_INT8, pk.QUANT_E4M3], ids=["int8", "e4m3"])
def test_steps_against_the_plain_forms(fmt):
    s = Step(fmt)
    host = lambda t: t.float().cpu().numpy().astype(np.float64)
    for x in s.steps:
        s.x.copy_(x)
        codes, scales = [c.cpu().numpy().copy() for c in s.codes], [a.cpu().numpy().copy() for a in s.scales]
        n, u = s.n.cpu().numpy().copy(), s.utility.cpu().numpy().astype(np.float64)
        s.calls()
        torch.cuda.synchronize()
        heads = host(x).reshape(B, -1, D)
        pos, freq = s.position.cpu().numpy(), s.inv_freq.cpu().numpy()
        for got, rows, w in ((s.q, heads[:, :HQ], s.w[0]), (s.k_new, heads[:, HQ:HQ + HKV], s.w[1])):
            want = ref.norm_rope(rows, host(w), EPS, pos, freq, D, False)
            # half a bf16 step, and fp32 errors of 16 roundings of a pair's values (at most 40 here: |z| <= sqrt(64) * 1.5, two of them)
            assert (np.abs(host(got) - want) <= 2.0 ** -8 * np.abs(want) + 16 * 2.0 ** -24 * 40).all()
        new = [host(s.k_new), host(s.v_new)]
        topk = s.topk.cpu().numpy()
        for b in range(B):
            for e in topk[b]:
                full = n[b, e] == S
                assert s.ecnt[b, e].item() == int(full)
                slot = int(np.flatnonzero(u[b, e] == u[b, e].min())[-1]) if full else int(n[b, e])
                before = S - 1 if full else int(n[b, e])
                for v, c, a in zip(new, codes, scales):
                    ref.append(v[b], slot, before, int(full), fmt, BLOCK, c[b, e], a[b, e], S)
                u[b, e, slot] = 0.0
                n[b, e] = before + 1
        np.testing.assert_array_equal(s.n.cpu().numpy(), n)
        for got, want, gs, ws in zip(s.codes, codes, s.scales, scales):
            np.testing.assert_array_equal(gs.cpu().numpy(), ws)
            np.testing.assert_array_equal(ref.decode(got.cpu().numpy(), fmt), ref.decode(want, fmt))
        K, V = (ref.values(c, a, fmt, BLOCK) for c, a in zip(codes, scales))
        want = ref.attend(host(s.q), K, V, n, topk, s.gates.cpu().numpy(), HKV)
        # scores of at most 8 * 1.5 * 12: 72 * 2^-24 * 150 off each, twice in a weight
        assert np.abs(s.y.cpu().numpy() - want["y"]).max() <= 4 * 72 * 2.0 ** -24 * 150 * np.abs(V).max()
        visited = np.zeros((B, E, 1), bool)
        for b in range(B):
            visited[b, topk[b]] = True
        live = (np.arange(S) < n[..., None]) & visited
        np.testing.assert_allclose(s.utility.cpu().numpy(), np.where(live, 0.9 * u + want["mass"], u), rtol=2e-3, atol=1e-9)


def test_on_another_stream_than_the_current_one():
    a, b = Step(seed=1), Step(seed=1)
    side = torch.cuda.Stream()
    for x in a.steps[:3]:
        a.x.copy_(x)
        b.x.copy_(x)
        a.calls()
        torch.cuda.synchronize()
        b.calls(stream=side)
        side.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(a.state(), b.state()))


def test_the_calls_through_ctypes_give_the_same_bits(monkeypatch):
    a, b = Step(pk.QUANT_E4M3, seed=5), Step(pk.QUANT_E4M3, seed=5)
    for x in a.steps[:3]:
        a.x.copy_(x)
        b.x.copy_(x)
        a.calls()
        with monkeypatch.context() as m:
            m.setattr(pk.binding, "_native", pk.binding._NoExtension())
            b.calls()
        assert all(torch.equal(u, v) for u, v in zip(a.state(), b.state()))


def test_two_captured_steps_replay_to_the_eager_bits():
    """Two graphs of two states, each with its own workspace, replayed in turn between eager steps of a third."""
    states, graphs = [Step(seed=2), Step(seed=3)], []
    for s in states:
        start = s.state()
        s.calls()                                          # (the library and its kernels are loaded)
        torch.cuda.synchronize()
        s.restore(start)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.calls()
        graphs.append(graph)
        s.restore(start)
    eager = [Step(seed=2), Step(seed=3)]
    for i in range(5):
        for s, g, twin in zip(states, graphs, eager):
            s.x.copy_(s.steps[i])
            g.replay()
            twin.x.copy_(twin.steps[i])
            twin.calls()
        for s, twin in zip(states, eager):
            assert all(torch.equal(u, v) for u, v in zip(s.state(), twin.state())), i
