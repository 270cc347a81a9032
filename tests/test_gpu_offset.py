"""Outputs that start at any float's address: raw scores, rows, statistics and pairs of the attention over pages, and of the 8-bit and whole shards whose
merge it shares."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

import paper_2508_06526_amd as pk  # noqa: E402
from test_gpu_paged import Attention  # noqa: E402

DEV = "cuda:0"
MARK = 7.0


class Off:
    """A tensor `by` floats into its buffer, with a margin of 8 floats behind it."""

    def __init__(self, shape, by):
        n = int(np.prod(shape))
        self.whole = torch.full((n + by + 8,), MARK, device=DEV)
        self.view = self.whole[by:by + n].view(shape)
        self.by, self.n = by, n

    def clean(self):
        return bool((self.whole[:self.by] == MARK).all() and (self.whole[self.by + self.n:] == MARK).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [0, 70], ids=["plain", "window"])
@pytest.mark.parametrize("G,S,k", [(4, 100, 2), (4, 9000, 2), (4, 103, 2), (20, 1200, 2), (2, 2048, 9)], ids=["one", "two", "odd", "tiles", "shards"])
def test_attention_over_pages(G, S, k, window, dtype):
    a = Attention(2, 10, 2, G, S, 64, dtype, 16, k, seed=1, window=window)
    a.run()
    a.check()
    want = [a.y, a.row_max, a.row_norm, a.scores, a.coef]
    for by in (1, 2, 3):
        outs = [Off(x.shape, by) for x in want]
        args = list(a.args)
        args[-6:-1] = [o.view for o in outs]
        pk.pikv_paged_attn(*args)
        torch.cuda.synchronize()
        for o, x in zip(outs, want):
            assert torch.equal(o.view, x) and o.clean()


@pytest.mark.parametrize("S", [128, 4096])
def test_attention_over_whole_shards(S):
    B, E, Hq, Hkv, D, k = 2, 4, 8, 2, 128, 2
    gen = torch.Generator(device=DEV)
    gen.manual_seed(2)
    draw = lambda *s: torch.randn(s, generator=gen, device=DEV).bfloat16()
    K, V, q = draw(B * E, Hkv, S, D), draw(B * E, Hkv, S, D), draw(B, Hq, D)
    desc = pk.make_desc(B, Hq, Hkv, D, E, S, dtype=pk.BF16)
    i32 = dict(device=DEV, dtype=torch.int32)
    n, topk = torch.full((B, E), S, **i32), torch.tensor([[0, 2], [3, 1]], **i32)
    ws = torch.empty(pk.pikv_attn_workspace_bytes(desc, k), device=DEV, dtype=torch.uint8)
    tables = pk.shard_table(list(K)), pk.shard_table(list(V))
    results = []
    for by in (0, 1, 2, 3):
        outs = [Off(s, by) for s in ((B, Hq, D), (B, Hq), (B, Hq), (B, Hq, k, S), (B, Hq, k, 2))]
        pk.pikv_sharded_attn(desc, q, *tables, None, None, n, topk, None, k, pk.COMBINE_LSE, 0.0, *[o.view for o in outs], ws)
        torch.cuda.synchronize()
        assert all(o.clean() for o in outs)
        results.append([o.view.clone() for o in outs])
    for r in results[1:]:
        assert all(torch.equal(x, y) for x, y in zip(r, results[0]))
