"""A step with more query rows than whole shards have, all of it with one descriptor: evict -> append -> attention over the pages."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

import paged_reference as ref  # noqa: E402
import paper_2508_06526_amd as pk  # noqa: E402
from test_gpu_paged import DEV, Attention, host, i32, up  # noqa: E402


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_step_with_drafts_of_320_rows(dtype):
    B, E, Hkv, G, S, D, k, tq = 2, 3, 8, 8, 60, 64, 2, 5
    a = Attention(B, E, Hkv, G, S, D, dtype, 16, k, tq=tq, seed=2, positions=True, full=True)
    assert a.Hq == 320
    rng = np.random.default_rng(3)
    u = rng.random((B, E, S)).astype(np.float32)
    new = [ref.stored(rng.normal(size=(B, Hkv, D)), dtype) for _ in range(2)]
    birth, last, freq = (torch.full((B, E, S), 3, device=DEV, dtype=torch.int32) for _ in range(3))
    a.c.set(a.K, a.V)
    c, n, topk, utility, pos = a.c, i32(a.n), i32(a.topk), up(u), i32(a.pos)
    eidx, ecnt = torch.zeros((B, E, 1), device=DEV, dtype=torch.int32), torch.zeros((B, E), device=DEV, dtype=torch.int32)
    out = torch.zeros((B, E, S), device=DEV)
    pk.pikv_policy_utility(c.desc, pk.POLICY_H2O, n, 9, 0.0, 0, 0, None, None, None, utility, out)
    assert torch.equal(out, utility)
    pk.pikv_evict(c.desc, out, n, S - 1, topk, k, eidx, ecnt, 1, False, None, None)
    pk.pikv_policy_stamp(c.desc, topk, k, eidx, ecnt, 1, n, 9, birth, last, freq)
    pk.pikv_paged_append(c.desc, c.pages, up(new[0], dtype), up(new[1], dtype), topk, k, eidx, ecnt, 1, i32(a.q_pos[:, 0]), *c.pools(), pos, out, n)
    for b in range(B):
        for e in a.topk[b]:
            s = int(u[b, e].argmin())
            assert int(eidx[b, e, 0]) == s and int(ecnt[b, e]) == 1
            a.K[b, e, :, s], a.V[b, e, :, s], a.pos[b, e, s] = new[0][b], new[1][b], a.q_pos[b, 0]
            assert int(birth[b, e, s]) == 9 and int(freq[b, e, s]) == 0
    np.testing.assert_array_equal(host(n), a.n)
    np.testing.assert_array_equal(host(pos), a.pos)
    for which, rows in enumerate((a.K, a.V)):
        np.testing.assert_array_equal(c.rows(which), rows)
    a.run()
    a.check()
