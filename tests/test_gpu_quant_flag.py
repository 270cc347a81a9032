"""The descriptor flag and the marked tables of an 8-bit cache, on the device: the same bits with them as without, and refusals of
the calls on dense rows by both paths of the binding."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

import paper_2508_06526_amd as pk  # noqa: E402
from test_gpu_quant_chain import D, HKV, K, B, Step  # noqa: E402

INVALID = -1


def test_a_step_with_the_flag_and_marked_tables_gives_the_same_bits():
    plain, flagged = Step(seed=31), Step(seed=31)
    flagged.desc.flags = pk.DESC_8BIT
    flagged.tabs = [pk.shard_table(c.view(torch.int8)) for c in flagged.codes]
    for x in plain.steps[:3]:
        for s in (plain, flagged):
            s.x.copy_(x)
            s.calls()
        assert all(torch.equal(a, b) for a, b in zip(plain.state(), flagged.state()))


@pytest.mark.parametrize("native", [True, False], ids=["extension", "ctypes"])
def test_calls_on_dense_rows_refuse_the_cache(native, monkeypatch):
    s = Step(seed=32)
    before = s.state()
    marked, bare = [pk.shard_table(c.view(torch.int8)) for c in s.codes], s.tabs
    dense = pk.make_desc(B, s.q.shape[1], HKV, D, s.desc.E, s.desc.S, dtype=pk.BF16)
    flagged = pk.make_desc(B, s.q.shape[1], HKV, D, s.desc.E, s.desc.S, dtype=pk.BF16, flags=pk.DESC_8BIT)
    ws = torch.zeros(pk.pikv_attn_workspace_bytes(dense, K), device="cuda:0", dtype=torch.uint8)
    if not native:
        monkeypatch.setattr(pk.binding, "_native", pk.binding._NoExtension())

    def calls(d, tabs):
        return [lambda: pk.pikv_sharded_attn(d, s.q, *tabs, None, None, s.n, s.topk, s.gates, K, pk.COMBINE_LSE, 0.0, s.y, None, None, s.scores, s.coef, ws),
                lambda: pk.pikv_sharded_attn_noalloc(d, s.q, *tabs, None, None, s.n, s.topk, s.gates, K, pk.COMBINE_LSE, 0.0, s.y, None, None, s.scores,
                                                     s.coef),
                lambda: pk.pikv_append(d, s.k_new, s.v_new, s.topk, K, None, None, 0, *tabs, s.utility, s.n),
                lambda: pk.pikv_evict(d, s.utility, s.n, 10, None, 0, s.eidx, s.ecnt, 1, True, *tabs),
                lambda: pk.pikv_decode_step(d, s.q, s.W_r, None, s.k_new, s.v_new, *tabs, None, None, s.n, s.utility, K, pk.COMBINE_LSE, 0.0, 1.0, s.topk,
                                            s.gates, s.eidx, s.ecnt, s.y, s.row_max, s.row_norm, s.scores, s.coef, ws)]

    for call in calls(flagged, bare):
        with pytest.raises(pk.PikvError) as e:
            call()
        assert e.value.status == INVALID
    for call in calls(dense, marked):
        with pytest.raises(TypeError, match="8-bit"):
            call()
    assert all(torch.equal(a, b) for a, b in zip(before, s.state()))
