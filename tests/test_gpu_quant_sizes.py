"""Tensors that are too small for a call around the 8-bit cache are refused by both paths of the binding, before anything is launched."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

import paper_2508_06526_amd as pk  # noqa: E402
from test_gpu_quant_chain import B, BLOCK, D, EPS, HKV, HQ, K, S, Step  # noqa: E402

NAMES = {
    "rope": "x tokens token_stride Hq Hkv D w_q w_k eps positions inv_freq rotary_dim interleaved q_out k_out v_out",
    "pack": "desc format block K_dense V_dense dense_stride_h dense_stride_s n_valid K_shards V_shards K_scales V_scales",
    "read": "desc format block K_shards V_shards K_scales V_scales n_valid K_dense V_dense dense_stride_h dense_stride_s",
    "append": "desc format block K_new V_new topk_idx k reuse_idx reuse_cnt max_evict K_shards V_shards K_scales V_scales utility n_valid",
    "attn": "desc format block q K_shards V_shards K_scales V_scales n_valid topk_idx gates k combine scale y row_max row_norm scores slot_coef workspace"}


def calls(s, dense):
    cache, strides = (*s.tabs, *s.scales), (S * D, D)
    return {
        "rope": (pk.pikv_norm_rope, [s.x, B, (HQ + 2 * HKV) * D, HQ, HKV, D, *s.w, EPS, s.position, s.inv_freq, D, False, s.q, s.k_new, s.v_new]),
        "pack": (pk.pikv_quant_pack, [s.desc, s.fmt, BLOCK, *dense, *strides, s.n, *cache]),
        "read": (pk.pikv_quant_read, [s.desc, s.fmt, BLOCK, *cache, s.n, *dense, *strides]),
        "append": (pk.pikv_quant_append, [s.desc, s.fmt, BLOCK, s.k_new, s.v_new, s.topk, K, s.eidx, s.ecnt, 1, *cache, s.utility, s.n]),
        "attn": (pk.pikv_quant_attn, [s.desc, s.fmt, BLOCK, s.q, *cache, s.n, s.topk, s.gates, K, pk.COMBINE_LSE, 0.0, s.y, s.row_max, s.row_norm, s.scores,
                                      s.coef, s.ws])}


@pytest.mark.parametrize("native", [True, False], ids=["extension", "ctypes"])
def test_each_tensor_one_element_short(native, monkeypatch):
    s = Step(seed=41)
    buffers = [torch.zeros((B, s.desc.E, HKV, S, D), device="cuda:0", dtype=torch.bfloat16) for _ in range(2)]
    dense = [pk.shard_table(t) for t in buffers]
    if not native:
        monkeypatch.setattr(pk.binding, "_native", pk.binding._NoExtension())
    before = s.state()
    for kind, (call, args) in calls(s, dense).items():
        for i, name in enumerate(NAMES[kind].split()):
            if isinstance(args[i], torch.Tensor) and name != "workspace":
                short = args[i].reshape(-1)[:-1]
                with pytest.raises(ValueError, match="%s has %d elements" % (name, short.numel())):
                    call(*args[:i], short, *args[i + 1:])
    with pytest.raises(pk.PikvError):
        call, args = calls(s, dense)["attn"]
        call(*args[:-1], s.ws[:256])
    assert all(torch.equal(a, b) for a, b in zip(before, s.state())) and all((t == 0).all() for t in buffers)


@pytest.mark.parametrize("native", [True, False], ids=["extension", "ctypes"])
def test_more_tokens_another_block_another_capacity(native, monkeypatch):
    s = Step(seed=42)
    if not native:
        monkeypatch.setattr(pk.binding, "_native", pk.binding._NoExtension())
    before = s.state()
    rope, args = calls(s, s.tabs)["rope"]
    for tokens, stride in ((B + 1, args[2]), (B, args[2] + 8)):
        with pytest.raises(ValueError, match="x has"):
            rope(args[0], tokens, stride, *args[3:])
    attn, args = calls(s, s.tabs)["attn"]
    with pytest.raises(ValueError, match="K_scales"):                # scales of blocks of 16, taken for others
        attn(args[0], args[1], 64, *args[3:])
    with pytest.raises(ValueError, match="scores"):
        attn(*args[:17], torch.zeros((B, HQ, K, S + 14), device="cuda:0"), *args[18:])
    assert all(torch.equal(a, b) for a, b in zip(before, s.state()))
