"""What each tensor of the calls around the 8-bit cache has to hold, as the binding counts it."""
import pytest
import torch

import paper_2508_06526_amd as pk
from paper_2508_06526_amd import binding

B, E, HQ, HKV, S, D, K, BLOCK = 2, 3, 8, 4, 100, 64, 2, 16
DESC = pk.make_desc(B, HQ, HKV, D, E, S, dtype=pk.BF16)


def z(*shape, t=torch.float32):
    return torch.zeros(shape, dtype=t)


def cache():
    i64 = torch.int64
    return dict(K_shards=z(B * E, t=i64), V_shards=z(B * E, t=i64), K_scales=z(B, E, HKV, 7), V_scales=z(B, E, HKV, 7), n_valid=z(B, E, t=torch.int32))


def rope(**kw):
    a = dict(x=z(5, 16 * D), tokens=5, token_stride=16 * D, Hq=8, Hkv=4, D=D, w_q=z(D), w_k=z(D), positions=z(5), inv_freq=z(D // 2), rotary_dim=D,
             q_out=z(5, 8, D), k_out=z(5, 4, D), v_out=z(5, 4, D))
    a.update(kw)
    return binding._rope_tensors(**a)


def append(**kw):
    a = dict(cache(), desc=DESC, block=BLOCK, K_new=z(B, HKV, D), V_new=z(B, HKV, D), topk_idx=z(B, K), k=K, reuse_idx=z(B, E, 2), reuse_cnt=z(B, E),
             max_evict=2, utility=z(B, E, S))
    a.update(kw)
    return binding._append_tensors(**a)


def attn(desc=DESC, rows=B, **kw):
    a = dict(cache(), desc=desc, block=BLOCK, q=z(B, HQ, D), topk_idx=z(rows, K), gates=z(rows, K), k=K, y=z(B, HQ, D), row_max=z(B, HQ), row_norm=z(B, HQ),
             scores=z(B, HQ, K, S), slot_coef=z(B, HQ, K, 2), workspace=z(1))
    a.update(kw)
    return binding._attn_tensors(**a)


@pytest.mark.parametrize("make", [rope, append, attn])
def test_exact_sizes_hold_and_one_element_less_does_not(make):
    sizes = make()
    binding._holds("call", sizes)
    for name, t, least, *_ in sizes:
        if name == "workspace":
            continue
        assert t.numel() == least, name
        with pytest.raises(ValueError, match="call: %s has %d elements, %d are needed" % (name, least - 1, least)):
            binding._holds("call", make(**{name: t.reshape(-1)[1:]}))


def test_scales_of_another_block_and_scores_of_another_capacity():
    for make, name, t, last in ((append, "K_scales", z(B, E, HKV, 13), 7), (attn, "V_scales", z(B, E, HKV, 13), 7), (attn, "scores", z(B, HQ, K, 128), 100)):
        with pytest.raises(ValueError, match="last dimension of %s is %d, not %d" % (name, t.shape[-1], last)):
            binding._holds("call", make(**{name: t}))
        binding._holds("call", make(**{name: t.flatten()}))          # a longer buffer without a shape


def test_routing_per_head_and_what_is_not_given():
    per_head = pk.make_desc(B, HQ, HKV, D, E, S, dtype=pk.BF16, route_rows_per_seq=HQ)
    binding._holds("call", attn(per_head, rows=B * HQ))
    with pytest.raises(ValueError, match="topk_idx"):
        binding._holds("call", attn(per_head))
    binding._holds("call", attn(gates=None, row_max=None, row_norm=None, scores=None, slot_coef=None))
    binding._holds("call", append(reuse_idx=None, reuse_cnt=None, max_evict=0))
    binding._holds("call", rope(w_q=None, w_k=None, positions=None, inv_freq=None, rotary_dim=0))


def test_rows_of_a_projection():
    wide = z(5, 20 * D)
    binding._holds("call", rope(x=wide[:, D:17 * D], token_stride=20 * D))
    binding._holds("call", rope(x=wide, token_stride=20 * D))
    binding._holds("call", rope(x=z(5, 12 * D), token_stride=12 * D, v_out=None))
    binding._holds("call", rope(x=z(0, 16 * D), tokens=0, positions=z(0), q_out=z(0, 8, D), k_out=z(0, 4, D), v_out=z(0, 4, D)))
    binding._holds("call", rope(x=z(4 * 20 * D + 16 * D), token_stride=20 * D))            # the last row need not be a whole stride
    for x, kw in ((wide[:, D:16 * D], dict(token_stride=20 * D)), (wide[1:, D:17 * D], dict(token_stride=20 * D)), (z(5, 15 * D), {}), (z(4, 16 * D), {}),
                  (z(5, 16 * D), dict(token_stride=20 * D))):
        with pytest.raises(ValueError, match="call: x"):
            binding._holds("call", rope(x=x, **kw))


def test_rows_of_one_head_may_be_a_slice_of_a_wider_one():
    wide = z(5, 1, 100)
    assert binding._rows(wide[:, :, 20:84], 100) == wide.data_ptr() + 80
    for x in (z(5, 2, 100)[:, :, 20:84], z(5, 64, 2).transpose(1, 2)[:, :1]):          # heads that do not follow each other, values that do not
        with pytest.raises(ValueError, match="contiguous"):
            binding._rows(x, 200)
