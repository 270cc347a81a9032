"""The plain forms that the GPU tests compare with, pinned to values worked out by hand and to torch's own 8-bit type."""
import math

import numpy as np
import pytest
import torch

import quant_reference as ref


def test_e4m3_table_and_rounding_are_torchs():
    codes = np.arange(256, dtype=np.uint8)
    theirs = torch.from_numpy(codes.copy()).view(torch.float8_e4m3fn).float().numpy()
    np.testing.assert_array_equal(ref.decode(codes, 1), theirs)
    rng = np.random.default_rng(0)
    v = np.concatenate([rng.uniform(-448, 448, 4000), rng.normal(0, 0.02, 4000), ref.E4M3[:126] + np.diff(ref.E4M3[:127]) / 2, [0.0, 448.0, -448.0]])
    theirs = torch.from_numpy(v.astype(np.float32)).to(torch.float8_e4m3fn).float().numpy()
    np.testing.assert_array_equal(ref.decode(ref.encode(v.astype(np.float32).astype(np.float64), 1), 1), theirs)


@pytest.mark.parametrize("fmt,most,scale", [(0, 127.0, 1.0), (0, 127.5, 2.0), (0, 254.0, 2.0), (0, 1.0, 2.0 ** -6), (0, 0.0, 2.0 ** -126),
                                            (1, 448.0, 1.0), (1, 449.0, 2.0), (1, 1.0, 2.0 ** -8), (1, 1.75, 2.0 ** -8), (1, 1.76, 2.0 ** -7)])
def test_scales_are_the_smallest_power_of_two(fmt, most, scale):
    assert ref.needed_scale(most, fmt) == scale


def test_codes_are_nearest_ties_to_even():
    x = np.array([[0.5, 1.5, 2.5, -0.5, -1.5, 126.5, 127.0, -127.0]])
    codes, scale = ref.quantise_block(x, 0)
    assert scale == 1.0 and ref.decode(codes, 0).tolist() == [[0, 2, 2, 0, -2, 126, 127, -127]]
    codes, scale = ref.quantise_block(np.array([[math.inf, 1.0]]), 0)
    assert math.isnan(scale) and (codes == 0).all()


def test_append_rounds_the_codes_of_a_block_whose_scale_grows():
    codes, scales = np.zeros((1, 8, 2), np.uint8), np.full((1, 1), np.nan, np.float32)
    ref.append(np.array([[100.0, 3.0]]), 0, 0, 0, 0, 16, codes, scales, 8)            # the block's first: its own scale
    assert scales[0, 0] == 1.0 and codes[0, 0].tolist() == [100, 3]
    ref.append(np.array([[200.0, 1.0]]), 1, 1, 0, 0, 16, codes, scales, 8)
    assert scales[0, 0] == 2.0 and codes[0, 0].tolist() == [50, 2] and codes[0, 1].tolist() == [100, 0]      # 1.5 -> 2, 0.5 -> 0
    ref.append(np.array([[4.0, 2.0]]), 2, 2, 0, 0, 16, codes, scales, 8)              # does not shrink
    assert scales[0, 0] == 2.0 and codes[0, 2].tolist() == [2, 1]


def test_rotation_keeps_lengths_and_is_a_quarter_turn_at_half_pi():
    x = np.arange(1.0, 17).reshape(1, 1, 16)
    pos, f = np.array([1]), np.full(8, math.pi / 2)
    out = ref.norm_rope(x, None, 0.0, pos, f, 16, False)
    np.testing.assert_allclose(out[0, 0], np.concatenate([-x[0, 0, 8:], x[0, 0, :8]]), atol=1e-14)
    out = ref.norm_rope(x, None, 0.0, pos, f[:4], 8, True)
    np.testing.assert_allclose(out[0, 0, :4], [-2, 1, -4, 3], atol=1e-14)
    np.testing.assert_array_equal(out[0, 0, 8:], x[0, 0, 8:])
    normed = ref.norm_rope(x, np.full(16, 2.0), 0.0, pos, f, 16, False)
    assert math.isclose((normed ** 2).mean(), 4.0)


def test_attention_over_every_shard_is_one_softmax():
    rng = np.random.default_rng(1)
    q, K, V = rng.normal(size=(1, 2, 4)), rng.normal(size=(1, 2, 1, 3, 4)), rng.normal(size=(1, 2, 1, 3, 4))
    out = ref.attend(q, K, V, np.full((1, 2), 3), np.array([[1, 0]]), None, 1)
    k, v = K.reshape(6, 4), V.reshape(6, 4)
    p = np.exp(q[0] @ k.T / 2)
    p /= p.sum(1, keepdims=True)
    np.testing.assert_allclose(out["y"][0], p @ v, rtol=1e-12)
    np.testing.assert_allclose(out["mass"].reshape(6), p.sum(0), rtol=1e-12)
    empty = ref.attend(q, K, V, np.zeros((1, 2), int), np.array([[1, 0]]), None, 1)
    assert (empty["y"] == 0).all() and (empty["row_max"] == -np.inf).all() and (empty["row_norm"] == 0).all()
