"""The plain forms of the paged tests against themselves: masks, sums, the order of what stays."""
import numpy as np

import paged_reference as ref


def test_masks():
    pos = np.arange(6)
    _, seen = ref.scores(np.ones((6, 4)), np.ones((6, 4)), pos, pos, 1.0, window=2, prefix=2)
    want = [[1, 1, 0, 0, 0, 0], [1, 1, 0, 0, 0, 0], [1, 1, 1, 0, 0, 0], [1, 1, 1, 1, 0, 0], [1, 1, 0, 1, 1, 0], [1, 1, 0, 0, 1, 1]]
    np.testing.assert_array_equal(seen, np.array(want, bool))
    _, seen = ref.scores(np.ones((1, 4)), np.ones((3, 4)), [5], [-1, 6, 5], 1.0)
    assert seen.tolist() == [[False, False, True]]


def test_a_prompts_attention_sums_to_its_heads():
    p = ref.Prompts([9, 0, 30], 4, 2, 32, "f32", cap=4.0, slopes=True, window=11, prefix=[3, 0, 2])
    out, top, norm, _, inside = p.attend()
    assert inside.all() and np.isfinite(out).all()
    mass = p.mass(top, norm)
    np.testing.assert_allclose([mass[:9].sum(), mass[9:].sum()], [36, 120], rtol=1e-12)
    dense = ref.Prompts([5], 1, 1, 32, "f32")
    s = dense.q[:, 0].astype(float) @ dense.k[:, 0].astype(float).T / 32 ** 0.5
    w = np.exp(np.where(np.tril(np.ones((5, 5))) > 0, s, -np.inf))
    np.testing.assert_allclose(dense.attend()[0][:, 0], (w / w.sum(1, keepdims=True)) @ dense.v[:, 0], rtol=1e-12)


def test_what_stays_of_a_prompt():
    topk = np.array([[0, 1], [0, 2], [0, 0], [1, 9], [0, 1]])
    n = np.zeros((1, 3), np.int64)
    n[0, 1] = 1
    slots, counts = ref.fill([0, 5], topk, np.float32([1, 2, 2, 5, np.nan]), lambda b, e: 3, n, 10)
    assert counts.tolist() == [[3, 3, 1]]
    assert slots.tolist() == [[0, 1], [1, 0], [2, -1], [2, -1], [-1, -1]]
    slots, counts = ref.fill([0, 5], topk, None, lambda b, e: 2, n, 10)
    assert slots.tolist() == [[0, 1], [1, 0], [-1, -1], [-1, -1], [-1, -1]] and counts.tolist() == [[2, 2, 1]]


def test_bf16_rounding():
    np.testing.assert_array_equal(ref.bf16(np.float32([1.0, 1.00390625, 1.01171875, -3.0e38, np.inf])),
                                  np.float32([1.0, 1.0, 1.015625, -3.0040553e38, np.inf]))
