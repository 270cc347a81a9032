"""The definition of a scale that comes down, on cases worked out by hand, and what it is for: a stream past one large entry."""
import numpy as np
import pytest

import quant_recovery as rec
import quant_reference as ref


def block_of(rows, fmt):
    """codes [1, S, D] and scales of one block that holds the rows."""
    rows = np.asarray(rows, np.float64)
    codes = np.zeros((1,) + rows.shape, np.uint8)
    codes[0], scale = ref.quantise_block(rows, fmt)
    return codes, np.full((1, 1), scale, np.float32)


def test_the_scale_comes_down_with_the_entry_that_kept_it_up():
    codes, scales = block_of([[127.0, 0.0], [9.0, 3.0], [-15.0, 1.0]], 0)
    assert scales[0, 0] == 1.0
    rec.append(np.array([[2.0, 0.25]]), 0, 2, 1, 0, 16, codes, scales, 3)
    assert scales[0, 0] == 0.125                                     # 15 / 127 rounded up to a power of two
    assert codes.view(np.int8)[0].tolist() == [[16, 2], [72, 24], [-120, 8]]


@pytest.mark.parametrize("rows,new,cnt", [([[127, 0], [16, 3]], 2, 1),           # what stays needs a quarter
                                          ([[127, 0], [15, 3]], 16, 1),          # the new entry does
                                          ([[15, 0], [127, 3]], 2, 1),           # another entry keeps it up
                                          ([[127, 0], [15, 3]], 2, 0)])          # no entry leaves
def test_the_scale_stays(rows, new, cnt):
    codes, scales = block_of(rows + [[0, 0]], 0)
    slot, n = (0, 2) if cnt else (2, 2)
    want = codes.copy(), scales.copy()
    rec.append(np.array([[new, 0.0]]), slot, n, cnt, 0, 16, codes, scales, 3)
    ref.append(np.array([[new, 0.0]]), slot, n, cnt, 0, 16, *want, 3)
    assert scales[0, 0] == 1.0 and (codes == want[0]).all()


def test_zeros_that_stay_leave_the_new_entry_its_own_scale():
    codes, scales = block_of([[448.0, 0.0], [0.0, 0.0]], 1)
    rec.append(np.array([[2.0 ** -100, 0.0]]), 0, 1, 1, 1, 16, codes, scales, 2)
    assert scales[0, 0] == 2.0 ** -108 and (ref.decode(codes, 1) * scales[0, 0] == [[[2.0 ** -100, 0], [0, 0]]]).all()


def stream(append, fmt, S, block, D, order, rows, first):
    codes, scales = np.zeros((1, S, D), np.uint8), np.zeros((1, -(-S // block)), np.float32)
    ref.pack(first[None, None, None], np.array([[S]]), fmt, block, codes[None, None], scales[None, None])
    for slot, row in zip(order, rows):
        append(row[None], slot, S - 1, 1, fmt, block, codes, scales, S)
    return ref.values(codes[None, None], scales[None, None], fmt, block)[0, 0, 0], scales


@pytest.mark.parametrize("fmt", [0, 1])
def test_a_stream_recovers_from_one_large_entry(fmt):
    """Every slot is rewritten after the large entry has left: a value is then off by at most a step of a scale that is at most four
    times what its block needs (half a step as it is written, less in all if the scale grows later: a quarter, an eighth ...)."""
    rng = np.random.default_rng(0)
    S, block, D = 100, 32, 64
    order = np.concatenate([[40]] + [rng.permutation(S) for _ in range(2)])
    rows = rng.normal(size=(len(order), D))
    rows[0] *= 1000
    held = np.zeros((S, D))
    for slot, row in zip(order, rows):
        held[slot] = row
    got, scales = stream(rec.append, fmt, S, block, D, order, rows, rng.normal(size=(S, D)))
    for i, lo in enumerate(range(0, S, block)):
        hold = slice(lo, min(lo + block, S))
        need = ref.needed_scale(np.abs(got[hold]).max(), fmt)
        assert need <= scales[0, i] <= 4 * need
        step = scales[0, i] if fmt == 0 else np.maximum(np.abs(held[hold]) / 8, scales[0, i] * 2.0 ** -9)
        assert (np.abs(got[hold] - held[hold]) <= step).all()
    worst = stream(ref.append, fmt, S, block, D, order, rows, rng.normal(size=(S, D)))[1]
    assert worst[0, 1] >= 64 * scales[0, 1]                          # (the scale of the large entry, had it stayed)


def word(scales):
    return int(rec.bits(scales)[0, 0])


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_a_row_that_is_not_finite_leaves_the_others_their_codes(bad):
    codes, scales = block_of([[100.0, 3.0], [7.0, 1.0], [-2.0, 5.0]], 0)
    assert scales[0, 0] == 1.0
    rec.append(np.array([[bad, 1.0]]), 1, 2, 1, 0, 16, codes, scales, 3)
    assert word(scales) == 0x7fc0007f and codes.view(np.int8)[0].tolist() == [[100, 3], [-128, -128], [-2, 5]]
    rec.append(np.array([[200.0, 1.0]]), 2, 2, 1, 0, 16, codes, scales, 3)      # its neighbour's scale grows meanwhile
    assert word(scales) == 0x7fc00080 and codes.view(np.int8)[0].tolist() == [[50, 2], [-128, -128], [100, 0]]
    rec.append(np.array([[4.0, 3.0]]), 1, 2, 1, 0, 16, codes, scales, 3)
    assert scales[0, 0] == 2.0 and codes.view(np.int8)[0].tolist() == [[50, 2], [2, 2], [100, 0]]


def test_a_block_that_kept_nothing_is_whole_again_once_every_slot_is_rewritten():
    codes, scales = block_of([[1.0, 2.0], [3.0, 4.0], [5.0, 6.0]], 1)
    rec.append(np.array([[np.nan, 0.0]]), 2, 2, 0, 1, 16, codes, scales, 3)     # behind the last entry: no freed slot
    assert np.isnan(scales[0, 0]) and (codes == 0).all()
    for slot in (0, 2, 1):
        assert np.isnan(scales[0, 0])
        rec.append(np.array([[448.0, slot + 1.0]]), slot, 2, 1, 1, 16, codes, scales, 3)
    assert (ref.decode(codes, 1) * scales[0, 0] == [[[448, 1], [448, 2], [448, 3]]]).all()


@pytest.mark.parametrize("fmt", [0, 1])
def test_packed_rows_that_are_not_finite_have_no_part_in_the_scale(fmt):
    rng = np.random.default_rng(1)
    clean = rng.normal(size=(1, 1, 1, 40, 32))
    dirty = clean.copy()
    dirty[0, 0, 0, [3, 5, 35], [0, 31, 7]] = [np.nan, np.inf, -np.inf]
    out = [(np.full(clean.shape, 9, np.uint8), np.zeros((1, 1, 1, 3), np.float32)) for _ in range(2)]
    for x, (c, s) in zip((np.where(np.isfinite(dirty).all(-1, keepdims=True), clean, 0), dirty), out):
        rec.pack(x, np.array([[38]]), fmt, 16, c, s)
    (want, ws), (got, gs) = out
    rows = np.isin(np.arange(40), [3, 5, 35])
    assert (got[0, 0, 0, ~rows] == want[0, 0, 0, ~rows]).all() and (got[0, 0, 0, rows] == rec.NO_CODES[fmt]).all()
    assert [rec.kept(w) for w in rec.bits(gs)[0, 0, 0]] == ws[0, 0, 0].tolist() and np.isnan(gs[0, 0, 0]).tolist() == [True, False, True]
