"""The bars of the attention's precision lie between what three parts of an operand give and what two do, by emulation in numpy."""
import numpy as np
import pytest

import quant_precision as prec


def test_scores_of_two_part_queries_exceed_the_bar():
    rng = np.random.default_rng(0)
    for fmt in (0, 1):
        for D in (32, 64, 128):
            q, K = prec.queries(rng, (8, D)), prec.sparse_codes(rng, (50, D), fmt)
            want = q @ K.T
            assert (np.abs(prec.parts(q, 2) @ K.T - want) >= prec.SCORE_SHORT * want).all()
            assert (np.abs(prec.parts(q, 3) @ K.T - want) <= 1e-12 * want).all()
    assert prec.SCORE_BAR < prec.SCORE_SHORT


@pytest.mark.parametrize("fmt", [0, 1])
def test_outputs_of_two_part_weights_exceed_the_bar(fmt):
    p = np.exp(-prec.weight_codes(fmt) * prec.KEY_STEP[fmt])
    want = p / (1 + p)
    assert (np.abs(prec.parts(np.float32(p), 2) / (1 + p) - want) >= prec.Y_SHORT * want * (1 - 1e-3)).all()
    assert (np.abs(prec.parts(np.float32(p), 3) / (1 + p) - want) <= 2.0 ** -24 * want).all()
    assert prec.Y_BAR < prec.Y_SHORT * (1 - 1e-3)
