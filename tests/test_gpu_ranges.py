"""Caps and scales near the ends of what the calls take: the plain forms' results, from products that are zero among them."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

import paged_reference as ref  # noqa: E402
from test_gpu_paged import Attention  # noqa: E402
from test_gpu_prompt import Device, check_attention, check_mass  # noqa: E402


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[140, 9], [300] * 12], ids=["split", "whole"])
@pytest.mark.parametrize("kw", [dict(cap=2.0 ** -127), dict(cap=1e-8, scale=1e30), dict(cap=1e-37, slopes=True)], ids=["cap", "factor", "slopes"])
def test_small_caps_over_prompts(kw, lens, dtype):
    p = ref.Prompts(lens, 8, 4, 64, dtype, seed=2, **kw)
    p.k[::3] = 0.0                               # products of zero
    p.q[5] = 0.0
    p.magnitude = lambda: 4.0                    # (scores are the cap at most; 4: bars of sums and exponentials as of ordinary ones)
    d = Device(p)
    d.attend()
    check_attention(d)
    d.weigh()
    check_mass(d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [dict(scale=2e38), dict(cap=2e38, scale=0.1)], ids=["scale", "cap"])
def test_large_scales_over_prompts(kw, dtype):
    p = ref.Prompts([200], 4, 2, 64, dtype, seed=3, **kw)
    if "cap" not in kw:
        p.q[:] = 0.0                             # (scores of anything else are beyond float32)
        p.magnitude = lambda: 0.0
    else:                                        # scale / cap lies below the normal numbers: a step of 2^-149 in 5e-40, 2^-18, and a half of one in 1 / cap
        m = ref.Prompts.magnitude
        p.magnitude = lambda: m(p)
        p.errors = lambda: tuple(x + y for x, y in zip(ref.error_of(m(p), 64, 200), (2.0 ** -17 * m(p), 2.0 ** -16 * m(p))))
    d = Device(p)
    d.attend()
    check_attention(d)
    d.weigh()
    check_mass(d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S", [100, 2500])
@pytest.mark.parametrize("kw", [dict(cap=2.0 ** -127), dict(cap=1e-8, scale=1e30), dict(cap=1e-37, window=60)], ids=["cap", "factor", "window"])
def test_small_caps_over_pages(kw, S, dtype):
    a = Attention(2, 3, 2, 4, S, 64, dtype, 16, 2, seed=5, **kw)
    a.K[:, :, :, ::3] *= 0.0
    a.run()
    reference = a.reference
    a.reference = lambda: (*reference()[:5], 4.0)
    a.check()
