"""Utilities of a prompt: a row whose row_norm is 0 gives nothing, whatever it holds."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

import paged_reference as ref  # noqa: E402
from test_gpu_prompt import Device, check_mass, host  # noqa: E402


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [dict(), dict(window=50), dict(prefix=[40]), dict(slopes=True, prefix=[40]), dict(cap=9.0), dict(cap=9.0, slopes=True, window=50)],
                         ids=lambda m: "_".join(m) or "causal")
@pytest.mark.parametrize("n,Hq,Hkv,D", [(190, 4, 2, 64), (700, 3, 1, 32), (260, 2, 2, 128)])
def test_rows_that_are_left_out_may_hold_anything(n, Hq, Hkv, D, kw, dtype):
    make = lambda: ref.Prompts([n], Hq, Hkv, D, dtype, seed=6, **kw)
    out = np.zeros((n, Hq), bool)
    out[100:103] = out[5, 0] = out[n - 1, Hq - 1] = True
    d = Device(make())
    d.attend()
    gone = torch.from_numpy(out).to(d.row_norm.device)
    d.row_norm[gone] = 0.0
    d.weigh()
    check_mass(d)
    want = host(d.mass)
    stats = d.row_max, d.row_norm
    for bad in (np.nan, np.inf, 3e38):
        p = make()
        p.q[out] = ref.stored(np.full(D, bad), dtype)
        d = Device(p)
        d.row_max, d.row_norm = (x.clone() for x in stats)
        d.row_max[gone] = bad
        d.weigh()
        np.testing.assert_array_equal(host(d.mass), want)
