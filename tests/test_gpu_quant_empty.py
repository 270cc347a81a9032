"""Calls with nothing to do, given what a program then has: tensors without elements."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

import paper_2508_06526_amd as pk  # noqa: E402


@pytest.mark.parametrize("native", [True, False], ids=["extension", "ctypes"])
def test_tensors_without_elements(native, monkeypatch):
    pk.load_library()
    if not native:
        monkeypatch.setattr(pk.binding, "_native", pk.binding._NoExtension())
    z = lambda *s, t=torch.float32: torch.zeros(s, device="cuda:0", dtype=t)
    bf, i32, i64 = torch.bfloat16, torch.int32, torch.int64
    pk.pikv_norm_rope(z(0, 12 * 64, t=bf), 0, 12 * 64, 4, 4, 64, z(64, t=bf), z(64, t=bf), 1e-6, z(0, t=i32), z(32), 64, False, z(0, 4, 64, t=bf),
                      z(0, 4, 64, t=bf), z(0, 4, 64, t=bf))
    d, tab, scales, n = pk.make_desc(0, 8, 4, 64, 8, 100, dtype=1), z(0, t=i64), z(0, 8, 4, 7), z(0, 8, t=i32)
    pk.pikv_quant_pack(d, 0, 16, tab, tab, 6400, 64, n, tab, tab, scales, scales)
    pk.pikv_quant_read(d, 0, 16, tab, tab, scales, scales, n, tab, tab, 6400, 64)
    row = z(0, 4, 64, t=bf)
    pk.pikv_quant_append(d, 0, 16, row, row, z(0, 2, t=i32), 2, z(0, 8, 1, t=i32), z(0, 8, t=i32), 1, tab, tab, scales, scales, z(0, 8, 100), n)
    pk.pikv_quant_attn(d, 0, 16, z(0, 8, 64, t=bf), tab, tab, scales, scales, n, z(0, 2, t=i32), z(0, 2), 2, 0, 0.0, z(0, 8, 64), z(0, 8), z(0, 8),
                       z(0, 8, 2, 100), z(0, 8, 2, 2), z(pk.pikv_quant_attn_workspace_bytes(d, 2), t=torch.uint8))
    torch.cuda.synchronize()
