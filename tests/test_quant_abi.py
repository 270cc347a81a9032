"""Refusals of the calls around the 8-bit cache: found on the host, before anything is launched."""
import ctypes as C

import pytest
import torch

import paper_2508_06526_amd as pk
from paper_2508_06526_amd import binding

INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3
FAKE = C.c_void_p(0x1000)        # never dereferenced: the calls below fail validation or have nothing to do


@pytest.fixture(scope="module")
def lib():
    return pk.load_library()


def desc(**kw):
    return pk.make_desc(**dict(dict(B=2, Hq=8, Hkv=4, D=64, E=8, S=100, dtype=1), **kw))


def rope(lib, x=FAKE, tokens=3, stride=None, Hq=4, Hkv=2, D=64, dtype=1, w=FAKE, eps=1e-6, pos=FAKE, freq=FAKE, rot=64, q=FAKE, k=FAKE, v=FAKE):
    stride = (Hq + 2 * Hkv) * D if stride is None else stride
    return lib.pikv_norm_rope(x, tokens, stride, Hq, Hkv, D, dtype, w, w, eps, pos, freq, rot, 0, q, k, v, None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), INVALID), (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(pos=None), INVALID), (dict(freq=None), INVALID),
    (dict(tokens=-1), INVALID), (dict(Hq=-1), INVALID), (dict(Hq=0, Hkv=0), INVALID), (dict(dtype=2), INVALID), (dict(D=96, rot=96), UNSUPPORTED),
    (dict(D=256), UNSUPPORTED), (dict(rot=8), INVALID), (dict(rot=80), INVALID), (dict(rot=-16), INVALID), (dict(eps=-1.0), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID), (dict(stride=8 * 64 - 8), INVALID), (dict(stride=8 * 64 + 4), INVALID),
    (dict(x=C.c_void_p(0x1008)), INVALID), (dict(q=C.c_void_p(0x1002)), INVALID), (dict(w=C.c_void_p(0x1004)), INVALID),
    (dict(tokens=1 << 24, Hq=64), UNSUPPORTED), (dict(tokens=0), 0), (dict(tokens=0, pos=None, freq=None, rot=0), 0),
    (dict(tokens=0, Hq=0, q=None), 0), (dict(tokens=0, Hkv=0, k=None, v=None), 0), (dict(tokens=0, v=None, stride=6 * 64), 0)])
def test_norm_rope_refusals(lib, kw, status):
    assert rope(lib, **kw) == status


COMMON = [(dict(fmt=2), INVALID), (dict(fmt=-1), INVALID), (dict(block=8), INVALID), (dict(block=48), INVALID), (dict(block=256), INVALID),
          (dict(d=dict(D=16)), UNSUPPORTED), (dict(d=dict(rank=32)), UNSUPPORTED), (dict(d=dict(stride_s=72)), INVALID),
          (dict(d=dict(stride_s=48)), INVALID), (dict(d=dict(stride_h=6408)), INVALID), (dict(d=dict(stride_h=6336)), INVALID),
          (dict(d=dict(Hq=6)), INVALID), (dict(d=dict(B=0)), 0)]


@pytest.mark.parametrize("kw,status", COMMON + [(dict(missing=i), INVALID) for i in range(7)] + [
    (dict(ds=56), INVALID), (dict(ds=68), INVALID), (dict(dh=100 * 64 - 8), INVALID), (dict(dh=-64), INVALID), (dict(d=dict(B=1 << 20)), UNSUPPORTED)])
def test_pack_and_read_refusals(lib, kw, status):
    d = desc(**kw.get("d", {}))
    ptr = [None if kw.get("missing") == i else FAKE for i in range(7)]
    args = kw.get("fmt", 0), kw.get("block", 16)
    strides = kw.get("dh", 100 * 64), kw.get("ds", 64)
    assert lib.pikv_quant_pack(C.byref(d), *args, ptr[0], ptr[1], *strides, ptr[2], *ptr[3:], None) == status
    assert lib.pikv_quant_read(C.byref(d), *args, *ptr[3:], ptr[2], ptr[0], ptr[1], *strides, None) == status


@pytest.mark.parametrize("kw,status", COMMON + [(dict(missing=i), INVALID) for i in (0, 1, 2, 5, 6, 7, 8, 9, 10)] + [
    (dict(k=0), INVALID), (dict(k=9), INVALID), (dict(missing=3), INVALID), (dict(missing=4), INVALID), (dict(me=0), INVALID),
    (dict(d=dict(route_rows_per_seq=8)), UNSUPPORTED)])
def test_append_refusals(lib, kw, status):
    d = desc(**kw.get("d", {}))
    ptr = [None if kw.get("missing") == i else FAKE for i in range(11)]
    assert lib.pikv_quant_append(C.byref(d), kw.get("fmt", 0), kw.get("block", 16), *ptr[:3], kw.get("k", 2), ptr[3], ptr[4],
                                 kw.get("me", 1), *ptr[5:], None) == status


@pytest.mark.parametrize("kw,status", COMMON + [(dict(missing=i), INVALID) for i in range(7)] + [
    (dict(k=0), INVALID), (dict(k=9), INVALID), (dict(combine=2), INVALID), (dict(scale=float("nan")), INVALID), (dict(y=None), INVALID),
    (dict(ws=None), WORKSPACE), (dict(ws_bytes=256), WORKSPACE), (dict(ws=C.c_void_p(0x1010)), INVALID),
    (dict(d=dict(tq=2, route_rows_per_seq=8)), UNSUPPORTED), (dict(d=dict(tq=3)), UNSUPPORTED), (dict(d=dict(tq=4)), UNSUPPORTED),
    (dict(d=dict(stride_s=(1 << 24) + 16)), UNSUPPORTED), (dict(d=dict(B=1 << 20), k=8), UNSUPPORTED)])
def test_attention_refusals(lib, kw, status):
    d = desc(**kw.get("d", {}))
    ptr = [None if kw.get("missing") == i else FAKE for i in range(7)]
    assert lib.pikv_quant_attn(C.byref(d), kw.get("fmt", 0), kw.get("block", 16), *ptr, None if kw.get("nogates") else FAKE, kw.get("k", 2),
                               kw.get("combine", 0), kw.get("scale", 0.0), kw.get("y", FAKE), None, None, None, None, kw.get("ws", FAKE),
                               kw.get("ws_bytes", 1 << 40), None) == status


def test_workspace_is_zero_where_the_call_is_refused(lib):
    assert pk.pikv_quant_attn_workspace_bytes(desc(), 2) > 0
    assert pk.pikv_quant_attn_workspace_bytes(desc(tq=2), 2) > 0
    for bad in (desc(D=16), desc(rank=32), desc(stride_s=72), desc(tq=3), desc(Hq=6)):
        assert pk.pikv_quant_attn_workspace_bytes(bad, 2) == 0
    assert pk.pikv_quant_attn_workspace_bytes(desc(), 0) == pk.pikv_quant_attn_workspace_bytes(desc(), 9) == 0


def test_splits_of_long_shards_stay_within_what_the_merge_holds(lib):
    d = desc(B=1, Hq=1, Hkv=1, D=128, E=64, S=1 << 24)
    rows = pk.pikv_quant_attn_workspace_bytes(d, 64) / (64 * 130 * 4)
    assert 1 <= rows < 2048 // 64 + 1


@pytest.mark.parametrize("name", ["pikv_norm_rope", "pikv_quant_pack", "pikv_quant_read", "pikv_quant_append", "pikv_quant_attn"])
def test_the_binding_refuses_host_memory_and_other_types(name):
    d, f = desc(), lambda *shape, t=torch.float32: torch.zeros(shape, dtype=t)
    i32, tab, bf = f(4, t=torch.int32), f(16, t=torch.int64), f(16, t=torch.bfloat16)
    calls = {
        "pikv_norm_rope": lambda i, s, tab=tab: pk.pikv_norm_rope(bf, 1, 512, 4, 2, 64, None, None, 1e-6, i, s, 64, False, bf, bf, bf),
        "pikv_quant_pack": lambda i, s, tab=tab: pk.pikv_quant_pack(d, 0, 16, tab, tab, 6400, 64, i, tab, tab, s, s),
        "pikv_quant_read": lambda i, s, tab=tab: pk.pikv_quant_read(d, 0, 16, tab, tab, s, s, i, tab, tab, 6400, 64),
        "pikv_quant_append": lambda i, s, tab=tab: pk.pikv_quant_append(d, 0, 16, bf, bf, i, 2, i, i, 1, tab, tab, s, s, s, i),
        "pikv_quant_attn": lambda i, s, tab=tab: pk.pikv_quant_attn(d, 0, 16, bf, tab, tab, s, s, i, i, s, 2, 0, 0.0, s, s, s, s, s, s)}
    with pytest.raises(ValueError, match="device memory"):
        calls[name](i32, f(4))
    with pytest.raises(TypeError, match="int32"):
        calls[name](i32.long(), f(4))
    with pytest.raises(TypeError, match="float32"):
        calls[name](i32, f(4, t=torch.float64))
    if name != "pikv_norm_rope":                 # the shards in place of the table of their addresses
        with pytest.raises(TypeError, match="int64"):
            calls[name](i32, f(4), tab=f(16, t=torch.uint8))


def test_the_binding_refuses_dense_tensors_of_another_type():
    f = torch.zeros(4)
    with pytest.raises(TypeError, match="bfloat16"):
        pk.pikv_quant_attn(desc(), 0, 16, f, f, f, f, f, f, f, f, 2, 0, 0.0, f, f, f, f, f, f)
    with pytest.raises(TypeError, match="bfloat16"):
        pk.pikv_quant_append(desc(), 0, 16, f, f, f, 2, f, f, 1, f, f, f, f, f, f)
    with pytest.raises(TypeError):
        pk.pikv_norm_rope(f, 1, 512, 4, 2, 64, f.bfloat16(), None, 1e-6, f, f, 64, False, f, f)


def test_rows_of_a_wider_projection_are_taken_as_they_lie():
    wide = torch.zeros((3, 100), dtype=torch.bfloat16)
    assert binding._rows(wide[:, 16:80], 100) == wide.data_ptr() + 32
    with pytest.raises(ValueError, match="token_stride"):
        binding._rows(wide[:, 16:80], 64)
    with pytest.raises(ValueError, match="contiguous"):
        binding._rows(wide.t(), 100)
