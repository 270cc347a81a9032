"""Refusals of the calls between a prompt and a paged cache: found on the host, before anything is launched."""
import ctypes as C

import pytest
import torch

import paper_2508_06526_amd as pk
from paper_2508_06526_amd import binding

INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3
FAKE = C.c_void_p(0x1000)        # never dereferenced: the calls below fail validation or have nothing to do
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    return pk.load_library()


def prompt(lib, missing=None, tokens=10, q_stride=512, k_stride=256, v_stride=256, Hq=8, Hkv=4, D=64, dtype=1, B=2, max_len=6, scale=0.0, cap=0.0,
           window=0, q=FAKE, out=FAKE, stats=(FAKE, FAKE)):
    q, k, v, cu, out = (None if missing == i else x for i, x in enumerate((q, FAKE, FAKE, FAKE, out)))
    return lib.pikv_prompt_attn(q, k, v, tokens, q_stride, k_stride, v_stride, Hq, Hkv, D, dtype, cu, B, max_len, None, scale, cap, None, window, out,
                                *stats, None)


def mass(lib, missing=None, tokens=10, q_stride=512, k_stride=256, Hq=8, Hkv=4, D=64, dtype=1, B=2, max_len=6, scale=0.0, cap=0.0, window=0, q=FAKE,
         ws=FAKE, ws_bytes=1 << 40):
    ptr = [None if missing == i else x for i, x in enumerate((q, FAKE, FAKE, FAKE, FAKE, FAKE))]
    return lib.pikv_prompt_mass(ptr[0], ptr[1], tokens, q_stride, k_stride, Hq, Hkv, D, dtype, ptr[2], B, max_len, None, scale, cap, None, window,
                                *ptr[3:], ws, ws_bytes, None)


BOTH = [(dict(tokens=-1), INVALID), (dict(B=-1), INVALID), (dict(max_len=-1), INVALID), (dict(Hq=0), INVALID), (dict(Hkv=0), INVALID),
        (dict(Hq=6), INVALID), (dict(dtype=2), INVALID), (dict(D=16), UNSUPPORTED), (dict(D=256, q_stride=2048, k_stride=1024), UNSUPPORTED),
        (dict(D=96), UNSUPPORTED), (dict(Hq=512, q_stride=1 << 16), UNSUPPORTED), (dict(tokens=(1 << 23) + 1), UNSUPPORTED), (dict(q_stride=504), INVALID),
        (dict(q_stride=516), INVALID), (dict(k_stride=248), INVALID), (dict(k_stride=260), INVALID), (dict(cap=-1.0), INVALID), (dict(cap=NAN), INVALID),
        (dict(cap=INF), INVALID), (dict(scale=NAN), INVALID), (dict(scale=INF), INVALID), (dict(q=C.c_void_p(0x1008)), INVALID),
        (dict(B=1 << 22, max_len=1 << 20, tokens=1 << 20), UNSUPPORTED), (dict(tokens=0), 0), (dict(B=0), 0), (dict(max_len=0), 0)]


@pytest.mark.parametrize("kw,status", BOTH + [(dict(missing=i), INVALID) for i in range(5)] + [
    (dict(v_stride=248), INVALID), (dict(out=C.c_void_p(0x1004)), INVALID), (dict(stats=(FAKE, None)), INVALID), (dict(stats=(None, FAKE)), INVALID)])
def test_prompt_attention_refusals(lib, kw, status):
    assert prompt(lib, **kw) == status


@pytest.mark.parametrize("kw,status", BOTH + [(dict(missing=i), INVALID) for i in range(6)] + [
    (dict(ws=None), WORKSPACE), (dict(ws_bytes=256), WORKSPACE), (dict(ws=C.c_void_p(0x1010)), INVALID)])
def test_prompt_mass_refusals(lib, kw, status):
    assert mass(lib, **kw) == status


def test_workspace_of_the_utilities(lib):
    need = pk.pikv_prompt_mass_workspace_bytes
    assert need(100, 4, 2, 60) >= 4 * 4 * 100
    assert need(100, 4, 2, 1 << 30) == need(100, 4, 2, 100)          # no sequence is longer than all of them
    assert need(1 << 20, 8, 1, 1 << 20) < 8 * 4 * (1 << 20) + 1024    # blocks enough: not cut
    for bad in ((-1, 4, 2, 60), (100, 0, 2, 60), (100, 4, -1, 60), (100, 4, 2, -1), ((1 << 23) + 1, 4, 2, 60), (100, 257, 2, 60)):
        assert need(*bad) == 0


def desc(**kw):
    return pk.make_desc(**dict(dict(B=2, Hq=8, Hkv=4, D=64, E=8, S=100, dtype=1), **kw))


def pages(**kw):
    return pk.make_pages(**dict(dict(n_pages=50, page=16, Hkv=4, D=64), **kw))


COMMON = [(dict(d=dict(D=16)), UNSUPPORTED), (dict(d=dict(rank=32)), UNSUPPORTED), (dict(d=dict(flags=pk.DESC_8BIT)), INVALID), (dict(d=dict(Hq=6)), INVALID),
          (dict(d=dict(S=0)), INVALID), (dict(d=dict(dtype=3)), INVALID), (dict(d=None), INVALID), (dict(g=None), INVALID), (dict(g=dict(n_pages=0)), INVALID),
          (dict(g=dict(page=8)), INVALID), (dict(g=dict(page=48)), INVALID), (dict(g=dict(page=512)), INVALID), (dict(g=dict(stride_s=56)), INVALID),
          (dict(g=dict(stride_s=68)), INVALID), (dict(g=dict(stride_h=1016)), INVALID), (dict(g=dict(stride_h=960)), INVALID),
          (dict(g=dict(stride_h=32, stride_s=256)), INVALID), (dict(g=dict(stride_h=64, stride_s=192)), INVALID), (dict(g=dict(stride_page=4032)), INVALID),
          (dict(g=dict(stride_page=4100)), INVALID), (dict(g=dict(stride_page=-4096)), INVALID), (dict(g=dict(stride_s=(1 << 23) + 8)), UNSUPPORTED),
          (dict(d=dict(B=0)), 0), (dict(d=dict(B=0), g=dict(stride_h=64, stride_s=256)), 0)]


def given(kw):
    d, g = kw.get("d", {}), kw.get("g", {})
    return None if d is None else C.byref(desc(**d)), None if g is None else C.byref(pages(**g))


@pytest.mark.parametrize("kw,status", COMMON + [(dict(missing=i), INVALID) for i in (0, 1, 2, 3, 5, 6, 7, 9, 10, 11)] + [
    (dict(missing=4), INVALID), (dict(missing=8), INVALID), (dict(k=0), INVALID), (dict(k=9), INVALID), (dict(tokens=-1), INVALID), (dict(tokens=0), 0),
    (dict(tokens=(1 << 23) + 1), UNSUPPORTED), (dict(d=dict(route_rows_per_seq=8)), UNSUPPORTED), (dict(odd=0), INVALID), (dict(odd=1), INVALID),
    (dict(odd=5), INVALID), (dict(odd=6), INVALID), (dict(d=dict(B=1 << 20)), UNSUPPORTED)])
def test_fill_refusals(lib, kw, status):
    at = lambda i: None if kw.get("missing") == i else C.c_void_p(0x1008) if kw.get("odd") == i else FAKE
    K, V, cu, topk, pos, Kp, Vp, table, entry, util, n, slots = (at(i) for i in range(12))
    assert lib.pikv_paged_fill(*given(kw), K, V, kw.get("tokens", 9), cu, topk, kw.get("k", 2), None, pos, Kp, Vp, table, entry, util, n, slots, None) == status


@pytest.mark.parametrize("kw,status", COMMON + [(dict(missing=i), INVALID) for i in range(12)] + [
    (dict(k=0), INVALID), (dict(k=9), INVALID), (dict(me=0), INVALID), (dict(d=dict(route_rows_per_seq=8)), UNSUPPORTED), (dict(odd=0), INVALID),
    (dict(odd=6), INVALID), (dict(odd=7), INVALID), (dict(d=dict(B=1 << 21), k=2), UNSUPPORTED)])
def test_append_refusals(lib, kw, status):
    at = lambda i: None if kw.get("missing") == i else C.c_void_p(0x1008) if kw.get("odd") == i else FAKE
    K, V, topk, ridx, rcnt, pos, Kp, Vp, table, entry, util, n = (at(i) for i in range(12))
    assert lib.pikv_paged_append(*given(kw), K, V, topk, kw.get("k", 2), ridx, rcnt, kw.get("me", 1), pos, Kp, Vp, table, entry, util, n, None) == status


@pytest.mark.parametrize("kw,status", COMMON + [(dict(missing=i), INVALID) for i in range(9)] + [
    (dict(k=0), INVALID), (dict(k=9), INVALID), (dict(combine=2), INVALID), (dict(scale=NAN), INVALID), (dict(scale=INF), INVALID), (dict(cap=-2.0), INVALID),
    (dict(cap=NAN), INVALID), (dict(ws=None), WORKSPACE), (dict(ws_bytes=256), WORKSPACE), (dict(ws=C.c_void_p(0x1010)), INVALID),
    (dict(d=dict(tq=2, route_rows_per_seq=8)), UNSUPPORTED), (dict(d=dict(tq=3)), UNSUPPORTED), (dict(d=dict(tq=4)), UNSUPPORTED), (dict(odd=1), INVALID),
    (dict(odd=2), INVALID), (dict(d=dict(B=1 << 20), k=8), UNSUPPORTED), (dict(unplaced=True, slopes=FAKE), INVALID), (dict(unplaced=True, window=5), INVALID),
    (dict(unplaced=True, prefix=FAKE), INVALID)])
def test_attention_refusals(lib, kw, status):
    at = lambda i: None if kw.get("missing") == i else C.c_void_p(0x1008) if kw.get("odd") == i else FAKE
    q, Kp, Vp, table, n, topk, entry, qpos, y = (at(i) for i in range(9))
    if kw.get("unplaced"):
        entry = qpos = None
    assert lib.pikv_paged_attn(*given(kw), q, Kp, Vp, table, n, topk, FAKE, kw.get("k", 2), kw.get("combine", 0), kw.get("scale", 0.0), kw.get("cap", 0.0),
                               kw.get("slopes"), kw.get("window", 0), kw.get("prefix"), entry, qpos, y, None, None, None, None, kw.get("ws", FAKE),
                               kw.get("ws_bytes", 1 << 40), None) == status


def test_workspace_is_zero_where_the_call_is_refused(lib):
    need = pk.pikv_paged_attn_workspace_bytes
    assert need(desc(), 2) > 0 and need(desc(tq=2), 2) > 0 and need(desc(stride_h=0, stride_s=1), 2) == need(desc(), 2)
    for bad in (desc(D=16), desc(rank=32), desc(flags=pk.DESC_8BIT), desc(tq=3), desc(Hq=6)):
        assert need(bad, 2) == 0
    assert need(desc(), 0) == need(desc(), 9) == 0
    rows = need(desc(B=1, Hq=1, Hkv=1, D=128, E=64, S=1 << 24), 64) / (64 * 130 * 4)
    assert 1 <= rows < 2048 // 64 + 1


def test_layouts_of_pages():
    one = pk.make_pages(7, 32, 4, 64)
    assert (one.stride_page, one.stride_h, one.stride_s) == (8192, 2048, 64)
    slots_first = pk.make_pages(7, 32, 4, 64, stride_h=64, stride_s=256)
    assert (slots_first.stride_page, slots_first.stride_h, slots_first.stride_s) == (8192, 64, 256)
    assert C.sizeof(pk.PikvPages) == 32 and pk.PikvPages.stride_page.offset == 8


def test_pools_may_be_parts_of_a_larger_one(monkeypatch):
    whole = torch.zeros((5, 2, 4, 16, 64), dtype=torch.bfloat16)
    monkeypatch.setattr(torch.Tensor, "is_cuda", True)
    g = pk.make_pages(5, 16, 4, 64, stride_page=2 * 4 * 16 * 64)
    for i in (0, 1):
        assert binding._pool("x", whole[:, i], desc(), g) == whole.data_ptr() + i * 4 * 16 * 64 * 2
    with pytest.raises(ValueError, match="pages take"):
        binding._pool("x", whole[1:, 1], desc(), g)
    with pytest.raises(ValueError, match="pages take"):
        binding._pool("x", whole[:, 0].contiguous(), desc(), g)
    with pytest.raises(ValueError, match="contiguous"):
        binding._pool("x", whole.transpose(-1, -2), desc(), g)


@pytest.mark.parametrize("name", ["pikv_prompt_attn", "pikv_prompt_mass", "pikv_paged_fill", "pikv_paged_append", "pikv_paged_attn"])
def test_the_binding_refuses_host_memory_and_other_types(name):
    d, g, f = desc(), pages(), lambda *shape, t=torch.float32: torch.zeros(shape, dtype=t)
    i32, bf = f(4, t=torch.int32), f(16, t=torch.bfloat16)
    calls = {
        "pikv_prompt_attn": lambda i, s, bf=bf: pk.pikv_prompt_attn(bf, bf if bf.dtype != torch.float16 else f(4), bf, 1, 512, 256, 256, 8, 4, 64, i, 1, 1,
                                                                    None, 0.0, 0.0, s, 0, bf, s, s),
        "pikv_prompt_mass": lambda i, s, bf=bf: pk.pikv_prompt_mass(bf, bf if bf.dtype != torch.float16 else f(4), 1, 512, 256, 8, 4, 64, i, 1, 1, None, 0.0,
                                                                    0.0, s, 0, s, s, s, s),
        "pikv_paged_fill": lambda i, s, bf=bf: pk.pikv_paged_fill(d, g, bf, bf, 1, i, i, 2, s, i, bf, bf, i, i, s, i, i),
        "pikv_paged_append": lambda i, s, bf=bf: pk.pikv_paged_append(d, g, bf, bf, i, 2, i, i, 1, i, bf, bf, i, i, s, i),
        "pikv_paged_attn": lambda i, s, bf=bf: pk.pikv_paged_attn(d, g, bf, bf, bf, i, i, i, s, 2, 0, 0.0, 0.0, s, 0, i, i, i, s, s, s, s, s, s)}
    with pytest.raises(ValueError, match="device memory"):
        calls[name](i32, f(4))
    with pytest.raises(TypeError, match="int32"):
        calls[name](i32.long(), f(4))
    with pytest.raises(TypeError, match="float32"):
        calls[name](i32, f(4, t=torch.float64))
    with pytest.raises(TypeError):
        calls[name](i32, f(4), f(16, t=torch.float16))


@pytest.mark.parametrize("call", [prompt, mass], ids=["attention", "mass"])
def test_strides_and_lengths_beyond_the_offsets_of_the_kernels(lib, call):
    """A row's stride of 2^25 bytes is the largest; none wraps around to one that fits."""
    names = ["q_stride", "k_stride"] + (["v_stride"] if call is prompt else [])
    for name in names:
        assert call(lib, **{name: (1 << 24) + 8}) == UNSUPPORTED
        assert call(lib, dtype=0, **{name: (1 << 23) + 4}) == UNSUPPORTED
        assert call(lib, **{name: 1 << 62}) == UNSUPPORTED


@pytest.mark.parametrize("name", ["stride_s", "stride_h", "stride_page"])
def test_strides_of_pages_beyond_the_offsets_of_the_kernels(lib, name):
    for value in (1 << 41, 1 << 61, 1 << 62):
        args = [FAKE] * 3, [2], [FAKE] * 2, [1], [FAKE] * 7, [None]
        assert lib.pikv_paged_append(*given(dict(g={"stride_page": 1 << 20, name: value})), *sum(args, [])) == UNSUPPORTED


def test_query_rows_of_a_sequence(lib):
    """Up to 1024 over pages, in every call on them."""
    need = pk.pikv_paged_attn_workspace_bytes
    for kw in (dict(Hq=320, Hkv=8, tq=5), dict(Hq=1024, Hkv=8), dict(Hq=1024, Hkv=256), dict(Hq=512, Hkv=1, route_rows_per_seq=512)):
        assert need(desc(**kw), 2) > 0
    for kw in (dict(Hq=1028), dict(Hq=512, Hkv=512), dict(Hq=322), dict(Hq=320, Hkv=8, tq=3), dict(Hq=320, route_rows_per_seq=32)):
        assert need(desc(**kw), 2) == 0
    assert lib.pikv_paged_append(*given(dict(d=dict(Hq=320, tq=5, B=0))), *sum(([FAKE] * 3, [2], [FAKE] * 2, [1], [FAKE] * 7, [None]), [])) == 0


def test_no_launch_of_the_utilities_has_too_many_threads(lib):
    """One head: 2^23 blocks of the sums' last step would be refused by the launch, after the first one has run."""
    one = dict(Hq=1, Hkv=1, q_stride=64, k_stride=64, tokens=1 << 23, max_len=1 << 23)
    assert mass(lib, B=64, **one) == UNSUPPORTED
    assert mass(lib, B=64, ws=None, **dict(one, max_len=(1 << 23) - 64)) == WORKSPACE       # (the next smaller one gets past these checks)
