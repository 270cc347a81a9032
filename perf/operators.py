"""Operators around an 8-bit cache, case by case: their plain forms in torch and the framework's kernels.

Three operators, in the order in which a decode step meets them:

  rope    norms of queries and keys for each head and the position rotation, out of a fused projection
          (pikv_norm_rope)
  quant   the cache held in 8 bits with a scale per block of slots and head: written from dense shards (pikv_quant_pack),
          by the step's new entry (pikv_evict, pikv_quant_append), read back (pikv_quant_read)
  attn    routed attention over that cache (pikv_quant_attn)
"""
import math

import torch

own = False
DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
FORMATS = {"int8": (torch.int8, 127.0), "e4m3": (torch.float8_e4m3fn, 448.0)}      # storage, largest code
EPS = 1e-6

ROPE = dict(kind="rope", T=1, Hq=32, Hkv=8, D=128, R=128, interleaved=False, norm=True, v=True, dtype="bf16", reach=8192)
CACHE = dict(B=1, Hkv=8, D=128, E=16, S=4096, dtype="bf16", format="int8", block=64, fill="full")
PACK = dict(CACHE, kind="pack")
STREAM = dict(CACHE, kind="stream", k=2)
ATTN = dict(CACHE, kind="attn", Hq=32, k=2, per_head=False, tq=1, local=False, scores=False)


def listed():
    return [
        # the token of one sequence: latency
        dict(ROPE, name="rope_token"),
        # a small fp32 model with a partial rotation of neighbouring values; a few drafts of a few sequences
        dict(ROPE, name="rope_drafts_f32", T=37, Hq=6, Hkv=2, D=64, R=32, interleaved=True, dtype="f32", v=False),
        # a long prompt, far into a million tokens of context
        dict(ROPE, name="rope_prompt", T=16384, reach=1 << 20),
        # one sequence streams through full shards: an entry leaves, the new one takes its slot
        dict(STREAM, name="stream_one", E=4, S=1024, block=16),
        # a batch of a small fp32 model, odd shard length
        dict(STREAM, name="stream_batch_f32", B=16, Hkv=4, D=64, E=4, S=777, dtype="f32", format="e4m3"),
        # ragged shards of odd length written after a prompt and read back
        dict(PACK, name="pack_ragged_f32", B=3, Hkv=4, D=64, E=5, S=1501, dtype="f32", format="e4m3", block=32, fill="ragged"),
        # the shards of a batch of long prompts
        dict(PACK, name="pack_prompts", B=8),
        # the smallest model: one routing decision per (token, head)
        dict(ATTN, name="attn_tiny_per_head", Hq=4, Hkv=4, D=64, E=4, S=256, per_head=True, dtype="f32", block=16, scores=True),
        # 128K tokens of context over 16 shards, one sequence, with the raw scores for the utility update
        dict(ATTN, name="attn_long_gqa", S=8192, k=4, scores=True),
        # 8 draft tokens share every load of that cache
        dict(ATTN, name="attn_draft8", Hq=256, S=8192, k=4, tq=8, format="e4m3"),
        # a serving batch of sequences of different lengths, one kv head per query head
        dict(ATTN, name="attn_ragged_mha", B=8, Hkv=32, fill="ragged", format="e4m3", block=32, local=True),
        # streaming at the memory bound, full shards; the largest
        dict(ATTN, name="attn_streaming_mha", B=32, Hkv=32, E=8, S=2048),
    ]


def _logint(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rope", "stream", "pack", "attn", "attn", "attn"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    D = rng.choice([32, 64, 64, 128, 128, 128])
    if kind == "rope":
        Hkv = rng.choice([1, 2, 4, 8, 16])
        c = dict(ROPE, T=_logint(rng, 1, 16384), Hkv=Hkv, Hq=Hkv * rng.choice([1, 2, 3, 4, 7, 8]), D=D, R=D // rng.choice([1, 1, 2]),
                 interleaved=rng.random() < 0.4, norm=rng.random() < 0.8, v=rng.random() < 0.6, dtype=dtype,
                 reach=_logint(rng, 256, 1 << 20))
        while c["T"] * (c["Hq"] + 2 * Hkv) * D * (2 if dtype == "bf16" else 4) > 16384 * 48 * 128 * 2:
            c["T"] = c["T"] // 2 + 1
        return c
    c = dict(D=D, dtype=dtype, format=rng.choice(["int8", "e4m3"]), block=rng.choice([16, 32, 64, 128]), E=rng.choice([2, 4, 6, 8, 16]))
    if kind == "pack":
        c = dict(PACK, **c)
        c.update(B=_logint(rng, 1, 8), Hkv=rng.choice([1, 2, 4, 8]), S=_logint(rng, 100, 4096), fill=rng.choice(["full", "ragged", "ragged"]))
        return c
    if kind == "stream":
        c = dict(STREAM, **c)
        c.update(B=_logint(rng, 1, 16), Hkv=rng.choice([1, 2, 4, 8]), S=_logint(rng, 100, 1024), k=rng.randint(1, 2))
        return c
    c = dict(ATTN, **c)
    G = rng.choice([1, 1, 2, 3, 4, 4, 7, 8, 16])
    c.update(B=_logint(rng, 1, 32), Hkv=rng.choice([1, 2, 4, 8, 16, 32] if G == 1 else [1, 2, 4, 8]), S=_logint(rng, 100, 8192),
             k=rng.randint(1, min(4, c["E"])), fill=rng.choice(["full", "ragged", "ragged"]), local=rng.random() < 0.3)
    c["Hq"] = G * c["Hkv"]
    c["scores"] = rng.random() < 0.4
    if G in (2, 4, 8) and rng.random() < 0.3:
        c["tq"] = rng.choice([2, 4, 5])
        c["Hq"] *= c["tq"]
        c["scores"] = False              # (of drafts they are the library's own, in its order of rows)
    elif rng.random() < 0.2:
        c["per_head"] = True
    heads = c["Hq"] if c["per_head"] else c["Hkv"]
    while c["B"] > 1 and (c["B"] * heads * c["k"] * c["S"] * D > 32 * 32 * 2 * 2048 * 128 or
                          c["B"] * c["E"] * c["Hkv"] * c["S"] * D > 32 * 8 * 32 * 2048 * 128):
        c["B"] //= 2
    return c


def _mean_fill(c):
    return c["S"] if c["fill"] == "full" else 0.55 * c["S"]


def work(case):
    """rope: rows in and out.  pack: dense rows in, codes out, codes in, dense rows out.  stream: utilities of the selected
    shards, the new rows, codes in, dense rows out.  attn: codes and scales of the selected shards, queries, outputs."""
    c = case
    es, D = (4 if c["dtype"] == "f32" else 2), c["D"]
    if c["kind"] == "rope":
        rows = c["T"] * (c["Hq"] + c["Hkv"] * (2 if c["v"] else 1))
        return {"bytes": 2 * rows * D * es + 4 * c["T"] + 2 * c["R"], "flops": rows * D * 8}
    cells = 2 * c["B"] * c["E"] * c["Hkv"] * _mean_fill(c) * D
    if c["kind"] == "pack":
        return {"bytes": cells * (2 * es + 2), "flops": 3 * cells}
    if c["kind"] == "stream":
        new = 2 * c["B"] * c["k"] * c["Hkv"] * D
        return {"bytes": cells * (es + 1) + c["B"] * c["k"] * c["S"] * 4 + new * (es + 1), "flops": cells}
    heads = c["B"] * c["Hq"]
    read = (heads if c["per_head"] else c["B"] * c["Hkv"]) * c["k"] * _mean_fill(c)
    bytes_ = 2 * read * (D + 4 / c["block"]) + heads * D * (es + 4) + heads * 8
    if c["scores"]:
        bytes_ += heads * c["k"] * _mean_fill(c) * 4
    return {"bytes": bytes_, "flops": 4 * heads * c["k"] * _mean_fill(c) * D}


# ------------------------------------------------------------------------------- inputs
def _normal(shape, gen, dtype=torch.float32, std=1.0):
    return (torch.randn(shape, generator=gen, device=DEV) * std).to(dtype)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    t, D = DTYPES[c["dtype"]], c["D"]
    s = dict(case=c)
    if own:
        import paper_2508_06526_amd as pk
        s["pk"] = pk
        pk.load_library()
    if c["kind"] == "rope":
        T, Hq, Hkv = c["T"], c["Hq"], c["Hkv"]
        s["x"] = _normal((T, (Hq + Hkv * (2 if c["v"] else 1)) * D), gen, t)
        s["w_q"], s["w_k"] = ((1 + _normal((D,), gen, std=0.1)).to(t) for _ in range(2)) if c["norm"] else (None, None)
        s["positions"] = torch.randint(0, c["reach"], (T,), generator=gen, device=DEV, dtype=torch.int32)
        s["inv_freq"] = (10000.0 ** (-torch.arange(0, c["R"], 2, dtype=torch.float64) / c["R"])).float().to(DEV)
        s["q"], s["key"] = torch.zeros((T, Hq, D), device=DEV, dtype=t), torch.zeros((T, Hkv, D), device=DEV, dtype=t)
        s["value"] = torch.zeros((T, Hkv, D), device=DEV, dtype=t) if c["v"] else None
        return s
    B, E, Hkv, S, block = c["B"], c["E"], c["Hkv"], c["S"], c["block"]
    i32 = dict(device=DEV, dtype=torch.int32)
    if c["fill"] == "full":
        s["n_valid"] = torch.full((B, E), S, **i32)
    else:                                # an empty shard now and then, a full one now and then
        u = torch.rand((B, E), generator=gen, device=DEV)
        s["n_valid"] = (S * (1.1 * u - 0.05)).int().clamp_(0, S)
    storage = FORMATS[c["format"]][0]
    blocks = (S + block - 1) // block
    for name in ("K", "V"):
        s[name] = torch.zeros((B, E, Hkv, S, D), device=DEV, dtype=storage)
        s[name + "_scales"] = torch.zeros((B, E, Hkv, blocks), device=DEV)
        if c["kind"] in ("pack", "stream"):
            s[name + "_dense"] = torch.zeros((B, E, Hkv, S, D), device=DEV, dtype=t)     # read back
        if c["kind"] == "pack":
            s[name + "_rows"] = torch.zeros((B, E, Hkv, S, D), device=DEV, dtype=t)
        for b in range(B):               # a large cache sequence by sequence
            rows = _normal((E, Hkv, S, D), gen) * torch.exp(_normal((E, 1, S, 1), gen, std=0.5))
            if c["kind"] == "pack":
                s[name + "_rows"][b] = rows.to(t)
            else:
                s[name][b], s[name + "_scales"][b] = _quantised(rows.to(t).float(), c)
    if own:
        s["desc"] = pk.make_desc(B, c.get("Hq", Hkv), Hkv, D, E, S, dtype=pk.F32 if c["dtype"] == "f32" else pk.BF16,
                                 route_rows_per_seq=c["Hq"] if c.get("per_head") else 1, tq=c.get("tq", 1))
        s["format"] = pk.QUANT_INT8 if c["format"] == "int8" else pk.QUANT_E4M3
        for name in ("K", "V"):
            s[name + "_tab"] = pk.shard_table(s[name])
            if c["kind"] == "pack":
                s[name + "_rows_tab"] = pk.shard_table(s[name + "_rows"])
            if c["kind"] in ("pack", "stream"):
                s[name + "_dense_tab"] = pk.shard_table(s[name + "_dense"])
    if c["kind"] == "pack":
        return s
    rows = B * (c["Hq"] if c.get("per_head") else 1)
    s["topk"] = torch.rand((rows, E), generator=gen, device=DEV).argsort(1)[:, :c["k"]].int().contiguous()
    if c["kind"] == "stream":
        s["K_new"], s["V_new"] = (_normal((B, Hkv, D), gen, t, std) for std in (1.5, 1.5))
        s["utility"] = (torch.rand((B, E, S), generator=gen, device=DEV) + 0.01) / S
        s["evicted"], s["evicted_cnt"] = torch.zeros((B, E, 1), **i32), torch.zeros((B, E), **i32)
        return s
    Hq, k = c["Hq"], c["k"]
    s["q"] = _normal((B, Hq, D), gen, t)
    s["gates"] = torch.softmax(_normal((rows, k), gen), 1)
    s["y"] = torch.zeros((B, Hq, D), device=DEV)
    s["row_max"], s["row_norm"] = torch.zeros((B, Hq), device=DEV), torch.zeros((B, Hq), device=DEV)
    s["scores"] = torch.zeros((B, Hq, k, S), device=DEV) if c["scores"] else None
    if own:
        s["slot_coef"] = torch.zeros((B, Hq, k, 2), device=DEV)
        s["workspace"] = torch.empty(pk.pikv_quant_attn_workspace_bytes(s["desc"], k), device=DEV, dtype=torch.uint8)
    return s


# --------------------------------------------------------------------------------- passes
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    c, pk = s["case"], s["pk"]
    if c["kind"] == "rope":
        T, row = s["x"].shape
        pk.pikv_norm_rope(s["x"], T, row, c["Hq"], c["Hkv"], c["D"], s["w_q"], s["w_k"], EPS, s["positions"], s["inv_freq"], c["R"],
                          c["interleaved"], s["q"], s["key"], s["value"])
        return _rope_outputs(s)
    d, fmt, block = s["desc"], s["format"], c["block"]
    codes = (s["K_tab"], s["V_tab"], s["K_scales"], s["V_scales"])
    if c["kind"] == "attn":
        pk.pikv_quant_attn(d, fmt, block, s["q"], *codes, s["n_valid"], s["topk"], s["gates"], c["k"],
                           pk.COMBINE_LOCAL if c["local"] else pk.COMBINE_LSE, 0.0, s["y"], s["row_max"], s["row_norm"], s["scores"],
                           s["slot_coef"], s["workspace"])
        return _attn_outputs(s)
    if c["kind"] == "pack":
        pk.pikv_quant_pack(d, fmt, block, s["K_rows_tab"], s["V_rows_tab"], c["S"] * c["D"], c["D"], s["n_valid"], *codes)
    else:
        pk.pikv_evict(d, s["utility"], s["n_valid"], c["S"] - 1, s["topk"], c["k"], s["evicted"], s["evicted_cnt"], 1, False, None, None)
        pk.pikv_quant_append(d, fmt, block, s["K_new"], s["V_new"], s["topk"], c["k"], s["evicted"], s["evicted_cnt"], 1, *codes,
                             s["utility"], s["n_valid"])
    pk.pikv_quant_read(d, fmt, block, *codes, s["n_valid"], s["K_dense_tab"], s["V_dense_tab"], c["S"] * c["D"], c["D"])
    return _cache_outputs(s)


def _rope_outputs(s):
    return {name: s[name] for name in ("q", "key", "value") if s[name] is not None}


def _cache_outputs(s):
    names = ["K_dense", "V_dense", "K_scales", "V_scales"]
    if s["case"]["kind"] == "stream":
        names += ["utility", "n_valid", "evicted_cnt"]
    return {name: s[name] for name in names}


def _attn_outputs(s):
    return {name: s[name] for name in ("y", "row_max", "row_norm", "scores") if s[name] is not None}


def _run_plain(s):
    c = s["case"]
    if c["kind"] == "rope":
        _rope_plain(s)
        return _rope_outputs(s)
    if c["kind"] == "attn":
        _attn_plain(s)
        return _attn_outputs(s)
    live = torch.arange(c["S"], device=DEV) < s["n_valid"][..., None]              # [B, E, S]
    if c["kind"] == "pack":
        block = torch.arange(s["K_scales"].shape[-1], device=DEV) * c["block"] < s["n_valid"][..., None]
        for name in ("K", "V"):
            rows = torch.where(live[:, :, None, :, None], s[name + "_rows"].float(), 0.0)
            codes, scales = _quantised(rows, c)
            s[name].copy_(torch.where(live[:, :, None, :, None], codes.view(torch.int8), s[name].view(torch.int8)).view(codes.dtype))
            s[name + "_scales"].copy_(torch.where(block[:, :, None], scales, s[name + "_scales"]))
    else:
        _stream_plain(s)
    for name in ("K", "V"):
        values = (s[name].float() * _per_slot(s[name + "_scales"], c)).to(DTYPES[c["dtype"]])
        s[name + "_dense"].copy_(torch.where(live[:, :, None, :, None], values, s[name + "_dense"]))
    return _cache_outputs(s)


def _rope_plain(s):
    c = s["case"]
    T, D, R = c["T"], c["D"], c["R"]
    heads = s["x"].reshape(T, -1, D).float()
    q, key, value = heads.split([c["Hq"], c["Hkv"], c["Hkv"] if c["v"] else 0], 1)
    angle = s["positions"].double()[:, None, None] * s["inv_freq"].double()        # 64 bits: far positions
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    for rows, weight, out in ((q, s["w_q"], s["q"]), (key, s["w_k"], s["key"])):
        if weight is not None:
            rows = rows / torch.sqrt((rows * rows).mean(-1, keepdim=True) + EPS) * weight.float()
        turn, rest = rows[..., :R], rows[..., R:]
        if c["interleaved"]:
            a, b = turn[..., 0::2], turn[..., 1::2]
            turn = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        else:
            a, b = turn[..., :R // 2], turn[..., R // 2:]
            turn = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        out.copy_(torch.cat([turn, rest], -1))
    if c["v"]:
        s["value"].copy_(value)


def _needed_scale(most, c):
    """The smallest power of two, 2^-126 at the least, that brings magnitudes up to `most` (fp32) within the largest code."""
    limit = FORMATS[c["format"]][1]
    m, x = torch.frexp(most)
    lm, lx = math.frexp(limit)
    e = (x - lx + (m > lm).int()).clamp(min=-126)
    return ((e + 127) << 23).view(torch.float32)


def _coded(x, c):
    """x / scale (exact: scales are powers of two), rounded to nearest, ties to even."""
    return (torch.round(x) if c["format"] == "int8" else x).to(FORMATS[c["format"]][0])


def _quantised(rows, c):
    """Codes and scales of rows [..., S, D] (fp32)."""
    S, block = rows.shape[-2], c["block"]
    most = rows.abs().amax(-1)
    most = torch.nn.functional.pad(most, (0, -S % block)).unflatten(-1, (-1, block)).amax(-1)
    scales = _needed_scale(most, c)
    return _coded(rows / _per_slot(scales, c), c), scales


def _per_slot(scales, c):
    return scales.repeat_interleave(c["block"], -1)[..., :c["S"], None]


def _stream_plain(s):
    """Per selected shard: the entry of the least utility (of equal ones the higher slot) leaves, the new one takes its slot."""
    c = s["case"]
    B, E, Hkv, S, D, k, block = (c[n] for n in ("B", "E", "Hkv", "S", "D", "k", "block"))
    b, e = torch.arange(B, device=DEV)[:, None], s["topk"].long()                  # [B, 1], [B, k]
    slot = S - 1 - s["utility"][b, e].flip(-1).argmin(-1)                          # (full shards)
    s["evicted"][b, e, 0] = slot.int()
    s["evicted_cnt"].zero_()
    s["evicted_cnt"][b, e] = 1
    at = slot // block
    slots = at[..., None] * block + torch.arange(block, device=DEV)                # [B, k, block]
    inside = slots < S
    slots = slots.clamp(max=S - 1)
    others = (inside & (slots != slot[..., None])).any(-1)[..., None]              # [B, k, 1]
    h = torch.arange(Hkv, device=DEV)
    for name in ("K", "V"):
        codes, scales, new = s[name], s[name + "_scales"], s[name + "_new"].float()[:, None]       # new [B, 1, Hkv, D]
        old = scales[b[..., None], e[..., None], h, at[..., None]]                 # [B, k, Hkv]
        need = _needed_scale(new.abs().amax(-1), c).expand(B, k, Hkv)
        scale = torch.where(others, torch.maximum(old, need), need)
        where = (b[..., None, None], e[..., None, None], h[:, None], slots[:, :, None])
        held = codes[where].float() * (old / scale)[..., None, None]               # [B, k, Hkv, block, D]
        held = torch.where((slots == slot[..., None])[:, :, None, :, None], new[..., None, :] / scale[..., None, None], held)
        codes.view(torch.int8)[where] = _coded(held, c).view(torch.int8)           # (slots clamped at the end carry the last slot's)
        scales[b[..., None], e[..., None], h, at[..., None]] = scale
    s["utility"][b, e, slot] = 0.0
    s["n_valid"][b, e] = S


def _selected(s, name, scaled=True):
    """Dense fp32 rows that every group of query rows reads: [B, groups, k, S, D], a group being a kv head or (per-head
    routing) a query head."""
    c = s["case"]
    B, Hkv, k = c["B"], c["Hkv"], c["k"]
    if c["per_head"]:
        b = torch.arange(B, device=DEV)[:, None, None]
        h = (torch.arange(c["Hq"], device=DEV) // (c["Hq"] // Hkv))[:, None]
    else:
        b, h = torch.arange(B, device=DEV)[:, None, None], torch.arange(Hkv, device=DEV)[:, None]
    e = s["topk"].long().reshape(B, -1, k)                                         # [B, 1 or Hq, k]
    return s[name].view(torch.int8)[b, e, h].view(s[name].dtype).float() * _per_slot(s[name + "_scales"][b, e, h], c)


def _grouped(t, c):
    """[B, Hq, ...] in the tokens' order (drafts outermost) -> [B, groups, rows, ...]."""
    if c["per_head"]:
        return t.unflatten(1, (c["Hq"], 1))
    tq, Hkv = c["tq"], c["Hkv"]
    t = t.unflatten(1, (tq, Hkv, c["Hq"] // tq // Hkv)).transpose(1, 2)
    return t.flatten(2, 3)


def _ungrouped(t, c):
    if c["per_head"]:
        return t.flatten(1, 2)
    tq, Hkv = c["tq"], c["Hkv"]
    return t.unflatten(2, (tq, c["Hq"] // tq // Hkv)).transpose(1, 2).flatten(1, 3)


def _attn_plain(s):
    c = s["case"]
    B, S, k = c["B"], c["S"], c["k"]
    K, V = _selected(s, "K"), _selected(s, "V")                                    # [B, g, k, S, D]
    q = _grouped(s["q"].float(), c)                                                # [B, g, r, D]
    sc = (q[:, :, None] @ K.transpose(-1, -2)) / math.sqrt(c["D"])                 # [B, g, k, r, S]
    e = s["topk"].long().reshape(B, -1, k)
    n = s["n_valid"].long().gather(1, e.flatten(1)).reshape(e.shape)[..., None, None]      # [B, 1 or Hq, k, 1, 1]
    live = torch.arange(S, device=DEV) < n
    if s["scores"] is not None:
        s["scores"].copy_(torch.where(_ungrouped((live.expand(sc.shape)).transpose(2, 3), c), _ungrouped(sc.transpose(2, 3), c), s["scores"]))
    sc = torch.where(live, sc, -math.inf)
    gate = s["gates"].reshape(e.shape)[..., None]                                  # [B, 1 or Hq, k, 1]
    top = sc.amax(-1)                                                              # [B, g, k, r]
    row_max = top.amax(2)
    used = (n[..., 0] > 0).expand(top.shape)
    if c["local"]:
        p = torch.exp(sc - torch.where(used, top, 0.0)[..., None])
        mass = p.sum(-1)
        norm = (gate * used).sum(2)
        weight = torch.where(used, gate / torch.where(used, mass, 1.0), 0.0)
    else:
        p = torch.exp(sc - torch.where(row_max > -math.inf, row_max, 0.0)[:, :, None, :, None])
        norm = (gate * p.sum(-1)).sum(2)
        weight = gate.expand(top.shape)
    y = ((p * weight[..., None]) @ V).sum(2) / torch.where(norm > 0, norm, 1.0)[..., None]
    s["y"].copy_(_ungrouped(y, c))
    s["row_max"].copy_(_ungrouped(row_max, c))
    s["row_norm"].copy_(_ungrouped(norm.expand(row_max.shape), c))


# ---------------------------------------------------------------------------- 64-bit values
def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "rope":
        return _rope_exact(s)
    if c["kind"] == "attn":
        return _attn_exact(s)
    return _cache_exact(s)


def _rope_exact(s):
    c = s["case"]
    T, D, R, Hq, Hkv = c["T"], c["D"], c["R"], c["Hq"], c["Hkv"]
    x = s["x"].double().view(T, -1, D)
    first = torch.arange(R // 2, device=DEV) * (2 if c["interleaved"] else 1)
    second = first + (1 if c["interleaved"] else R // 2)
    turn = torch.polar(torch.ones((T, R // 2), device=DEV, dtype=torch.float64),
                       s["positions"].double().outer(s["inv_freq"].double()))
    out = {}
    for name, rows, weight in (("q", x[:, :Hq], s["w_q"]), ("key", x[:, Hq:Hq + Hkv], s["w_k"])):
        z = rows.clone()
        if weight is not None:
            z *= (z.square().sum(-1, keepdim=True) / D + EPS).rsqrt() * weight.double()
        turned = torch.complex(z[..., first], z[..., second]) * turn[:, None]
        z[..., first], z[..., second] = turned.real, turned.imag
        out[name] = z
    if c["v"]:
        out["value"] = x[:, Hq + Hkv:]
    return out


def _exact_scale(most, c):
    limit = FORMATS[c["format"]][1]
    e = torch.ceil(torch.log2(most.double().clamp(min=2.0 ** -140) / limit))
    e += (most > limit * torch.exp2(e)).double()                # the logarithm's own rounding, either way
    e -= (most <= limit * torch.exp2(e - 1)).double()
    return torch.exp2(e.clamp(min=-126))


def _exact_value(v, scale, c):
    """The value that v is held as."""
    v = v / scale
    if c["format"] == "int8":
        return torch.round(v) * scale
    step = torch.exp2((torch.frexp(v)[1] - 1).clamp(min=-6).double() - 3)          # 4 significant bits, 2^-9 at the least
    return torch.round(v / step) * step * scale


def _cache_exact(s):
    c = s["case"]
    B, E, S, block = c["B"], c["E"], c["S"], c["block"]
    out = {}
    if c["kind"] == "pack":
        for name in ("K", "V"):
            dense, scales = s[name + "_dense"].clone(), s[name + "_scales"].clone()
            for b in range(B):
                for e in range(E):
                    n = int(s["n_valid"][b, e])
                    whole = n // block * block
                    for lo, hi, rows in ((0, whole, block), (whole, n, n - whole)):
                        if hi > lo:
                            x = s[name + "_rows"][b, e, :, lo:hi].double().unflatten(1, (-1, rows))
                            scale = _exact_scale(x.abs().amax((2, 3)), c)
                            scales[b, e, :, lo // block:lo // block + scale.shape[1]] = scale.float()
                            dense[b, e, :, lo:hi] = _exact_value(x, scale[..., None, None], c).flatten(1, 2).to(dense.dtype)
            out[name + "_dense"], out[name + "_scales"] = dense, scales            # (values of the codes are exact in either type)
        return out
    utility, n_valid, cnt = s["utility"].clone(), s["n_valid"].clone(), torch.zeros_like(s["evicted_cnt"])
    value, scales = {}, {}
    for name in ("K", "V"):
        scales[name] = s[name + "_scales"].double()
        value[name] = s[name].double() * scales[name].repeat_interleave(block, -1)[..., :S, None]
    for b in range(B):
        for e in s["topk"][b].tolist():
            u = utility[b, e]
            slot = int((u == u.min()).nonzero()[-1])
            lo = slot // block * block
            hi = min(lo + block, S)
            for name in ("K", "V"):
                rows, new = value[name][b, e, :, lo:hi], s[name + "_new"][b].double()
                scale = _exact_scale(new.abs().amax(-1), c)
                if hi - lo > 1:
                    scale = torch.maximum(scale, scales[name][b, e, :, lo // block])
                rows[:, slot - lo] = new
                rows.copy_(_exact_value(rows, scale[:, None, None], c))
                scales[name][b, e, :, lo // block] = scale
            u[slot] = 0.0
            cnt[b, e] = 1
    for name in ("K", "V"):
        out[name + "_dense"], out[name + "_scales"] = value[name], scales[name]
    out.update(utility=utility, n_valid=n_valid, evicted_cnt=cnt)
    return out


def _attn_exact(s):
    c = s["case"]
    B, Hq, Hkv, D, S, k, block, tq = (c[n] for n in ("B", "Hq", "Hkv", "D", "S", "k", "block", "tq"))
    y = torch.zeros((B, Hq, D), device=DEV, dtype=torch.float64)
    row_max = torch.full((B, Hq), -math.inf, device=DEV, dtype=torch.float64)
    row_norm = torch.zeros((B, Hq), device=DEV, dtype=torch.float64)
    scores = torch.zeros((B, Hq, k, S), device=DEV, dtype=torch.float64) if c["scores"] else None
    model_heads = Hq // tq
    head = torch.arange(Hq, device=DEV) % model_heads // (model_heads // Hkv)       # kv head of a query row
    n, topk = s["n_valid"].tolist(), s["topk"].tolist()
    for b in range(B):
        # (query rows, gates, selection) sharing a routing decision
        rows = [(torch.arange(Hq, device=DEV), b)] if not c["per_head"] else [(torch.tensor([h], device=DEV), b * Hq + h) for h in range(Hq)]
        for at, r in rows:
            q, gates = s["q"][b, at].double(), s["gates"][r].double()
            kv = head[at]
            parts = []
            for j, e in enumerate(topk[r]):
                m = n[b][e]
                if m == 0:
                    continue
                heads = kv.unique()
                entry = lambda name: (s[name][b, e, heads, :m].double() *
                                      s[name + "_scales"][b, e, heads].double().repeat_interleave(block, 1)[:, :m, None])
                K, V = entry("K"), entry("V")
                sc = torch.empty((len(at), m), device=DEV, dtype=torch.float64)
                for i, hk in enumerate(heads.tolist()):
                    mine = kv == hk
                    sc[mine] = q[mine] @ K[i].T * D ** -0.5
                if scores is not None:
                    scores[b, at, j, :m] = sc
                parts.append((gates[j], sc, heads, V))
            if not parts:
                continue
            top = torch.stack([sc.amax(1) for _, sc, _, _ in parts]).amax(0)
            row_max[b, at] = top
            if c["local"]:
                total = sum(g for g, _, _, _ in parts)
                weights = [g / total * torch.softmax(sc, 1) for g, sc, _, _ in parts]
                row_norm[b, at] = total
            else:
                raw = [g * torch.exp(sc - top[:, None]) for g, sc, _, _ in parts]
                total = sum(w.sum(1) for w in raw)
                weights = [w / total[:, None] for w in raw]
                row_norm[b, at] = total
            for w, (_, _, heads, V) in zip(weights, parts):
                for i, hk in enumerate(heads.tolist()):
                    mine = kv == hk
                    y[b, at[mine]] += w[mine] @ V[i]
    out = {"y": y, "row_max": row_max, "row_norm": row_norm}
    if scores is not None:
        out["scores"] = scores
    return out
