"""Plain 64-bit forms of the operators around the 8-bit cache, in numpy, written from their definitions."""
import math

import numpy as np

LIMIT = {0: 127.0, 1: 448.0}           # largest code: int8, e4m3


def bf16(x):
    """Rounded to bf16 (nearest, ties to even), as float32; the bits of a bf16 tensor are the upper half."""
    bits = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    rounded = ((bits + 0x7fff + ((bits >> 16) & 1)) & 0xffff0000).astype(np.uint32)
    return np.where(np.isnan(x), np.float32(np.nan), rounded.view(np.float32))


def rounded(x, dtype):
    return bf16(x) if dtype == "bf16" else np.asarray(x, np.float32)


# ------------------------------------------------------------------------------ rope
def norm_rope(x, weight, eps, positions, inv_freq, rotary, interleaved):
    """x [tokens, heads, D] float64 -> the same."""
    z = x.copy()
    if weight is not None:
        z = z / np.sqrt((z * z).mean(-1, keepdims=True) + eps) * weight
    angle = positions.astype(np.float64)[:, None] * inv_freq[:rotary // 2].astype(np.float64)
    cos, sin = np.cos(angle)[:, None], np.sin(angle)[:, None]
    i = np.arange(rotary // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)
    out = z.copy()
    out[..., a], out[..., b] = z[..., a] * cos - z[..., b] * sin, z[..., b] * cos + z[..., a] * sin
    return out


# ------------------------------------------------------------------------------ 8 bits
def _e4m3_table():
    value = np.empty(256)
    for code in range(256):
        s, e, m = code >> 7, code >> 3 & 15, code & 7
        v = (m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        value[code] = math.nan if e == 15 and m == 7 else -v if s else v
    return value


E4M3 = _e4m3_table()


def decode(codes, fmt):
    """Bytes -> the values of the codes."""
    return codes.view(np.int8).astype(np.float64) if fmt == 0 else E4M3[codes.view(np.uint8)]


def encode(v, fmt):
    """|v| <= LIMIT -> bytes, nearest, ties to even."""
    if fmt == 0:
        return np.rint(v).astype(np.int8).view(np.uint8)
    grid = E4M3[:127]                                        # ascending; the parity of a code is that of its mantissa
    hi = np.searchsorted(grid, np.abs(v)).clip(0, 126)
    lo = (hi - 1).clip(0)
    to_lo, to_hi = np.abs(v) - grid[lo], grid[hi] - np.abs(v)
    code = np.where(to_lo < to_hi, lo, np.where(to_hi < to_lo, hi, np.where(lo % 2 == 0, lo, hi)))
    return (code + 128 * (v < 0)).astype(np.uint8)


def needed_scale(most, fmt):
    if not np.isfinite(most):
        return math.nan
    e = -126
    while most > LIMIT[fmt] * 2.0 ** e:
        e += 1
    return 2.0 ** e


def quantise_block(rows, fmt, scale=None):
    """rows [slots, D] float64 -> bytes, scale."""
    if scale is None:
        scale = needed_scale(np.abs(rows).max(), fmt)
    if math.isnan(scale):
        return np.zeros(rows.shape, np.uint8), scale
    return encode(rows / scale, fmt), scale


def pack(dense, n_valid, fmt, block, codes, scales):
    """dense [B, E, Hkv, S, D] float64 into codes (bytes) and scales, in place."""
    B, E, Hkv, S, _ = dense.shape
    for b in range(B):
        for e in range(E):
            n = min(int(n_valid[b, e]), S)
            for h in range(Hkv):
                for lo in range(0, n, block):
                    hi = min(lo + block, n)
                    codes[b, e, h, lo:hi], scales[b, e, h, lo // block] = quantise_block(dense[b, e, h, lo:hi], fmt)


def values(codes, scales, fmt, block):
    S = codes.shape[3]
    return decode(codes, fmt) * np.repeat(scales.astype(np.float64), block, -1)[..., :S, None]


def append(new, slot, n, cnt, fmt, block, codes, scales, S):
    """new [Hkv, D] into slot of one shard: codes [Hkv, S, D] bytes, scales [Hkv, blocks], in place; n before, cnt freed slots."""
    live = min(S, n + max(cnt, 1))
    lo = slot // block * block
    others = [s for s in range(lo, min(lo + block, live)) if s != slot]
    for h in range(new.shape[0]):
        scale, old = needed_scale(np.abs(new[h]).max(), fmt), float(scales[h, slot // block])
        if others:
            if math.isnan(old) or math.isnan(scale):
                scale = math.nan
            elif scale > old:
                codes[h, others] = encode(decode(codes[h, others], fmt) * (old / scale), fmt)
            else:
                scale = old
            if math.isnan(scale) and not math.isnan(old):
                codes[h, others] = 0
        codes[h, slot] = 0 if math.isnan(scale) else encode(new[h] / scale, fmt)
        scales[h, slot // block] = scale


# ------------------------------------------------------------------------------ attention
def attend(q, K, V, n_valid, topk, gates, Hkv, local=False, tq=1, per_head=False, scale=None):
    """q [B, Hq, D] in the tokens' order, K and V [B, E, Hkv, S, D], all float64.  y, row_max, row_norm in the tokens' order,
    scores [B, Hq, k, S] (NaN where nothing is) in the order of kv heads, mass [B, E, S] the attention of every entry."""
    B, Hq, D = q.shape
    E, S, k = K.shape[1], K.shape[3], topk.shape[1]
    heads = Hq // tq
    g = heads // Hkv
    scale = 1 / math.sqrt(D) if scale is None else scale
    y, row_max, row_norm = np.zeros((B, Hq, D)), np.full((B, Hq), -np.inf), np.zeros((B, Hq))
    scores, mass = np.full((B, Hq, k, S), np.nan), np.zeros((B, E, S))
    for b in range(B):
        for row in range(Hq):
            t, h = divmod(row, heads)
            hk = h // g
            inner = (hk * tq + t) * g + h % g                # kv head, draft query, head of the group
            r = b * Hq + row if per_head else b
            parts = []
            for j, e in enumerate(topk[r]):
                n = min(int(n_valid[b, e]), S)
                if n > 0:
                    s = K[b, e, hk, :n] @ q[b, row] * scale
                    scores[b, inner, j, :n] = s
                    parts.append((1.0 if gates is None else float(gates[r, j]), e, s, V[b, e, hk, :n]))
            if not parts:
                continue
            M = max(s.max() for _, _, s, _ in parts)
            row_max[b, row] = M
            if local:
                total = sum(w for w, _, _, _ in parts)
                ps = [w / total * np.exp(s - s.max()) / np.exp(s - s.max()).sum() for w, _, s, _ in parts]
            else:
                ps = [w * np.exp(s - M) for w, _, s, _ in parts]
                total = sum(p.sum() for p in ps)
                ps = [p / total for p in ps]
            row_norm[b, row] = total
            for p, (_, e, s, v) in zip(ps, parts):
                y[b, row] += p @ v
                mass[b, e, :len(s)] += p
    return dict(y=y, row_max=row_max, row_norm=row_norm, scores=scores, mass=mass)
