"""What an entry that takes a freed slot does to its block's scale, and what entries that hold a NaN or an infinity do, in numpy,
written from the definition: beside quant_reference, which holds wherever neither the entry that leaves kept the scale up nor a row
was not finite."""
import math

import numpy as np

import quant_reference as ref

NAN = 0x7fc00000
NO_CODES = (0x80, 0x7f)                # int8, e4m3: the byte of an entry without codes, in all its places


def bits(scales):
    return scales.view(np.uint32)


def kept(word):
    """The scale of a block's codes by the bits of its own: None where none were kept."""
    word = int(word) & 0x7fffffff
    if word < 0x7f800000:
        return float(np.uint32(word).view(np.float32))
    return 2.0 ** ((word & 0xff) - 127) if word >> 8 == NAN >> 8 and word & 0xff else None


def poisoned(scale):
    return NAN | int(np.float32(scale).view(np.uint32)) >> 23


def pack(dense, n_valid, fmt, block, codes, scales):
    """quant_reference.pack; rows that are not finite have no codes and no part in the scale."""
    ref.pack(np.where(np.isfinite(dense).all(-1, keepdims=True), dense, 0.0), n_valid, fmt, block, codes, scales)
    B, E, Hkv, S, _ = dense.shape
    for b, e, h, s in zip(*np.nonzero(~np.isfinite(dense).all(-1))):
        if s < min(n_valid[b, e], S):
            codes[b, e, h, s] = NO_CODES[fmt]
            bits(scales)[b, e, h, s // block] = poisoned(kept(bits(scales)[b, e, h, s // block]))


def append(new, slot, n, cnt, fmt, block, codes, scales, S):
    """quant_reference.append with a scale that comes down again: where the slot held an entry that has left, and what stays needs
    an eighth of the scale or less, the block takes the scale that it needs (exact for the codes it holds).

    Into a freed slot, or a block whose codes were kept, a row that is not finite leaves the other entries their codes: the block's scale
    is a NaN that tells theirs as long as an entry without codes is there."""
    lo = slot // block * block
    others = [s for s in range(lo, min(lo + block, min(S, n + max(cnt, 1)))) if s != slot]
    before, words = codes.copy(), bits(scales)[:, slot // block].copy()
    with np.errstate(invalid="ignore"):
        ref.append(new, slot, n, cnt, fmt, block, codes, scales, S)
    if not others:
        return
    for h in range(new.shape[0]):
        finite, old = np.isfinite(new[h]).all(), kept(words[h])
        need = ref.needed_scale(np.abs(new[h]).max(), fmt) if finite else 2.0 ** -126
        was_poisoned = math.isnan(words[h:h + 1].view(np.float32)[0])
        if cnt < 1 and (old is None or (not was_poisoned and not finite)):
            continue                                                 # as quant_reference has it
        held = before[h, others]
        if old is None:                                              # of a block that kept nothing only the new row is known
            scale, held = need, np.full_like(held, NO_CODES[fmt])
        without = (held == NO_CODES[fmt]).all(-1) if was_poisoned else np.zeros(len(others), bool)
        if old is not None:
            scale = max(need, old)
            rest = np.where(without[:, None], 0.0, ref.decode(np.where(without[:, None], 0, held).astype(np.uint8), fmt)) * old
            top = np.abs(np.nan_to_num(ref.decode(before[h, slot], fmt))).max() if cnt > 0 else 0.0
            enough = max(need, ref.needed_scale(np.abs(rest).max(), fmt))
            if cnt > 0 and finite and enough <= old / 8 and (was_poisoned or top > ref.LIMIT[fmt] / 8):
                scale = enough
            held = np.where(without[:, None], NO_CODES[fmt], ref.encode(rest / scale, fmt).view(np.uint8)).astype(np.uint8)
        codes[h, others] = held
        codes[h, slot] = ref.encode(new[h] / scale, fmt) if finite else NO_CODES[fmt]
        bits(scales)[h, slot // block] = poisoned(scale) if without.any() or not finite else np.float32(scale).view(np.uint32)
