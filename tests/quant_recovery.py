"""What an entry that takes a freed slot does to its block's scale, in numpy, written from the definition: beside
quant_reference.append, which holds wherever the entry that leaves was not the one that kept the scale up."""
import math

import numpy as np

import quant_reference as ref


def append(new, slot, n, cnt, fmt, block, codes, scales, S):
    """quant_reference.append with a scale that comes down again: where the slot held an entry that has left, and what stays needs
    an eighth of the scale or less, the block takes the scale that it needs (exact for the codes it holds)."""
    lo = slot // block * block
    others = [s for s in range(lo, min(lo + block, min(S, n + max(cnt, 1)))) if s != slot]
    before = codes.copy()
    old = scales[:, slot // block].astype(np.float64)
    ref.append(new, slot, n, cnt, fmt, block, codes, scales, S)
    if not others or cnt < 1:
        return
    for h in range(new.shape[0]):
        top = np.abs(ref.decode(before[h, slot], fmt)).max()
        need = ref.needed_scale(np.abs(new[h]).max(), fmt)
        if math.isnan(old[h]) or math.isnan(need) or need > old[h] / 8 or not top > ref.LIMIT[fmt] / 8:
            continue
        rest = np.abs(ref.decode(before[h, others], fmt)).max() * old[h]
        scale = max(need, ref.needed_scale(rest, fmt))
        if scale <= old[h] / 8:
            codes[h, others] = ref.encode(ref.decode(before[h, others], fmt) * (old[h] / scale), fmt)
            codes[h, slot] = ref.encode(new[h] / scale, fmt)
            scales[h, slot // block] = scale
