"""Plain forms, in 64 bits, of the operators between a prompt and a paged cache: changed scores and masks, attention, utilities, slots.

Errors of a kernel in fp32, from which the tests take their bars.  A: the largest sum of |q_d k_d| * scale of a call.  A product of D terms summed in
fp32 is off by (D + 8) 2^-24 A, a cap adds 2^-21 cap (an exponential, a reciprocal, the scalings), a distance term of size b, added in one
fused step to a score, 2^-24 (A + b) and the slope's own product nothing else.  A weight exp(s - M) is then off by twice that (s and M) and by
2^-22 |s - M| (the argument of the exponential times log2 e, rounded twice) + 2^-22, relative.  Sums of n terms add n 2^-24.  With e the sum of these,
|dy| <= 2 e sum p |v|; weights rounded to bf16 for the product add 2^-8 sum p |v|, rows stored in bf16 2^-8 |y|."""
import numpy as np


def bf16(a):
    """Nearest bf16 values (ties to even), as float32; NaN and infinities stay."""
    bits = np.asarray(a, np.float32).view(np.uint32)
    rounded = ((bits + 0x7fff + ((bits >> 16) & 1)) & np.uint32(0xffff0000)).view(np.float32)
    return np.where(np.isfinite(a), rounded, np.asarray(a, np.float32))


def stored(a, dtype):
    return bf16(a) if dtype == "bf16" else np.asarray(a, np.float32)


def scores(q, k, q_pos, k_pos, scale, cap=0.0, slope=0.0, window=0, prefix=0, positioned=True):
    """[queries, entries] scores of one head in 64 bits, -inf where an entry is not seen; the entries seen."""
    with np.errstate(invalid="ignore", over="ignore"):
        s = (q.astype(np.float64) @ k.astype(np.float64).T) * scale
        if cap > 0:
            s = cap * np.tanh(s / cap)
    far = np.asarray(q_pos, np.int64)[:, None] - np.asarray(k_pos, np.int64)
    pos = np.broadcast_to(np.asarray(k_pos, np.int64), far.shape)
    seen = (pos >= 0) & ((pos < prefix) | ((far >= 0) & ((window <= 0) | (far < window)))) if positioned else np.ones(far.shape, bool)
    s = s - float(slope) * np.abs(far) if slope else s
    return np.where(seen, s, -np.inf), seen


def error_of(A, D, n, cap=0.0, bias=0.0, spread=None):
    """(absolute error of a score, relative error of a weight and of sums of up to n of them)."""
    ds = (D + 8) * 2.0 ** -24 * A + 2.0 ** -21 * cap + 2.0 ** -24 * (A + bias)
    spread = 2 * (min(A, cap) if cap > 0 else A) if spread is None else spread
    return ds, 2 * ds + 2.0 ** -22 * (spread + 1) + n * 2.0 ** -24


def attention(s, v):
    """(rows, row_max, row_norm, sum p |v|) of scores [queries, entries]."""
    top = s.max(1, initial=-np.inf)
    base = np.where(np.isfinite(top), top, 0.0)
    p = np.exp(s - base[:, None])
    norm = p.sum(1)
    p = p / np.where(norm > 0, norm, 1.0)[:, None]
    v = v.astype(np.float64)
    return p @ v, top, norm, p @ np.abs(v)


class Prompts:
    """Packed prompts as numpy arrays, with everything the calls take."""

    def __init__(self, lens, Hq, Hkv, D, dtype, seed=0, std=1.5, cap=0.0, slopes=False, window=0, prefix=None, lead=0, tail=0, scale=0.0):
        rng = np.random.default_rng(seed)
        self.lens, self.Hq, self.Hkv, self.D, self.dtype = list(lens), Hq, Hkv, D, dtype
        self.cu = lead + np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
        self.tokens = int(self.cu[-1]) + tail
        self.q = stored(rng.normal(size=(self.tokens, Hq, D)) * std, dtype)
        self.k = stored(rng.normal(size=(self.tokens, Hkv, D)), dtype)
        self.v = stored(rng.normal(size=(self.tokens, Hkv, D)), dtype)
        self.cap, self.window, self.scale = cap, window, scale
        self.prefix = None if prefix is None else np.asarray(prefix, np.int32)
        self.slopes = None if not slopes else np.exp2(-8.0 * np.arange(1, Hq + 1) / Hq).astype(np.float32)

    def head_scores(self, b, h, upto=None):
        rows = slice(int(self.cu[b]), int(self.cu[b]) + (self.lens[b] if upto is None else min(upto, self.lens[b])))
        pos = np.arange(rows.stop - rows.start)
        g = h // (self.Hq // self.Hkv)
        s, seen = scores(self.q[rows, h], self.k[rows, g], pos, pos, self.scale if self.scale > 0 else self.D ** -0.5, self.cap,
                         0.0 if self.slopes is None else self.slopes[h], self.window, 0 if self.prefix is None else int(self.prefix[b]))
        return rows, g, s, seen

    def magnitude(self):
        """A of the module's text."""
        most = 0.0
        for b in range(len(self.lens)):
            rows = slice(int(self.cu[b]), int(self.cu[b + 1]))
            for h in range(self.Hq):
                if self.lens[b]:
                    most = max(most, float((np.abs(self.q[rows, h]) @ np.abs(self.k[rows, h // (self.Hq // self.Hkv)]).T).max()))
        return most * (self.scale if self.scale > 0 else self.D ** -0.5)

    def errors(self):
        longest = max(self.lens)
        bias = 0.0 if self.slopes is None else float(self.slopes.max()) * longest
        # (of a weight that counts: beyond 2 A below the maximum a distance term leaves less than any bar)
        return error_of(self.magnitude(), self.D, longest, self.cap, min(bias, 40.0))

    def attend(self, upto=None):
        out, top, norm, weight = (np.zeros((self.tokens, self.Hq) + tail) for tail in ((self.D,), (), (), (self.D,)))
        inside = np.zeros(self.tokens, bool)
        for b in range(len(self.lens)):
            for h in range(self.Hq):
                rows, g, s, _ = self.head_scores(b, h, upto)
                inside[rows] = True
                out[rows, h], top[rows, h], norm[rows, h], weight[rows, h] = attention(s, self.v[rows, g])
        return out, top, norm, weight, inside

    def mass(self, row_max, row_norm):
        total = np.zeros(self.tokens)
        for b in range(len(self.lens)):
            for h in range(self.Hq):
                rows, _, s, seen = self.head_scores(b, h)
                norm = row_norm[rows, h].astype(np.float64)[:, None]
                with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
                    p = np.where(seen & (norm != 0), np.exp(s - row_max[rows, h].astype(np.float64)[:, None]) / norm, 0.0)
                total[rows] += p.sum(0)
        return total


def fill(cu, topk, weight, room_of, n_valid, S):
    """Slots [tokens, k] and new counts.  room_of(b, e): the slots that have pages."""
    tokens, k = topk.shape
    slots = np.full((tokens, k), -1, np.int64)
    counts = n_valid.copy()
    for b in range(n_valid.shape[0]):
        for e in range(n_valid.shape[1]):
            mine = []
            for t in range(cu[b], cu[b + 1]):
                places = [j for j in range(k) if topk[t, j] == e]
                if places:
                    mine.append((t, places[0]))
            room = max(min(S, room_of(b, e)) - int(n_valid[b, e]), 0) if n_valid[b, e] >= 0 else 0
            key = lambda at: 0.0 if weight is None else (-np.inf if np.isnan(weight[at[0]]) else float(weight[at[0]]))
            nan = lambda at: weight is not None and np.isnan(weight[at[0]])
            stay = sorted(sorted(mine, key=lambda at: (-key(at), nan(at), at[0]))[:room])
            for i, (t, j) in enumerate(stay):
                slots[t, j] = n_valid[b, e] + i
            if stay:
                counts[b, e] = n_valid[b, e] + len(stay)
    return slots, counts
