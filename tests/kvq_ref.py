"""Plain 64-bit implementations of the operators on caches held in 4 bits and of sampling, for their tests."""
import math

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 64


def encode(x):
    """float [..][hd] -> (codes [..][hd / 2], scales [..][hd / 32]) uint8, by the definition: distances to the eight magnitudes."""
    x = np.asarray(x, np.float64)
    g = x.reshape(x.shape[:-1] + (-1, 32))
    with np.errstate(all="ignore"):
        top = np.abs(g).max(-1)
        power = np.where(top > 0, np.frexp(top)[1] - 3.0, -120.0)        # floor(log2(top)) - 2
        power = np.where(np.isfinite(top), np.maximum(power, -120), 128).astype(np.int64)
        a = np.minimum(np.abs(g) * np.ldexp(1.0, -power)[..., None], 6.0)
        far = np.abs(a[..., None] - E2M1)
        code = np.zeros(a.shape, np.uint8)
        best = np.full(a.shape, np.inf)
        for c in (0, 2, 4, 6, 1, 3, 5, 7):                               # half-way the even code stays
            nearer = far[..., c] < best
            code, best = np.where(nearer, c, code), np.where(nearer, far[..., c], best)
        code = code + 8 * np.signbit(g)
        code = np.where(np.isfinite(top)[..., None], code, 0).astype(np.uint8).reshape(x.shape)
    return code[..., 0::2] | (code[..., 1::2] << 4), (power + 127).astype(np.uint8)


def decode(codes, scales):
    """-> float64 [..][hd]; a scale of 255: NaN"""
    c = np.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[:-1] + (-1,))
    x = np.where(c >= 8, -1.0, 1.0) * E2M1[c & 7]
    unit = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return x * np.repeat(unit, 32, -1)


def bounds_of(keys):
    """keys [slots][hd] -> [2][hd], NaN passed over"""
    lo = np.fmin.reduce(keys, 0, initial=np.inf)
    hi = np.fmax.reduce(keys, 0, initial=-np.inf)
    return np.stack((lo, hi))


def attention_row(q, k, v):
    """One query head of one token over the slots it sees, float64: (result, bound on what fp32 arithmetic may be off by).  The bound:
    the scores' products and additions, (hd + 3) u sum|q||k| / sqrt(hd) (twice: numerator and sum), the exponential's argument
    and value, (range + 4) u (twice), the running sums and their rescalings, (slots + 32) u (twice); each relative to a weight, u = 2^-24.
    The three bf16 terms of a probability leave 2^-24 of it: one u, in the constants.  The five 6-bit terms of a query leave 2^-24 of the largest
    magnitude m of 32 neighbouring channels (scales 2^-5 apart, the first one's places worth a quarter where m is 2 .. 4: an eighth 2^-20 of the scale,
    at most 2^-24 m): 2 u sum m |k| / sqrt(hd)."""
    hd, u = q.shape[0], 2.0 ** -24
    if k.shape[0] == 0:
        return np.zeros(hd), np.zeros(hd)
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    with np.errstate(all="ignore"):
        s = k @ q / math.sqrt(hd)
        size = (np.abs(k) @ np.abs(q)).max() / math.sqrt(hd)
        e = np.exp(s - s.max())
        p = e / e.sum()
        most = np.repeat(np.abs(q).reshape(-1, 32).max(1), 32)
        left = (np.abs(k) @ most).max() / math.sqrt(hd)
        off = 2 * (hd + 3) * u * size + 2 * u * left + 2 * (s.max() - s.min() + 4) * u + 2 * (len(s) + 32) * u
        return p @ v, off * (p @ np.abs(v)) + 1e-37


def counted(blocks, seen):
    """The entries of a list that count."""
    out, before = [], -1
    for b in (int(x) for x in blocks):
        if b > before and b >= 0 and b * BLOCK < seen:
            out.append(b)
        before = b
    return out


def attention(q, k, v, n_tokens, lens, blocks=None):
    """q [L, T, Hq, hd], k, v [L, B, H, S, hd] float64; blocks [L, T, H, n] or None.  (out, bound)"""
    L, _, Hq, _ = q.shape
    H = k.shape[2]
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    first = 0
    for b, (n, length) in enumerate(zip(n_tokens, lens)):
        for t in range(first, first + n):
            seen = length - n + (t - first) + 1
            for layer in range(L):
                for j in range(Hq):
                    h = j // (Hq // H)
                    slots = np.arange(seen)
                    if blocks is not None:
                        slots = np.array([s for x in counted(blocks[layer, t, h], seen) for s in range(x * BLOCK, min(x * BLOCK + BLOCK, seen))], np.int64)
                    out[layer, t, j], tol[layer, t, j] = attention_row(q[layer, t, j], k[layer, b, h, slots], v[layer, b, h, slots])
        first += n
    return out, tol


def select(q, bounds, n_tokens, lens, keep_first, keep_last, n_select):
    """q [L, T, Hq, hd], bounds [L, B, H, N, 2, hd] -> blocks [L, T, H, n_select]"""
    L, T, Hq, _ = q.shape
    H = bounds.shape[2]
    G = Hq // H
    out = np.full((L, T, H, n_select), -1, np.int32)
    first = 0
    for b, (n, length) in enumerate(zip(n_tokens, lens)):
        for t in range(first, first + n):
            held = (length - n + (t - first) + BLOCK) // BLOCK
            for layer in range(L):
                for h in range(H):
                    x = q[layer, t, h * G:(h + 1) * G].astype(np.float64)[:, None]
                    with np.errstate(all="ignore"):
                        s = (x * np.where(x > 0, bounds[layer, b, h, :held, 1], bounds[layer, b, h, :held, 0])).sum(-1)
                        s = np.fmax.reduce(s, 0)

                    def key(j):
                        forced = j < keep_first or j >= held - keep_last
                        return (0 if forced else 2 if np.isnan(s[j]) else 1, 0.0 if forced or np.isnan(s[j]) else -s[j], j)
                    chosen = sorted(sorted(range(held), key=key)[:n_select])
                    out[layer, t, h, :len(chosen)] = chosen
        first += n
    return out


def sample(logits, u, temperature, top_k, top_p, min_p):
    """One row: (token, kept logits).  Settings are taken as numbers of 32 bits."""
    T, top_p, min_p = (float(np.float32(x)) for x in (temperature, top_p, min_p))
    left = np.full(logits.shape, -np.inf, np.float32)
    words = np.flatnonzero(logits > -np.inf)
    if len(words) == 0 or np.isposinf(logits[words]).any():
        return -1, left
    order = words[np.argsort(-(logits[words] + np.float32(0)), kind="stable")]
    if top_k:
        order = order[:top_k]
    x = logits[order].astype(np.float64)
    mass = np.exp((x - x[0]) / T)
    sums = np.cumsum(mass)
    n = len(order)
    if top_p < 1:
        n = max(1, int(np.searchsorted(np.concatenate([[0.0], sums[:-1]]), top_p * sums[-1], side="left")))
    if min_p > 0:
        n = min(n, int((x - x[0] >= T * math.log(min_p)).sum()))
    left[order[:n]] = logits[order[:n]]
    if u is None:
        return None, left
    u = float(u)
    at = int(np.searchsorted(sums[:n], u * sums[n - 1], side="right")) if u < 1 else n
    weighs = int(np.flatnonzero(np.diff(np.concatenate([[0.0], sums[:n]])) > 0)[-1])       # the last word with a weight
    return int(order[min(at, weighs)]), left
