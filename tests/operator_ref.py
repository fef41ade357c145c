"""Plain 64-bit implementations of the operators on beams and bounded caches, for their tests."""
import math

import numpy as np


def beam_select(logits, scores, ended, n_select, temperature, end_token):
    """One group: logits [W, V] float32, scores [W], ended [W] or None.  (tokens, parents, scores in float64), each [n_select]."""
    W, V = logits.shape
    found = []
    for w in range(W):
        c = float(scores[w])
        if not c > -math.inf:
            continue
        if ended is not None and ended[w]:
            found.append((-c, w, 0.0, end_token))
            continue
        x = logits[w].astype(np.float64)
        x = np.where(np.isnan(x), -np.inf, x)
        top = x.max()
        if not np.isfinite(top):
            continue
        z = (x - top) * (1.0 / temperature)
        s = c + (z - math.log(np.exp(z).sum()))
        for v in np.argsort(-x, kind="stable")[:n_select]:
            if x[v] > -np.inf:
                found.append((-s[v], w, -x[v], int(v)))
    found.sort()
    tokens, parents = np.full(n_select, -1, np.int32), np.full(n_select, -1, np.int32)
    out = np.full(n_select, -np.inf)
    for i, (s, w, _, v) in enumerate(found[:n_select]):
        tokens[i], parents[i], out[i] = v, w, -s
    return tokens, parents, out


def attn_weights(q, k, n_tokens, lens, weights):
    """q [L, T, Hq, hd], k [L, B, H, S, hd], weights [L, B, H, S] or None; float64.  The sums, NaN where nothing is written, and a
    bound on what fp32 arithmetic may be off by: per row (query head of a token) the scores' products and additions,
    (hd + 3) u sum|q||k| / sqrt(hd) (twice: numerator and sum), the exponential's argument and value, (range + 4) u, the running
    sums, a quarter of the slots u; each relative to the probability, u = 2^-24; then the sums over rows and chunks."""
    L, _, Hq, hd = q.shape
    B, H, S = k.shape[1:4]
    G, u = Hq // H, 2.0 ** -24
    out, tol = np.full((L, B, H, S), np.nan), np.zeros((L, B, H, S))
    first = 0
    for b in range(B):
        n, length = int(n_tokens[b]), int(lens[b])
        if n == 0:
            continue
        old = length - n
        for layer in range(L):
            for h in range(H):
                keys = k[layer, b, h, :length].astype(np.float64)
                out[layer, b, h, :length] = 0.0
                if weights is not None:
                    out[layer, b, h, :old] = weights[layer, b, h, :old]
                for t in range(n):
                    seen = old + t + 1
                    for j in range(h * G, h * G + G):
                        x = q[layer, first + t, j].astype(np.float64)
                        s = keys[:seen] @ x / math.sqrt(hd)
                        size = (np.abs(keys[:seen]) @ np.abs(x)).max() / math.sqrt(hd)
                        e = np.exp(s - s.max())
                        p = e / e.sum()
                        out[layer, b, h, :seen] += p
                        off = 2 * (hd + 3) * u * size + 2 * (s.max() - s.min() + 4) * u + (seen / 4 + 8) * u
                        tol[layer, b, h, :seen] += p * off
                tol[layer, b, h, :length] += (n * G + 2) * u * out[layer, b, h, :length] + 1e-37
        first += n
    return out, tol


def kept_slots(weights, length, keep, recent):
    """One (layer, sequence, KV head): the slots that stay, in order."""
    keep = min(keep, length)
    recent = min(recent, keep)
    w = weights[: length - recent].astype(np.float64)
    w = np.where(np.isnan(w), -np.inf, w)
    nan = np.isnan(weights[: length - recent])
    order = sorted(range(length - recent), key=lambda s: (nan[s], -w[s], s))[: keep - recent]
    return np.array(sorted(order) + list(range(length - recent, length)), np.int32)
