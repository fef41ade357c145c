"""Attention over caches in 4 bits where steps of slots score far below others: what a slot's weight may be off by goes by its own score."""
import math

import numpy as np
import pytest

import kvq_gpu as K

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def es():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device; none is visible")
    import paper_2502_02493_amd as es
    return es


def row(q, k, v):
    """One query head of one token over the slots it sees, in 64 bits: (result, bound on what fp32 arithmetic may be off by), u = 2^-24.
    A weight relative to the highest is off by d_s of itself:
      its score's products and sums, hd + 6 roundings of sum |q||k_s| / sqrt(hd) (the factor log2(e) / sqrt(hd) two of them), and what five 6-bit terms
      leave of a query, u of the largest magnitude of 32 channels;
      the differences from references on the way to the highest, each within 8 of the score or between two of them: 2 u (distance + 16);
      and the sum of all such roundings enters results with |v_s| and their divisor with |result|.
    Sums, exponentials and rescalings: (slots + 32) u, twice.  Weights below 2^-120 may be lost."""
    hd, u = q.shape[0], 2.0 ** -24
    s = k @ q / math.sqrt(hd)
    p = np.exp(s - s.max())
    p /= p.sum()
    most = np.repeat(np.abs(q).reshape(-1, 32).max(1), 32)
    d = u * ((hd + 6) * (np.abs(k) @ np.abs(q)) + np.abs(k) @ most) / math.sqrt(hd) + 2 * u * (s.max() - s + 16)
    d = np.where(p > 0, d, 0)
    out = p @ v
    size = p @ np.abs(v)
    return out, (p * d) @ np.abs(v) + (p * d).sum() * np.abs(out) + 2 * (len(s) + 32) * u * size + len(s) * 2.0 ** -120 * np.abs(v).max(0) + 1e-37


def low_steps(seed, slots, hd, direction, far, share):
    """Keys of which whole steps of 32 slots lie `far` (in scores, about) below the others."""
    g = np.random.default_rng(seed)
    k = g.normal(0, 1, (slots, hd))
    low = np.repeat(g.random(-(-slots // 32)) < share, 32)[:slots]
    low[:32] = True
    low[-32:] = False
    return k - np.where(low, far / math.sqrt(hd), 0.0)[:, None] * direction    # a query that is about `direction` has a score of about -far


@pytest.mark.parametrize("far", [30.0, 2e3, 1e5, 1e7, 1e30])
@pytest.mark.parametrize("heads,hd,n,length", [((1, 1), 128, 1, 512), ((4, 1), 64, 1, 500), ((8, 1), 128, 1, 512), ((7, 1), 64, 3, 511), ((8, 1), 128, 5, 512), ((4, 1), 128, 1, 9000), ((8, 1), 64, 4, 9000)])
def test_steps_far_below_the_others(es, heads, hd, n, length, far):
    Hq = heads[0]
    L = 1 if length < 1000 else 24                                # enough layers that a wave takes several steps of a long context
    g = np.random.default_rng(length + Hq)
    direction = g.choice([-1.0, 1.0], hd)
    k = np.stack([low_steps(layer + hd, length, hd, direction, far, 0.6) for layer in range(L)])[:, None, None]
    v = g.normal(0, 1, k.shape)
    cache = K.Cache(es, L, 1, 1, length, hd).put(k, v)
    q = (direction * np.abs(g.normal(1, 0.2, (L, n, Hq, hd)))).astype(np.float32)
    out = K.attend(cache, K.dev(q), [n], [length]).double().cpu().numpy()
    keys, values = cache.values()
    for layer in range(0, L, 7):
        for t in range(n):
            seen = length - n + t + 1
            for j in range(Hq):
                want, tol = row(q[layer, t, j].astype(np.float64), keys[layer, 0, 0, :seen], values[layer, 0, 0, :seen])
                err = np.abs(out[layer, t, j] - want)
                assert (err <= tol).all(), (layer, t, j, float((err / tol).max()))
