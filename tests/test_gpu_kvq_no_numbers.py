"""Blocks of a stored cache that hold no number in some channel (easyspec_kvq_select): behind all others, whatever the query."""
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


def score(queries, lo, hi):
    """Query heads [G][hd] of a KV head on a block's bounds, as the header has it: None for NaN."""
    best = None
    for q in queries:
        terms = [float(x) * float(h if x > 0 else l) for x, l, h in zip(q, lo, hi)]
        s = math.nan if any(math.isnan(t) for t in terms) or {math.inf, -math.inf} <= set(terms) else math.fsum(terms)
        if not math.isnan(s) and (best is None or s > best):
            best = s
    return best


def expected(queries, bounds, held, first, last, n_select):
    scores = [score(queries, *bounds[j]) for j in range(held)]
    kept = [j for j in range(held) if j < first or j >= held - last]
    others = [j for j in range(held) if j not in kept]
    others.sort(key=lambda j: (scores[j] is None, 0.0 if scores[j] is None else -scores[j], j))
    chosen = sorted((kept + others)[:n_select])
    return chosen + [-1] * (n_select - len(chosen))


@pytest.mark.parametrize("heads,hd", [((4, 2), 64), ((7, 1), 128), ((2, 2), 128)])
def test_a_block_without_a_number_goes_last(es, heads, hd):
    import torch
    Hq, H = heads
    g = np.random.default_rng(hd + Hq)
    S = 6 * 64 + 1                                                 # the last block holds one slot
    k = g.normal(0, 1, (1, 1, H, S, hd)).astype(np.float32)
    k[0, 0, :, 64:128, 40] = np.nan                                # block 1: nothing in channels 32 .. 63
    k[0, 0, :, 130, 3] = np.inf                                    # block 2: one slot of many
    k[0, 0, :, 256:320, 8] = 1e4                                   # block 4: the highest scores where q_8 > 0
    k[0, 0, 0, 384, hd - 1] = -np.inf                              # block 6, KV head 0: its only slot
    cache = K.Cache(es, 1, 1, H, S, hd, "fp32")
    kk = K.dev(k)
    es.easyspec_kvq_store(kk, kk, cache.layout, S, [0], [S], [0], [S], cache.c, K.stream())
    torch.cuda.synchronize()
    bounds = cache.bounds.double().cpu().numpy()[0, 0]
    assert np.isposinf(bounds[:, 1, 0, 32:64]).all() and np.isneginf(bounds[:, 1, 1, 32:64]).all() and np.isfinite(bounds[:, 2]).all()
    assert np.isposinf(bounds[0, 6, 0, -1]) and np.isfinite(bounds[1:, 6]).all()
    q = np.stack([K.queries(1, 1, 1, Hq, hd), np.abs(K.queries(2, 1, 1, Hq, hd)), -np.abs(K.queries(3, 1, 1, Hq, hd))])
    q = np.concatenate([q, q * (np.arange(hd) % 32 != 8), q * (np.arange(hd) // 32 != 1)])      # ... and with zeros in those channels
    for one in q:
        x = K.dev(one.astype(np.float32))
        for first, last, n_select in ((0, 0, 1), (0, 0, 5), (0, 0, 6), (0, 0, 7), (2, 0, 3), (0, 1, 4), (1, 1, 2)):
            got = K.select(cache, x, [1], [S], first, last, n_select).cpu().numpy()[0, 0]
            for h in range(H):
                own = one[0, 0, h * Hq // H:(h + 1) * Hq // H].astype(np.float64)
                assert got[h].tolist() == expected(own, bounds[h], 7, first, last, n_select), (h, first, last, n_select)
                if first == last == 0 and n_select <= 5:
                    assert 1 not in got[h] and not (h == 0 and 6 in got[h])


def test_what_is_read_without_such_a_block_is_finite(es):
    import torch
    k = np.random.default_rng(5).normal(0, 1, (1, 1, 1, 320, 64)).astype(np.float32)
    v = np.random.default_rng(6).normal(0, 1, k.shape).astype(np.float32)
    k[0, 0, 0, 64:128, 7] = np.nan
    cache = K.Cache(es, 1, 1, 1, 320, 64, "fp32")
    es.easyspec_kvq_store(K.dev(k), K.dev(v), cache.layout, 320, [0], [320], [0], [320], cache.c, K.stream())
    q = K.dev(K.queries(5, 1, 1, 4, 64))
    blocks = K.select(cache, q, [1], [320], 0, 1, 4)
    torch.cuda.synchronize()
    assert blocks[0, 0, 0].tolist() == [0, 2, 3, 4]
    out = K.attend(cache, q, [1], [320], blocks)
    assert bool(out.isfinite().all())
    K.check_attention(cache, q, [1], [320], out, blocks)
    assert bool(K.attend(cache, q, [1], [320]).isnan().all())
