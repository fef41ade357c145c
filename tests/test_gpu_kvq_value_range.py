"""Attention over caches in 4 bits on large and small values: nothing overflows while the slots times the largest value stay below 2^119,
and small values keep their bits."""
import math

import numpy as np
import pytest

import kvq_gpu as K
from test_gpu_kvq_low_scores import row

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def es():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device; none is visible")
    import paper_2502_02493_amd as es
    return es


def check(es, k, v, q, n, length, unit=1.0):
    hd, Hq = k.shape[-1], q.shape[2]
    cache = K.Cache(es, 1, 1, 1, length, hd).put(k, v)
    out = K.attend(cache, K.dev(q), [n], [length]).double().cpu().numpy()
    assert np.isfinite(out).all()
    keys, values = cache.values()
    for t in range(n):
        seen = length - n + t + 1
        for j in range(Hq):
            want, tol = row(q[0, t, j].astype(np.float64), keys[0, 0, 0, :seen], values[0, 0, 0, :seen])
            err = np.abs(out[0, t, j] - want)
            assert (err <= tol).all(), (t, j, float((err / tol).max()))


@pytest.mark.parametrize("power", [108, 60, 0, -100])
@pytest.mark.parametrize("heads,hd,n", [(1, 128, 1), (4, 64, 1), (8, 128, 1), (7, 64, 3), (8, 128, 4)])
def test_scores_that_rise_slowly(es, heads, hd, n, power):
    """512 slots, two steps a wave: scores of 0, then one in each step 5.3 higher (2^7.65 of the weight), which moves no reference that leaves 8 places of room.
    512 values under 2^109."""
    g = np.random.default_rng(hd + heads + n)
    direction = g.choice([-1.0, 1.0], hd)
    k = np.zeros((1, 1, 1, 512, hd))
    k[0, 0, 0, 256 + 5::32] = direction
    v = g.choice([-1.0, 1.0], k.shape[-1]) * g.uniform(1, 2, k.shape) * 2.0 ** power       # a channel's values have one sign: nothing cancels
    q = np.broadcast_to(direction * 5.3 / math.sqrt(hd), (1, n, heads, hd)).astype(np.float32)
    check(es, k, v, q, n, 512)


@pytest.mark.parametrize("heads,hd", [(1, 64), (8, 128)])
def test_equal_values_at_the_end_of_the_range(es, heads, hd):
    """One slot, and thirty alike: their mean is one of them."""
    g = np.random.default_rng(3)
    for length, value in ((1, 1.5 * 2.0 ** 118), (30, 2.0 ** 114)):
        k, v = np.repeat(g.normal(0, 1, (1, 1, 1, 1, hd)), length, 3), np.full((1, 1, 1, length, hd), value)
        v[..., 1::2] *= -1
        check(es, k, v, K.queries(3, 1, 1, heads, hd), 1, length)


@pytest.mark.parametrize("heads,hd", [(1, 64), (4, 128), (8, 64)])
def test_large_values_of_slots_that_do_not_count(es, heads, hd):
    """Half of the slots, the first of every wave, with values of 2^109 and scores 700 and more below the others': their weights are below 2^-1000."""
    g = np.random.default_rng(hd)
    direction = g.choice([-1.0, 1.0], hd)
    k = g.normal(0, 1, (1, 1, 1, 512, hd)) - np.where(np.arange(512) < 256, 1000 / math.sqrt(hd), 0.0)[:, None] * direction
    v = g.normal(0, 1, k.shape)
    v[0, 0, 0, :256] = 2.0 ** 109 * g.choice([-1.0, 1.0], (256, hd))
    q = np.broadcast_to(direction, (1, 1, heads, hd)).astype(np.float32)
    cache = K.Cache(es, 1, 1, 1, 512, hd).put(k, v)
    out = K.attend(cache, K.dev(q), [1], [512]).double().cpu().numpy()
    keys, values = cache.values()
    scores = keys[0, 0, 0] @ direction / math.sqrt(hd)
    assert scores[256:].max() - scores[:256].max() > 700
    for j in range(heads):
        want, tol = row(q[0, 0, j].astype(np.float64), keys[0, 0, 0, 256:], values[0, 0, 0, 256:])
        assert (np.abs(out[0, 0, j] - want) <= tol).all(), (j, float((np.abs(out[0, 0, j] - want) / tol).max()))
