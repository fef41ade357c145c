"""Selection of more than 32 continuations: the bound on a slice's candidates, which slices of every length have to hold to."""
import numpy as np
import pytest

from test_gpu_beam_select import check, es, rows  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("W,V,K,T", [
    (1, 128256, 33, 1.0), (1, 128256, 64, 0.8),       # 256 slices of 501 words
    (2, 128256, 64, 1.0), (3, 100000, 40, 1.0),       # of 1002 and 782
    (4, 128256, 64, 1.0), (6, 152064, 50, 1.2),       # of 2004 and 2001
    (16, 128256, 64, 1.0),                            # of 4008
    (1, 256, 64, 1.0), (1, 257, 33, 1.0), (1, 300, 64, 1.0), (1, 511, 64, 1.0), (1, 512, 64, 1.0), (1, 513, 64, 1.0), (2, 255, 64, 1.0),
    (1, 12290, 64, 1.0),                              # a last slice of few words
])
def test_sizes(es, W, V, K, T):
    logits, scores = rows(W * V + K, 2, W, V)
    check(es, logits, scores, None, K, T)


def test_masks_and_ties_in_short_slices(es):
    logits, scores = rows(91, 4, 2, 128256)
    logits[0] = np.where(np.arange(128256) % 8 < 4, logits[0], -np.inf)       # every second group of four threads without a logit
    logits[1] = np.round(logits[1])
    logits[2, :, 1000:] = -np.inf
    logits[3, 0] = 0.25
    for k in (33, 64):
        check(es, logits, scores, None, k)
