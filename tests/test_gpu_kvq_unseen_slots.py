"""Attention over caches in 4 bits: the bits of a token's results do not depend on slots that it does not see, whatever later tokens of its step find there."""
import numpy as np
import pytest

import kvq_gpu as K
import kvq_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def es():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device; none is visible")
    import paper_2502_02493_amd as es
    return es


@pytest.mark.parametrize("heads,hd,n", [((2, 1), 64, 2), ((2, 1), 128, 2), ((4, 1), 128, 4), ((7, 1), 64, 2), ((8, 1), 128, 4), ((8, 1), 64, 16)])
def test_a_later_tokens_score_moves_no_other_rows_reference(es, heads, hd, n):
    """The last slot, which the last token alone sees, from a score among the others' to one far above them: sixteen layers of contexts of 512 slots, of
    which a wave takes two steps or more, the new tokens' behind others."""
    import torch
    L, S, Hq = 16, 512, heads[0]
    g = np.random.default_rng(hd + n)
    cache = K.random_cache(es, hd + n, L, 1, 1, S, hd)
    q = K.queries(hd + n, L, n, Hq, hd)
    out = []
    for size in (0.0, 1.0, 40.0):
        last = g.normal(0, 1, (L, 1, 1, 1, hd)) * 0.1 if size == 0 else size * q[:, None, None, -1:, 0]     # along the last token's first query
        codes, scales = ref.encode(last)
        cache.kc[:, :, :, -1:], cache.ks[:, :, :, -1:] = K.dev(codes), K.dev(scales)
        x = K.dev(q)
        out.append(K.attend(cache, x, [n], [S]))
        torch.cuda.synchronize()
    for other in out[1:]:
        assert torch.equal(other[:, :-1], out[0][:, :-1])
        assert not torch.equal(other[:, -1], out[0][:, -1])
