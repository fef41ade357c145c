"""How attention over a cache in 4 bits cuts contexts (easyspec_kvq_attention_workspace_bytes), which is host arithmetic: pieces of a row are a multiple of its size."""
import numpy as np
import pytest

import paper_2502_02493_amd as es


def pieces(n, lens, q_heads, kv_heads, hd, layers=1, n_blocks=0):
    """Pieces of all rows of a layer, of which a row has `hd` sums, a maximum and a weight."""
    layout = es.easyspec_kv_layout(layers, len(n), kv_heads, max(lens + [1]), hd, es.EASYSPEC_DTYPE_BF16)
    need = es.easyspec_kvq_attention_workspace_bytes(layout, n, lens, q_heads, n_blocks)
    assert need >= 0 and need % (layers * kv_heads * (hd * 4 + 8)) == 0
    return need // (layers * kv_heads * (hd * 4 + 8))


@pytest.mark.parametrize("q_heads,kv_heads,hd", [(32, 8, 128), (28, 4, 128), (4, 2, 64), (2, 2, 64)])
def test_short_contexts_are_whole(q_heads, kv_heads, hd):
    for n, lens in (([1], [1]), ([1], [512]), ([16], [512]), ([1, 16, 0, 6], [512, 16, 0, 100]), ([0, 0], [0, 0]), ([0], [1])):
        assert pieces(n, lens, q_heads, kv_heads, hd) == 0
    assert pieces([1], [65536], q_heads, kv_heads, hd, n_blocks=8) == 0
    assert pieces([1], [513], q_heads, kv_heads, hd) > 0


def test_no_more_workgroups_than_the_card_has_cus():
    rng = np.random.default_rng(3)
    for _ in range(300):
        group, kv, layers, n = int(rng.choice([1, 2, 4, 7, 8])), int(rng.choice([1, 2, 4, 8, 32, 300])), int(rng.choice([1, 1, 4, 32])), int(rng.integers(1, 17))
        length = int(max(n, np.exp(rng.uniform(0, np.log(65536)))))
        rows = n * group
        p = pieces([n], [length], group * kv, kv, 64, layers)
        assert p % rows == 0 and p // rows <= -(-length // 32)
        tiles = -(-rows // (32 if rows > 16 else 16))
        assert p == 0 or p // rows * tiles * kv * layers <= 256


def test_pieces_of_many_contexts_and_lists():
    rng = np.random.default_rng(4)
    for _ in range(200):
        group, B, n_blocks = int(rng.choice([1, 2, 4, 7, 8])), int(rng.integers(1, 17)), int(rng.choice([0, 1, 40, 1024]))
        n = [int(x) for x in rng.integers(0, 17, B)]
        lens = [int(max(a, x)) for a, x in zip(n, np.exp(rng.uniform(0, np.log(65536), B)))]
        steps = [0 if not a else n_blocks or -(-x // 32) for a, x in zip(n, lens)]
        assert pieces(n, lens, group * 4, 4, 128, 1, n_blocks) <= sum(a * group * s for a, s in zip(n, steps))


def test_one_long_context_is_cut_beside_short_ones():
    """Sixteen tokens, one of them at 60 000 slots: its pieces are no longer than twice what a CU has to do on average."""
    n, lens = [1] * 16, [60000] + [100] * 15
    p = pieces(n, lens, 32, 8, 128)
    steps = sum(-(-x // 32) for x in lens) * 8
    assert p / 4 - 15 >= (60000 / 32) / (2 * -(-steps // 256) + 8)
