"""What easyspec_kvq_attention_workspace_bytes and _limit promise: a workspace sized once holds every shorter call.  All of it is host arithmetic."""
import math

import numpy as np
import pytest

import paper_2502_02493_amd as es

GROUPS = [1, 2, 4, 7, 8]


def layout(n_seqs, kv_heads=8, layers=1, hd=128, slots=65536):
    return es.easyspec_kv_layout(layers, n_seqs, kv_heads, slots, hd, es.EASYSPEC_DTYPE_BF16)


def need(lay, n, lens, group, n_blocks=0):
    got = es.easyspec_kvq_attention_workspace_bytes(lay, n, lens, group * lay.n_kv_heads, n_blocks)
    assert got >= 0
    return got


def used(lay, n, lens, group, n_blocks=0):
    """Bytes that a call writes, from how contexts are cut: steps of 32 slots (lists: blocks, two steps each) in chunks for no more workgroups
    than 256 CUs, a chunk no longer than twice what a CU has to do on average; contexts of up to sixteen steps whole."""
    e = [(a, s) for a, s in zip(n, lens) if a]
    if not e:
        return 0
    hl = lay.n_kv_heads * lay.n_layers
    pieces = [n_blocks or -(-s // 32) for _, s in e]
    longest = max(2 * n_blocks if n_blocks else x for x in pieces)
    if longest <= 16:
        return 0
    rows = group if n_blocks else max(a * group for a, _ in e)
    tiles = 2 if rows > 16 else 1
    steps = sum(2 * a * n_blocks if n_blocks else x for (a, _), x in zip(e, pieces))
    waves = 8 if tiles == 2 or steps * hl > 4096 else 4
    least = waves // 2 if n_blocks else waves
    wgs = [a if n_blocks else -(-a * group // (16 * tiles)) for a, _ in e]

    def count(chunk):
        return sum(-(-p // chunk) * w for p, w in zip(pieces, wgs)) * hl
    most = min(64 if n_blocks else 2048, max(least, -(-(2 * count(1) // 256) // least) * least))
    chunk = next((c for c in range(least, most, least) if count(c) <= 256), most)
    cut = [-(-p // chunk) for p in pieces]
    return 0 if max(cut) == 1 else sum(a * group * c for (a, _), c in zip(e, cut)) * hl * (lay.head_dim * 4 + 8)


def random_call(rng, lists):
    B = int(rng.choice([1, 1, 2, 5, 16]))
    lay = layout(B, int(rng.choice([1, 2, 4, 8, 9, 32, 300])), int(rng.choice([1, 1, 3, 32])), int(rng.choice([64, 128])))
    n = [int(x) for x in rng.integers(0, 17, B)]
    lens = [int(max(a, 1, x)) for a, x in zip(n, np.exp(rng.uniform(0, math.log(65536), B)))]
    blocks = int(np.exp(rng.uniform(0, math.log(1024.99)))) if lists else 0
    return lay, n, lens, int(rng.choice(GROUPS)), blocks


@pytest.mark.parametrize("lists", [False, True])
def test_holds_what_the_call_writes(lists):
    rng = np.random.default_rng(1)
    for _ in range(1500):
        lay, n, lens, group, blocks = random_call(rng, lists)
        assert need(lay, n, lens, group, blocks) >= used(lay, n, lens, group, blocks), (lay.n_kv_heads, lay.n_layers, n, lens, group, blocks)


def test_never_falls_as_contexts_grow():
    one = layout(1)
    last = 0
    for s in range(1, 65537, 7):
        now = need(one, [1], [s], 4)
        assert now >= last, s
        last = now
    assert need(one, [1], [4097], 4) >= used(one, [1], [4096], 4) == 532480
    rng = np.random.default_rng(2)
    for _ in range(1500):
        lay, n, lens, group, _ = random_call(rng, False)
        shorter = [int(rng.integers(max(a, 1), s + 1)) if rng.random() < 0.7 else s for a, s in zip(n, lens)]
        assert need(lay, n, shorter, group) <= need(lay, n, lens, group), (n, shorter, lens)


def test_never_falls_as_lists_grow():
    rng = np.random.default_rng(3)
    for _ in range(100):
        lay, n, lens, group, _ = random_call(rng, True)
        sizes = sorted(set(range(1, 70)) | set(range(70, 1025, 37)) | {1024})
        got = [need(lay, n, lens, group, b) for b in sizes]
        assert got == sorted(got)


@pytest.mark.parametrize("lists", [False, True])
def test_the_limit_holds_every_call_of_a_layout(lists):
    rng = np.random.default_rng(4)
    for _ in range(1500):
        lay, n, lens, group, blocks = random_call(rng, lists)
        lay.max_slots = max(lens + [1]) if rng.random() < 0.3 else 65536
        most = es.easyspec_kvq_attention_workspace_limit(lay, max(max(n), 1), group * lay.n_kv_heads, blocks)
        assert most >= need(lay, n, lens, group, blocks) and most >= need(lay, n, lens, group)
        fewer = [int(rng.integers(0, a + 1)) for a in n]
        assert most >= need(lay, fewer, lens, group, blocks) and most >= need(lay, fewer, lens, group)
        if blocks:
            assert most >= need(lay, fewer, lens, group, int(rng.integers(1, blocks + 1)))


def test_the_limit_is_no_waste():
    """A batch of drafting on 8 KV heads, one layer at a time: megabytes."""
    assert es.easyspec_kvq_attention_workspace_limit(layout(4), 6, 32, 0) < 8 << 20
    assert es.easyspec_kvq_attention_workspace_limit(layout(16), 1, 32, 32) < 2 << 20
    assert es.easyspec_kvq_attention_workspace_limit(layout(16, slots=512), 16, 32, 8) == 0


def test_the_limit_refuses():
    lay = layout(2)
    for bad in ((0, 32, 0), (17, 32, 0), (-1, 32, 0), (1, 0, 0), (1, 24, 0), (1, 33, 0), (1, 32, -1), (1, 32, 1025)):
        assert es.easyspec_kvq_attention_workspace_limit(lay, *bad) == -1
    assert es.easyspec_kvq_attention_workspace_limit(layout(0), 1, 32, 0) == -1
