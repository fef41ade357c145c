"""Attention over caches held in 4 bits (easyspec_kvq_attention) against a 64-bit evaluation, within the bound that kvq_ref derives."""
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


def cache_with_rest(es, seed, L, B, H, S, hd, lens):
    """What lies behind a sequence's slots is NaN."""
    cache = K.random_cache(es, seed, L, B, H, S, hd)
    for b, n in enumerate(lens):
        for x in (cache.ks, cache.vs):
            x[:, b, :, n:] = 255
    return cache


SIZES = [
    (1, (1, 1), 64, [1], [1], 1),                     # one token that sees itself
    (1, (1, 1), 128, [1], [1], 5),
    (1, (4, 2), 64, [1], [128], 130),
    (2, (7, 1), 64, [5], [61], 64),
    (1, (32, 8), 128, [1], [777], 800),
    (1, (8, 2), 128, [6], [63], 64),
    (2, (28, 4), 128, [16], [65], 65),                # 112 rows a KV head
    (1, (8, 1), 128, [16], [16], 16),                 # nothing but the new tokens, 128 rows
    (1, (8, 1), 64, [16], [1500], 1501),
    (3, (4, 4), 64, [3, 0, 16, 1], [3, 50, 700, 129], 700),   # ragged; one sequence left alone
    (1, (16, 2), 128, [2, 9], [1025, 2049], 2100),
    (1, (2, 1), 64, [1] * 16, list(range(1, 17)), 20),
    (2, (8, 2), 128, [6, 2, 1], [1111, 300, 1], 1200),
    (1, (2, 2), 64, [4], [33], 33),
    (1, (2, 1), 128, [2], [4097], 4097),              # four rows
    (1, (7, 1), 128, [1], [2500], 2500),
    (1, (8, 1), 64, [2], [96], 96),                   # sixteen rows
    (1, (8, 1), 64, [3], [97], 97),                   # ... and one tile more
]


@pytest.mark.parametrize("L,heads,hd,n,lens,slots", SIZES)
def test_sizes(es, L, heads, hd, n, lens, slots):
    Hq, H = heads
    cache = cache_with_rest(es, sum(lens), L, len(lens), H, slots, hd, lens)
    q = K.dev(K.queries(sum(lens), L, sum(n), Hq, hd))
    K.check_attention(cache, q, n, lens, K.attend(cache, q, n, lens))


@pytest.mark.parametrize("L,heads,hd,n,lens,slots", [
    (24, (4, 2), 64, [1], [3000], 3000),              # chunks of several steps
    (64, (8, 1), 64, [3], [700], 700),
    (1, (1, 1), 64, [1], [65536], 65536),
    (1, (16, 16), 64, [1, 1], [9000, 40], 9000),
])
def test_cuts(es, L, heads, hd, n, lens, slots):
    Hq, H = heads
    cache = cache_with_rest(es, sum(lens) + L, L, len(lens), H, slots, hd, lens)
    q = K.dev(K.queries(L, L, sum(n), Hq, hd))
    K.check_attention(cache, q, n, lens, K.attend(cache, q, n, lens))


LISTS = [
    ([[0, 1, 2, 3]], "all"), ([[3]], "the own"), ([[0, -1, -1]], "one that is far"), ([[1, 1, 3, 3]], "repeated"), ([[2, 0, 3]], "one that goes back"),
    ([[-1, -1]], "none"), ([[4, 5, 2 ** 30]], "none that is there"), ([[-5, 2, 9]], "others are no blocks"), ([[3, -1, 3]], "twice behind a gap"),
    ([[-2 ** 31, 0, 3]], "the lowest number"),
]


@pytest.mark.parametrize("lists,what", LISTS)
@pytest.mark.parametrize("heads,hd", [((4, 1), 128), ((7, 1), 64), ((1, 1), 64), ((8, 1), 128)])
def test_lists(es, lists, what, heads, hd):
    cache = cache_with_rest(es, 3, 1, 1, 1, 256, hd, [250])
    q = K.dev(K.queries(3, 1, 1, heads[0], hd))
    blocks = K.dev(np.array(lists, np.int32).reshape(1, 1, 1, -1))
    out = K.attend(cache, q, [1], [250], blocks)
    if what == "twice behind a gap":                  # it counts twice: every weight of its slots doubles, which leaves their shares as they are
        blocks = K.dev(np.array([[3]], np.int32).reshape(1, 1, 1, -1))
    K.check_attention(cache, q, [1], [250], out, blocks)
    if what.startswith("none"):
        assert not out.any()


@pytest.mark.parametrize("L,heads,hd,n,lens,slots,n_blocks", [
    (1, (8, 2), 128, [1], [4000], 4000, 20),
    (2, (14, 2), 64, [3, 0, 16], [70, 5, 1000], 1000, 9),        # tokens that do not see the blocks of later ones
    (1, (4, 4), 64, [1] * 16, [60 * i + 1 for i in range(16)], 1000, 16),
    (1, (2, 1), 128, [2], [30000], 30000, 300),
    (1, (8, 1), 64, [1], [65536], 65536, 1024),
    (1, (4, 2), 64, [5], [66], 66, 1),
])
def test_lists_of_many(es, L, heads, hd, n, lens, slots, n_blocks):
    Hq, H = heads
    g = np.random.default_rng(slots)
    cache = cache_with_rest(es, slots, L, len(lens), H, slots, hd, lens)
    q = K.dev(K.queries(slots, L, sum(n), Hq, hd))
    blocks = np.full((L, sum(n), H, n_blocks), -1, np.int32)
    for at in np.ndindex(L, sum(n), H):
        m = -(-slots // 64)
        chosen = np.sort(g.choice(m, min(m, g.integers(1, n_blocks + 1)), replace=False))
        blocks[at][:len(chosen)] = chosen
    blocks = K.dev(blocks)
    K.check_attention(cache, q, n, lens, K.attend(cache, q, n, lens, blocks), blocks)


def test_a_list_of_all_blocks_is_the_whole_cache(es):
    n, lens = [2, 5], [333, 640]
    cache = cache_with_rest(es, 11, 1, 2, 2, 640, 128, lens)
    q = K.dev(K.queries(11, 1, 7, 8, 128))
    blocks = K.dev(np.broadcast_to(np.arange(10, dtype=np.int32), (1, 7, 2, 10)))
    K.check_attention(cache, q, n, lens, K.attend(cache, q, n, lens, blocks))


@pytest.mark.parametrize("heads,hd", [((4, 1), 128), ((8, 1), 64), ((2, 1), 64)])
def test_what_a_token_does_not_see_has_no_effect(es, heads, hd):
    """NaN in slots that the last tokens alone see: theirs are the only results that show it."""
    import torch
    n, lens = [4], [90]
    cache = cache_with_rest(es, 12, 1, 1, 1, 100, hd, lens)
    q = K.dev(K.queries(12, 1, 4, heads[0], hd))
    before = K.attend(cache, q, n, lens)
    cache.vs[0, 0, 0, 88, 1] = 255                    # V of token 2, channels 32 .. 63
    after = K.attend(cache, q, n, lens)
    assert torch.equal(after[:, :2], before[:, :2]) and bool(after[:, 2:, :, 32:64].isnan().all())
    assert torch.equal(after[:, 2:, :, :32], before[:, 2:, :, :32]) and torch.equal(after[:, 2:, :, 64:], before[:, 2:, :, 64:])
    cache.vs[0, 0, 0, 88, 1] = 127
    cache.ks[0, 0, 0, 89, 0] = 255                    # K of token 3
    after = K.attend(cache, q, n, lens)
    assert torch.equal(after[:, :2], before[:, :2]) and bool(after[:, 3].isnan().all()) and bool(after[:, 2].isfinite().all())
    one = K.attend(cache, q[:, :1].contiguous(), [1], [87])
    K.check_attention(cache, q[:, :1], [1], [87], one)
    cache.ks[0, 0, 0, 40, 0] = 255                    # one that all see
    assert bool(K.attend(cache, q, n, lens).isnan().all())


def test_far_scores(es):
    """Scores of thousands: one slot has all the weight; and equal ones: all have the same."""
    n, lens = [3], [200]
    cache = K.random_cache(es, 13, 1, 1, 1, 200, 64, std=100.0)
    q = K.dev(K.queries(13, 1, 3, 4, 64, std=30.0))
    K.check_attention(cache, q, n, lens, K.attend(cache, q, n, lens))
    zero = q * 0
    K.check_attention(cache, zero, n, lens, K.attend(cache, zero, n, lens))


@pytest.mark.parametrize("heads,hd", [((4, 1), 128), ((8, 1), 64), ((7, 1), 128), ((2, 1), 64)])
def test_queries_of_every_size(es, heads, hd):
    """Channels six decades apart in one query; queries far from 1 on keys as far on the other side; zeros but for one channel."""
    g = np.random.default_rng(hd + heads[0])
    n, lens = [5], [77]
    for shift in (-90, -20, 0, 20, 90):
        k = g.normal(0, 1, (1, 1, 1, 77, hd)) * 2.0 ** -shift
        cache = K.Cache(es, 1, 1, 1, 77, hd).put(k, g.normal(0, 1, (1, 1, 1, 77, hd)))
        q = g.normal(0, 2, (1, 5, heads[0], hd)) * 2.0 ** shift
        q[:, 1] *= np.exp2(g.integers(-10, 11, hd))
        q[:, 2] *= np.exp2(-g.integers(0, 60, hd))
        q[:, 3, :, 1:] = 0
        q[:, 4, :, :32] = 0
        q = K.dev(q.astype(np.float32))
        K.check_attention(cache, q, n, lens, K.attend(cache, q, n, lens))


@pytest.mark.parametrize("heads,hd", [((4, 1), 128), ((8, 1), 64), ((7, 1), 128)])
def test_queries_that_are_not_finite(es, heads, hd):
    """A query with an infinity or NaN has no result; the others of its token and sequence are what they were."""
    import torch
    n, lens = [3], [130]
    cache = K.random_cache(es, 21, 1, 1, 1, 130, hd)
    q = K.dev(K.queries(21, 1, 3, heads[0], hd))
    before = K.attend(cache, q, n, lens)
    for value in (float("inf"), float("-inf"), float("nan")):
        bad = q.clone()
        bad[0, 1, 1, hd - 3] = value
        after = K.attend(cache, bad, n, lens)
        assert bool(after[0, 1, 1].isnan().all())
        after[0, 1, 1] = before[0, 1, 1]
        assert torch.equal(after, before)


def test_stays_inside_its_arrays(es):
    import torch
    for heads, hd, n, lens, nb in (((8, 2), 128, [6, 16], [900, 2000], 0), ((4, 2), 64, [1, 1], [3000, 70], 0), ((28, 4), 128, [16, 2], [100, 90], 0), ((8, 2), 64, [3, 1], [700, 90], 11)):
        cache = cache_with_rest(es, 3, 1, 2, heads[1], max(lens), hd, lens)
        q = K.dev(K.queries(4, 1, sum(n), heads[0], hd))
        blocks = K.dev(np.broadcast_to(np.arange(nb, dtype=np.int32), (1, sum(n), heads[1], nb))) if nb else None
        need = es.easyspec_kvq_attention_workspace_bytes(cache.layout, n, lens, heads[0], nb)
        ws = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
        out = torch.full((q.numel() + 512,), -3.0, device="cuda")
        K.attend(cache, q, n, lens, blocks, ws, out)
        torch.cuda.synchronize()
        assert bool((ws[need:] == 0xA5).all()) and bool((out[q.numel():] == -3).all())
        K.check_attention(cache, q, n, lens, out[:q.numel()].reshape(q.shape), blocks)


def test_same_bits_on_streams_and_in_graphs(es):
    """Two captured calls with workspaces of their own, replayed in turn with eager calls between."""
    import torch
    n, lens = [3, 1], [1500, 70]
    cache = cache_with_rest(es, 21, 1, 2, 2, 1500, 128, lens)
    q = K.dev(K.queries(21, 1, 4, 8, 128))
    blocks = K.dev(np.broadcast_to(np.array([0, 1, 20, 23], np.int32), (1, 4, 2, 4)))
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    a = K.attend(cache, q, n, lens)
    b = K.attend(cache, q, n, lens, on=other)
    other.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(a, b)
    outs, graphs, spaces = [], [], []
    for lists in (None, blocks):
        need = es.easyspec_kvq_attention_workspace_bytes(cache.layout, n, lens, 8, 0 if lists is None else 4)
        spaces.append(torch.empty(need // 4 + 4, device="cuda"))
        outs.append(torch.empty_like(q))
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            K.attend(cache, q, n, lens, lists, spaces[-1], outs[-1])
    for turn in range(4):
        q.normal_(0, 1.5)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for lists, out in zip((None, blocks), outs):
            assert torch.equal(out, K.attend(cache, q, n, lens, lists))


def test_a_layer_of_a_larger_cache_and_offsets_beyond_32_bits(es):
    """Layer by layer from the arrays of all layers, whose scales need not lie on 16 bytes; codes of 4.3 GB."""
    import torch
    cache = K.random_cache(es, 31, 3, 1, 1, 77, 64)
    q = K.dev(K.queries(31, 3, 2, 2, 64))
    whole = K.attend(cache, q, [2], [77])
    one = es.easyspec_kv_layout(1, 1, 1, 77, 64, es.EASYSPEC_DTYPE_BF16)
    for layer in range(3):
        c = es.make_kvq(cache.kc[layer], cache.ks[layer], cache.vc[layer], cache.vs[layer])
        out = torch.empty(1, 2, 2, 64, device="cuda")
        ws = torch.empty(es.easyspec_kvq_attention_workspace_bytes(one, [2], [77], 2, 0) // 4 + 4, device="cuda")
        es.easyspec_kvq_attention(q[layer], c, one, [2], [77], 2, None, 0, out, ws, K.stream())
        torch.cuda.synchronize()
        tail = K.Cache(es, 1, 1, 1, 77, 64)
        tail.kc, tail.ks, tail.vc, tail.vs = (x[layer:layer + 1] for x in (cache.kc, cache.ks, cache.vc, cache.vs))
        K.check_attention(tail, q[layer:layer + 1], [2], [77], out)
        K.check_attention(tail, q[layer:layer + 1], [2], [77], whole[layer:layer + 1])
    H, S = 2048, 65536                                   # 2^32 bytes of codes of K
    big = K.Cache(es, 1, 1, H, S, 64, bounds=False, fill=127)
    g = np.random.default_rng(5)
    k, v = g.normal(0, 1, (1, 1, 1, 100, 64)), g.normal(0, 1, (1, 1, 1, 100, 64))
    for codes, scales, x in ((big.kc, big.ks, k), (big.vc, big.vs, v)):
        c, s = ref.encode(x)
        codes[:, :, -1:, -100:], scales[:, :, -1:, -100:] = K.dev(c), K.dev(s)
    q = torch.zeros(1, 1, H, 64, device="cuda")
    q[0, 0, -1] = K.dev(K.queries(5, 1, 1, 1, 64))[0, 0, 0]
    blocks = torch.full((1, 1, H, 2), -1, dtype=torch.int32, device="cuda")
    blocks[0, 0, -1] = torch.tensor([S // 64 - 1, -1], dtype=torch.int32)
    out = K.attend(big, q, [1], [S], blocks)
    small = K.Cache(es, 1, 1, 1, 64, 64).put(k[:, :, :, -64:], v[:, :, :, -64:])
    K.check_attention(small, q[:, :, -1:], [1], [64], out[:, :, -1:])
    assert not out[:, :, :-1].any()


def test_scales_at_odd_addresses(es):
    """Scales need no alignment: arrays that start anywhere."""
    import torch
    cache = K.random_cache(es, 41, 1, 1, 2, 133, 128)
    q = K.dev(K.queries(41, 1, 3, 4, 128))
    want = K.attend(cache, q, [3], [133])
    for shift in (1, 2, 3, 5, 14):
        moved = []
        for s in (cache.ks, cache.vs):
            room = torch.full((s.numel() + 32,), 255, dtype=torch.uint8, device="cuda")
            room[shift:shift + s.numel()] = s.reshape(-1)
            moved.append(room)
        c = es.make_kvq(cache.kc, moved[0].data_ptr() + shift, cache.vc, moved[1].data_ptr() + shift)
        out = torch.empty_like(q)
        ws = torch.empty(es.easyspec_kvq_attention_workspace_bytes(cache.layout, [3], [133], 4, 0) // 4 + 4, device="cuda")
        es.easyspec_kvq_attention(q, c, cache.layout, [3], [133], 4, None, 0, out, ws, K.stream())
        torch.cuda.synchronize()
        assert torch.equal(out, want)
