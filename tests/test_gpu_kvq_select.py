"""Selection of blocks (easyspec_kvq_select): equal lists."""
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


def with_bounds(es, seed, L, B, H, S, hd):
    cache = K.Cache(es, L, B, H, S, hd)
    g = np.random.default_rng(seed)
    N = -(-S // 64)
    middle = g.normal(0, 1, (L, B, H, N, hd))
    reach = np.abs(g.normal(0, 1, (L, B, H, N, hd)))
    import torch
    cache.bounds.copy_(torch.from_numpy(np.stack((middle - reach, middle + reach), 4)).to(torch.bfloat16))
    return cache


def check(cache, q, n, lens, first, last, n_select):
    import torch
    got = K.select(cache, q, n, lens, first, last, n_select)
    torch.cuda.synchronize()
    want = ref.select(q.double().cpu().numpy(), cache.bounds.double().cpu().numpy(), n, lens, first, last, n_select)
    assert np.array_equal(got.cpu().numpy(), want), np.argwhere(got.cpu().numpy() != want)[:5].tolist()
    return want


@pytest.mark.parametrize("L,heads,hd,n,lens,slots,first,last,n_select", [
    (1, (1, 1), 64, [1], [1], 1, 0, 1, 1),
    (1, (1, 1), 64, [1], [64], 64, 0, 0, 3),
    (1, (1, 1), 128, [1], [65], 70, 0, 0, 1),
    (1, (32, 8), 128, [1], [5000], 5001, 1, 2, 16),
    (2, (14, 2), 64, [3, 0, 16], [70, 5, 1000], 1000, 0, 1, 5),
    (1, (8, 1), 128, [16], [70], 70, 0, 1, 1),                      # tokens on both sides of a block's end
    (1, (4, 4), 64, [1] * 16, [60 * i + 1 for i in range(16)], 1000, 1, 1, 6),
    (3, (7, 1), 128, [2, 1], [4096, 4097], 4100, 2, 3, 40),
    (1, (2, 2), 64, [1], [65536], 65536, 1, 1, 100),
    (1, (2, 2), 64, [2], [65536], 65536, 0, 0, 1024),
    (1, (2, 1), 64, [1], [2000], 2000, 5, 7, 4),                    # fewer than the first and the last
    (1, (2, 1), 64, [1], [2000], 2000, 0, 0, 1),
    (1, (2, 1), 64, [1], [300], 300, 2 ** 31 - 1, 2 ** 31 - 1, 3),
    (1, (2, 1), 64, [1], [300], 300, 0, 2 ** 31 - 1, 3),
])
def test_lists(es, L, heads, hd, n, lens, slots, first, last, n_select):
    cache = with_bounds(es, slots, L, len(lens), heads[1], slots, hd)
    q = K.dev(K.queries(slots, L, sum(n), heads[0], hd))
    check(cache, q, n, lens, first, last, n_select)


def test_ties_and_scores_that_are_not_numbers(es):
    import torch
    cache = with_bounds(es, 1, 1, 1, 1, 1280, 64)
    q = K.dev(K.queries(1, 1, 1, 2, 64))
    cache.bounds[:, :, :, 3:17] = cache.bounds[:, :, :, 3:4].clone()    # fourteen alike
    for n_select in (1, 2, 5, 10, 17, 20):
        check(cache, q, [1], [1280], 0, 0, n_select)
    zero = q * 0
    for n_select in (1, 7, 20):
        want = check(cache, zero, [1], [1280], 0, 1, n_select)           # all scores are 0: the lowest, and the last
        assert want[0, 0, 0].tolist()[:-1] == list(range(n_select - 1)) and want[0, 0, 0, -1] == 19
    cache.bounds[0, 0, 0, 5, :, 7] = float("nan")
    cache.bounds[0, 0, 0, 9, 0] = float("inf")
    cache.bounds[0, 0, 0, 9, 1] = -float("inf")                         # a block of nothing but NaN
    cache.bounds[0, 0, 0, 11, 1, 3] = float("inf")
    cache.bounds[0, 0, 0, 12, 0, 3] = -float("inf")
    for n_select in (1, 4, 17, 18, 19, 20, 21):
        check(cache, q, [1], [1280], 0, 0, n_select)
    q[0, 0, 0, 3] = float("nan")                                         # one query head passed over
    for n_select in (1, 4, 19, 20):
        check(cache, q, [1], [1280], 1, 1, n_select)
    q[0, 0, 1, 0] = float("inf")
    for n_select in (3, 20):
        check(cache, q, [1], [1280], 0, 0, n_select)
    torch.cuda.synchronize()


def test_bounds_are_bounds(es):
    """Of a stored cache no product of a query and a key exceeds its block's score."""
    import torch
    g = np.random.default_rng(9)
    k = torch.from_numpy(g.normal(0, 2, (1, 1, 2, 500, 64))).cuda().to(torch.bfloat16)
    cache = K.Cache(es, 1, 1, 2, 500, 64)
    es.easyspec_kvq_store(k, k, cache.layout, 500, [0], [500], [0], [500], cache.c, K.stream())
    q = K.queries(9, 1, 1, 4, 64)
    torch.cuda.synchronize()
    keys, b = cache.values()[0], cache.bounds.double().cpu().numpy()
    for j in range(4):
        x = q[0, 0, j].astype(np.float64)
        scores = np.where(x > 0, b[0, 0, j // 2, :, 1], b[0, 0, j // 2, :, 0]) @ x
        products = keys[0, 0, j // 2] @ x
        assert all(products[64 * i:64 * i + 64].max() <= scores[i] + 1e-9 for i in range(8))
    check(cache, K.dev(q), [1], [500], 1, 1, 4)


def test_inside_its_arrays_in_a_graph(es):
    import torch
    n, lens = [2, 1], [3000, 100]
    cache = with_bounds(es, 2, 2, 2, 2, 3000, 128)
    q = K.dev(K.queries(2, 2, 3, 8, 128))
    need = es.easyspec_kvq_select_workspace_bytes(cache.layout, n, lens, 8, 7)
    ws = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    out = torch.full((2 * 3 * 2 * 7 + 100,), -9, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        K.select(cache, q, n, lens, 1, 1, 7, out, ws)
    for turn in range(3):
        q.normal_(0, 1.5)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(out[:84].reshape(2, 3, 2, 7).cpu().numpy(), ref.select(q.double().cpu().numpy(), cache.bounds.double().cpu().numpy(), n, lens, 1, 1, 7))
    assert bool((ws[need:] == 0xA5).all()) and bool((out[84:] == -9).all())
