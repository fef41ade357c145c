"""Slots brought into caches of 4 bits and read back (easyspec_kvq_store, easyspec_kvq_load): every byte against the definition."""
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


def source(seed, dtype, *shape):
    import torch
    x = torch.from_numpy(np.random.default_rng(seed).normal(0, 1, shape) * np.exp(np.random.default_rng(seed + 1).normal(0, 3, shape[:-1] + (1,)))).cuda()
    return x.to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def store(es, cache, k, v, src_from, n, to, lens):
    es.easyspec_kvq_store(k, v, cache.layout, k.shape[3], src_from, n, to, lens, cache.c, K.stream())


def expect(cache, before, k, v, src_from, n, to, lens):
    """The bytes of the cache's arrays after a store, from those before it."""
    L, B, H, S, hd = cache.shape
    kc, ks, vc, vs, bounds = [x.copy() for x in before]
    k, v = k.double().cpu().numpy(), v.double().cpu().numpy()
    for b in range(B):
        if n[b] == 0:
            continue
        src, dst = slice(src_from[b], src_from[b] + n[b]), slice(to[b], to[b] + n[b])
        kc[:, b, :, dst], ks[:, b, :, dst] = ref.encode(k[:, b, :, src])
        vc[:, b, :, dst], vs[:, b, :, dst] = ref.encode(v[:, b, :, src])
        keys = ref.decode(kc[:, b], ks[:, b])
        for j in range(to[b] // 64, (to[b] + n[b] - 1) // 64 + 1):
            for layer in range(L):
                for h in range(H):
                    bounds[layer, b, h, j] = ref.bounds_of(keys[layer, h, 64 * j:min(64 * j + 64, lens[b])])
    return kc, ks, vc, vs, bounds


def check(cache, want):
    for name, a, b in zip(("k_codes", "k_scales", "v_codes", "v_scales", "k_bounds"), cache.bytes(), want):
        assert np.array_equal(a, b, equal_nan=a.dtype.kind == "f"), (name, np.argwhere(a != b)[:5].tolist())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("L,B,H,S,hd,src,src_from,n,to,lens", [
    (1, 1, 1, 1, 64, 1, [0], [1], [0], [1]),
    (1, 1, 1, 1, 128, 3, [2], [1], [0], [1]),
    (2, 3, 2, 130, 64, 70, [0, 5, 69], [70, 0, 1], [0, 0, 129], [70, 0, 130]),        # a whole block and part of one; nothing; the last slot
    (1, 2, 3, 200, 128, 64, [0, 1], [64, 63], [64, 65], [128, 200]),                     # a block; one that others lie behind
    (3, 1, 1, 65, 64, 65, [0], [65], [0], [65]),
    (1, 16, 2, 77, 128, 1, [0] * 16, [1] * 16, [4 * i + 3 for i in range(16)], [4 * i + 4 for i in range(16)]),
    (2, 1, 5, 300, 128, 300, [0], [300], [0], [300]),
])
def test_store(es, dtype, L, B, H, S, hd, src, src_from, n, to, lens):
    import torch
    cache = K.Cache(es, L, B, H, S, hd, dtype)
    g = np.random.default_rng(S)
    cache.ks.copy_(K.dev(g.integers(120, 131, tuple(cache.ks.shape)).astype(np.uint8)))       # what is there already
    cache.kc.copy_(K.dev(g.integers(0, 256, tuple(cache.kc.shape)).astype(np.uint8)))
    k, v = source(S, dtype, L, B, H, src, hd), source(S + 7, dtype, L, B, H, src, hd)
    before = cache.bytes()
    store(es, cache, k, v, src_from, n, to, lens)
    torch.cuda.synchronize()
    check(cache, expect(cache, before, k, v, src_from, n, to, lens))
    # the way back, into the other half of larger arrays
    out = [torch.full((L, B, H, src + 2, hd), -3.0, device="cuda", dtype=k.dtype) for _ in range(2)]
    es.easyspec_kvq_load(cache.c, cache.layout, to, n, src + 2, [2] * B, *out, K.stream())
    torch.cuda.synchronize()
    for x, values in zip(out, cache.values()):
        want = np.full(tuple(x.shape), -3.0)
        for b in range(B):
            want[:, b, :, 2:2 + n[b]] = values[:, b, :, to[b]:to[b] + n[b]]
        assert np.array_equal(x.double().cpu().numpy(), want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_every_magnitude_half_way_values_and_what_is_not_finite(es, dtype):
    import torch
    g = np.random.default_rng(0)
    x = np.zeros((1, 1, 1, 600, 64))
    half = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.9, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 0.0])
    for i in range(600):
        row = g.choice(half, 64) * g.choice([1, -1], 64)
        row[g.integers(0, 32)] = 4.0
        x[0, 0, 0, i] = row * 2.0 ** (i % 250 - 124)
    finfo = np.finfo(np.float32)
    x[0, 0, 0, 0, :3] = np.inf, 1, 2
    x[0, 0, 0, 1, 40] = np.nan
    x[0, 0, 0, 2, 3] = -np.inf
    x[0, 0, 0, 3] = 0.0
    x[0, 0, 0, 4] = -0.0
    x[0, 0, 0, 5] = 2.0 ** -149 * np.arange(64)                       # below the normal numbers
    x[0, 0, 0, 6, :2] = 2.0 ** -122, -(2.0 ** -123)
    x[0, 0, 0, 7, :2] = 2.0 ** -118, 2.0 ** -123
    x[0, 0, 0, 8, :2] = float(finfo.max), -float(finfo.max) / 3
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    k = torch.from_numpy(x).cuda().to(torch.float32).to(dt)
    v = k.flip(3).contiguous()
    cache = K.Cache(es, 1, 1, 1, 600, 64, dtype)
    before = cache.bytes()
    store(es, cache, k, v, [0], [600], [0], [600])
    torch.cuda.synchronize()
    check(cache, expect(cache, before, k, v, [0], [600], [0], [600]))
    kb, vb = torch.zeros_like(k), torch.zeros_like(k)
    es.easyspec_kvq_load(cache.c, cache.layout, [0], [600], 600, [0], kb, vb, K.stream())
    torch.cuda.synchronize()
    for got, want in zip((kb, vb), cache.values()):
        assert np.array_equal(got.double().cpu().numpy(), want, equal_nan=True)
    again = K.Cache(es, 1, 1, 1, 600, 64, dtype)                       # numbers of 4 bits stay what they are
    fine = torch.where(kb.isnan(), torch.zeros_like(kb), kb)
    store(es, again, fine, fine, [0], [600], [0], [600])
    back = torch.zeros_like(k), torch.zeros_like(k)
    es.easyspec_kvq_load(again.c, again.layout, [0], [600], 600, [0], *back, K.stream())
    torch.cuda.synchronize()
    assert torch.equal(back[0], fine) and torch.equal(back[1], fine)


def test_appended_one_by_one_as_at_once(es):
    """Bounds too: whatever the calls, they are those of the slots."""
    import torch
    L, B, H, S, hd = 2, 2, 2, 140, 64
    k, v = source(3, "fp32", L, B, H, S, hd), source(4, "fp32", L, B, H, S, hd)
    whole, single = K.Cache(es, L, B, H, S, hd, "fp32"), K.Cache(es, L, B, H, S, hd, "fp32")
    store(es, whole, k, v, [0, 0], [S, 100], [0, 0], [S, 100])
    step = 0
    while step < S:
        n = min(1 + step % 5, S - step)
        m = max(0, min(n, 100 - step))
        store(es, single, k, v, [step, step if m else 0], [n, m], [step, step if m else 0], [step + n, step + m])
        step += n
    torch.cuda.synchronize()
    for a, b in zip(whole.bytes(), single.bytes()):
        assert np.array_equal(a, b)


def test_rejected_slots_leave_the_bounds_with_the_next_store(es):
    import torch
    k, v = source(5, "fp32", 1, 1, 1, 80, 64), source(6, "fp32", 1, 1, 1, 80, 64)
    k[:, :, :, 70:] *= 1000
    cache, fresh = K.Cache(es, 1, 1, 1, 80, 64, "fp32"), K.Cache(es, 1, 1, 1, 80, 64, "fp32")
    store(es, cache, k, v, [0], [80], [0], [80])
    k[:, :, :, 70:] /= 3000
    store(es, cache, k, v, [70], [1], [70], [71])                        # the sequence was cut back to 70
    store(es, fresh, k, v, [0], [71], [0], [71])
    torch.cuda.synchronize()
    assert torch.equal(cache.bounds, fresh.bounds)


def test_without_bounds_on_another_stream_and_replayed(es):
    import torch
    k, v = source(8, "bf16", 1, 2, 2, 100, 128), source(9, "bf16", 1, 2, 2, 100, 128)
    want = K.Cache(es, 1, 2, 2, 100, 128)
    store(es, want, k, v, [0, 0], [100, 30], [0, 0], [100, 30])
    cache = K.Cache(es, 1, 2, 2, 100, 128, bounds=False)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    es.easyspec_kvq_store(k, v, cache.layout, 100, [0, 0], [100, 30], [0, 0], [100, 30], cache.c, other.cuda_stream)
    other.synchronize()
    for a, b in zip(cache.bytes(), want.bytes()[:4]):
        assert np.array_equal(a, b)
    out = torch.zeros_like(k), torch.zeros_like(v)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        store(es, want, k, v, [0, 0], [100, 30], [0, 0], [100, 30])
        es.easyspec_kvq_load(want.c, want.layout, [0, 0], [100, 30], 100, [0, 0], *out, K.stream())
    for turn in range(3):
        k.normal_()
        v.normal_()
        graph.replay()
        torch.cuda.synchronize()
        fresh = K.Cache(es, 1, 2, 2, 100, 128)
        store(es, fresh, k, v, [0, 0], [100, 30], [0, 0], [100, 30])
        torch.cuda.synchronize()
        for a, b in zip(want.bytes(), fresh.bytes()):
            assert np.array_equal(a, b)
        assert np.array_equal(out[0].double().cpu().numpy()[:, 0], want.values()[0][:, 0])


def test_offsets_beyond_32_bits(es):
    """Values of 4.3 GB: the last rows of a cache of 65536 slots."""
    import torch
    L, H, S, hd = 1, 512, 65536, 64
    src = torch.zeros(L, 1, H, S, hd, dtype=torch.bfloat16, device="cuda")
    src[:, :, -1, -3:] = torch.arange(3 * hd, device="cuda", dtype=torch.bfloat16).reshape(3, hd)
    cache = K.Cache(es, L, 1, H, S, hd)
    es.easyspec_kvq_store(src, src, cache.layout, S, [S - 5], [5], [S - 5], [S], cache.c, K.stream())
    out = torch.zeros_like(src)
    es.easyspec_kvq_load(cache.c, cache.layout, [S - 5], [5], S, [S - 5], out, src, K.stream())
    torch.cuda.synchronize()
    want = ref.decode(*ref.encode(np.arange(3.0 * hd).reshape(3, hd)))
    assert np.array_equal(out[0, 0, -1, -3:].double().cpu().numpy(), want) and np.array_equal(src[0, 0, -1, -3:].double().cpu().numpy(), want)
    assert not out[0, 0, :-1].any() and not out[0, 0, -1, :-3].any()
