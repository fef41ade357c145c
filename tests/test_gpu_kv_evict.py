"""Eviction by accumulated weight (easyspec_kv_evict): slots, rows and weights equal to a plain selection."""
import numpy as np
import pytest

import operator_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def es():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device; none is visible")
    import paper_2502_02493_amd as es
    return es


def make(seed, L, B, H, S, hd, dtype):
    import torch
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    k, v = (torch.empty(L, B, H, S, hd, dtype=dt, device="cuda").normal_(generator=g) for _ in range(2))
    w = torch.exp(2 * torch.empty(L, B, H, S, device="cuda").normal_(generator=g)) * 0.01
    w[torch.rand(w.shape, device="cuda", generator=g) < 0.1] = 0.0
    return k, v, w


def check(es, k, v, w, lens, keep, recent, out_slots=None, in_place=False, rows=None):
    import torch
    L, B, H, S, hd = k.shape
    So = S if out_slots is None else out_slots
    layout = es.easyspec_kv_layout(L, B, H, S, hd, es.EASYSPEC_DTYPE_BF16 if k.dtype == torch.bfloat16 else es.EASYSPEC_DTYPE_F32)
    slots = torch.full((L, B, H, So), -9, dtype=torch.int32, device="cuda")
    if in_place:
        ki, vi, wi = k.clone(), v.clone(), w.clone()
        ko, vo, wo = ki, vi, wi
        k0, v0, w0 = k, v, w
    else:
        ki, vi, wi = k, v, w
        ko, vo = (torch.full((L, B, H, So, hd), 7.0, dtype=k.dtype, device="cuda") for _ in range(2))
        wo = torch.full((L, B, H, So), -5.0, device="cuda")
        k0, v0, w0 = ko.clone(), vo.clone(), wo.clone()
    torch.cuda.synchronize()
    es.easyspec_kv_evict(ki, vi, wi, layout, lens, keep, recent, So, ko, vo, wo, slots, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    heavy = w.cpu().numpy()
    for l, b, h in rows or [(l, b, h) for l in range(L) for b in range(B) for h in range(H)]:
        kept = ref.kept_slots(heavy[l, b, h], lens[b], keep[b], recent)
        n = len(kept)
        assert np.array_equal(slots[l, b, h, :n].cpu().numpy(), kept), (l, b, h)
        assert torch.all(slots[l, b, h, n:] == -9)
        at = torch.from_numpy(kept.astype(np.int64)).cuda()
        for got, src, old in ((ko, k, k0), (vo, v, v0), (wo, w, w0)):
            assert torch.equal(got[l, b, h, :n].view(torch.uint8), src[l, b, h].index_select(0, at).view(torch.uint8)), (l, b, h)
            # in place, rows between the last one that stays and the sequence's old length are as they were too
            assert torch.equal(got[l, b, h, n:].view(torch.uint8), old[l, b, h, n:].view(torch.uint8)), (l, b, h)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("L,B,H,S,hd,dtype,lens,keep,recent", [
    (1, 1, 1, 1, 64, "fp32", [1], [1], 0),
    (1, 1, 1, 2, 64, "bf16", [2], [1], 0),
    (1, 1, 1, 2, 64, "bf16", [2], [1], 1),
    (2, 1, 2, 61, 64, "fp32", [61], [24], 8),
    (1, 3, 2, 100, 128, "bf16", [100, 40, 0], [50, 50, 10], 50),       # one keeps everything, one is empty
    (2, 2, 3, 70, 64, "bf16", [64, 70], [0, 69], 5),                   # one of which nothing stays: left alone
    (1, 1, 2, 1025, 128, "fp32", [1025], [1024], 0),
    (1, 1, 8, 4096, 128, "bf16", [4096], [1], 0),
    (2, 2, 2, 5000, 64, "bf16", [4097, 4999], [300, 4000], 128),
    (1, 16, 1, 300, 64, "bf16", list(range(1, 17)), [4] * 16, 2),
    (1, 1, 2, 20000, 64, "bf16", [19999], [7000], 1000),
    (1, 1, 1, 40000, 64, "bf16", [40000], [39999], 10),
    (1, 1, 1, 65536, 64, "bf16", [65536], [1234], 100),
])
def test_sizes(es, in_place, L, B, H, S, hd, dtype, lens, keep, recent):
    k, v, w = make(S + recent, L, B, H, S, hd, dtype)
    check(es, k, v, w, lens, keep, recent, None if in_place else max(1, max(min(a, b) for a, b in zip(lens, keep))) + recent % 3, in_place)


def test_equal_weights_go_to_the_lowest_slot(es):
    k, v, w = make(1, 1, 1, 8, 3000, 64, "bf16")
    w[0, 0, 0] = 0.0
    w[0, 0, 1] = 2.5
    w[0, 0, 2, ::3] = 0.25                        # some tied over the border
    w[0, 0, 3] = (w[0, 0, 3] * 20).round() / 20
    w[0, 0, 4, ::2] = -0.0
    w[0, 0, 4, 1::2] = 0.0                        # one weight, two signs
    w[0, 0, 5] = -w[0, 0, 5]
    w[0, 0, 6, 5:2000] = 1e-42                    # denormal
    for keep, recent in ((1, 0), (777, 0), (2999, 13), (2000, 1999)):
        check(es, k, v, w, [3000], [keep], recent)
        check(es, k, v, w, [3000], [keep], recent, in_place=True)


def test_non_finite_weights(es):
    k, v, w = make(2, 1, 1, 4, 500, 64, "fp32")
    w[0, 0, 0, 10:20] = float("nan")
    w[0, 0, 1] = float("nan")
    w[0, 0, 2, 7], w[0, 0, 2, 8] = float("inf"), -float("inf")
    for keep in (1, 40, 485, 495, 499):
        check(es, k, v, w, [500], [keep], 3)


def test_weights_of_whole_model_and_graph(es):
    import torch
    L, B, H, S, hd = 32, 1, 8, 2112, 128
    k, v, w = make(3, L, B, H, S, hd, "bf16")
    rows = [(0, 0, 0), (13, 0, 5), (31, 0, 7)]
    check(es, k, v, w, [2048], [1024], 128, 1024, rows=rows)
    check(es, k, v, w, [2048], [1024], 128, in_place=True, rows=rows)
    layout = es.easyspec_kv_layout(L, B, H, S, hd, es.EASYSPEC_DTYPE_BF16)
    out = [torch.zeros(L, B, H, 1024, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    wo, so = torch.zeros(L, B, H, 1024, device="cuda"), torch.zeros(L, B, H, 1024, dtype=torch.int32, device="cuda")
    run = lambda: es.easyspec_kv_evict(k, v, w, layout, [2048], [1024], 128, 1024, out[0], out[1], wo, so, torch.cuda.current_stream().cuda_stream)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for seed in range(3):
        w.copy_(make(50 + seed, L, B, H, S, hd, "bf16")[2])
        so.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        for l, b, h in rows:
            assert np.array_equal(so[l, b, h].cpu().numpy(), ref.kept_slots(w[l, b, h].cpu().numpy(), 2048, 1024, 128))


def test_more_rows_than_a_grid_extent(es):
    """72 000 (layer, sequence, KV head) rows: the moving launch goes in pieces."""
    L, B, H, S, hd = 4500, 2, 8, 6, 64
    k, v, w = make(9, L, B, H, S, hd, "bf16")
    rows = [(0, 0, 0), (4095, 1, 7), (4096, 0, 0), (4499, 1, 7), (2500, 0, 3)]
    check(es, k, v, w, [6, 5], [4, 2], 1, 4, rows=rows)
    check(es, k, v, w, [6, 5], [4, 2], 1, in_place=True, rows=rows)


def test_rows_that_the_selecting_workgroup_moves_and_those_it_does_not(es):
    """Up to 256 rows and 32 KB of K a list is moved at once; one row more is another launch."""
    for hd, dtype, most in ((64, "bf16", 256), (64, "fp32", 128), (128, "bf16", 128), (128, "fp32", 64)):
        for S in (700, 3000):
            k, v, w = make(S + most, 2, 2, 1, S, hd, dtype)
            for keep in (most, most + 1):
                check(es, k, v, w, [S, S - 1], [keep, keep - 3], 7, keep)
                check(es, k, v, w, [S, S - 1], [keep, keep - 3], 7, in_place=True)


@pytest.mark.parametrize("in_place", [False, True])
def test_offsets_beyond_32_bits(es, in_place):
    """Caches of more than 2^31 elements and 4 GiB: the last rows, of a long sequence and a short one."""
    import torch
    L, B, H, S, hd = 2, 16, 17, 65536, 64
    k, v = (torch.zeros(L, B, H, S, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert k.numel() > 1 << 31
    w = torch.zeros(L, B, H, S, device="cuda")
    few = make(70, 1, 2, H, S, hd, "bf16")
    for whole, part in zip((k, v, w), few):
        whole[-1, 14:] = part[0]
    lens, keep, So = [0] * 14 + [70, S], [8] * 14 + [50, 1000], S if in_place else 1000
    layout = es.easyspec_kv_layout(L, B, H, S, hd, es.EASYSPEC_DTYPE_BF16)
    slots = torch.full((L, B, H, So), -9, dtype=torch.int32, device="cuda")
    ko, vo, wo = (k, v, w) if in_place else (torch.zeros(L, B, H, So, *x, dtype=t, device="cuda") for x, t in (((hd,), k.dtype), ((hd,), k.dtype), ((), w.dtype)))
    torch.cuda.synchronize()
    es.easyspec_kv_evict(k, v, w, layout, lens, keep, 30, So, ko, vo, wo, slots, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for b in (0, 1):
        for h in (0, H - 1):
            kept = ref.kept_slots(few[2][0, b, h].cpu().numpy(), lens[14 + b], keep[14 + b], 30)
            assert np.array_equal(slots[-1, 14 + b, h, :len(kept)].cpu().numpy(), kept) and torch.all(slots[-1, 14 + b, h, len(kept):] == -9)
            at = torch.from_numpy(kept.astype(np.int64)).cuda()
            for got, was in zip((ko, vo, wo), few):
                assert torch.equal(got[-1, 14 + b, h, :len(kept)], was[0, b, h].index_select(0, at))
    assert torch.all(slots[:, :14] == -9) and not bool(ko[:, :14].any()) and not bool(vo[:, :14].any()) and not bool(wo[:, :14].any())
