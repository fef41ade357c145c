"""The beams' caches in the order of their parents (easyspec_kv_reorder): bytes are moved, so results are equal."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def es():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device; none is visible")
    import paper_2502_02493_amd as es
    return es


def caches(seed, shape, dtype):
    import torch
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    return [torch.empty(shape, dtype=dtype, device="cuda:0").normal_(generator=g) for _ in range(2)]


def want(src, out, parents, beams, a, z):
    res = out.clone()
    for i, p in enumerate(parents):
        j = i - i % beams + p if 0 <= p < beams else i
        res[:, i, :, a:z] = src[:, j, :, a:z]
    return res


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("L,B,W,H,S,hd,dtype,a,z", [
    (1, 1, 1, 1, 1, 64, "bf16", 0, 1), (2, 2, 2, 3, 9, 64, "fp32", 0, 9), (3, 4, 4, 2, 37, 128, "bf16", 5, 6), (2, 5, 5, 1, 61, 64, "bf16", 60, 61),
    (5, 8, 4, 2, 130, 128, "fp32", 1, 129), (4, 16, 16, 8, 70, 128, "bf16", 33, 70), (2, 15, 3, 1, 257, 64, "fp32", 0, 257),
    (32, 4, 2, 8, 300, 128, "bf16", 250, 255), (2, 9, 3, 7, 20, 64, "bf16", 7, 7), (9000, 2, 2, 8, 2, 64, "bf16", 0, 2),
])
def test_reorder(es, in_place, L, B, W, H, S, hd, dtype, a, z):
    import torch
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    rng = np.random.default_rng(L * B + S)
    k, v = caches(S, (L, B, H, S, hd), dt)
    layout = es.easyspec_kv_layout(L, B, H, S, hd, es.EASYSPEC_DTYPE_BF16 if dtype == "bf16" else es.EASYSPEC_DTYPE_F32)
    orders = [rng.integers(0, W, B), np.zeros(B, int), (np.arange(B) + 1) % W, np.where(rng.random(B) < 0.5, rng.choice([-1, -5, W, 1 << 30], B), rng.integers(0, W, B))]
    for parents in orders:
        ko, vo = (k.clone(), v.clone()) if in_place else caches(S + 1, (L, B, H, S, hd), dt)
        ks, vs = (ko, vo) if in_place else (k, v)
        wk, wv = want(k, ko, parents, W, a, z), want(v, vo, parents, W, a, z)
        p = torch.from_numpy(parents.astype(np.int32)).cuda()
        es.easyspec_kv_reorder(ks, vs, layout, p, W, a, z, ko, vo, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(ko.view(torch.uint8), wk.view(torch.uint8)) and torch.equal(vo.view(torch.uint8), wv.view(torch.uint8)), parents


def test_non_finite_values_move_as_they_are(es):
    import torch
    k, v = caches(1, (1, 2, 1, 16, 64), torch.float32)
    k[0, 0, 0, 3], v[0, 1, 0, 2] = float("nan"), float("inf")
    layout = es.easyspec_kv_layout(1, 2, 1, 16, 64, es.EASYSPEC_DTYPE_F32)
    wk, wv = want(k, k, [1, 0], 2, 0, 16), want(v, v, [1, 0], 2, 0, 16)
    es.easyspec_kv_reorder(k, v, layout, torch.tensor([1, 0], dtype=torch.int32, device="cuda"), 2, 0, 16, k, v, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(k.view(torch.int32), wk.view(torch.int32)) and torch.equal(v.view(torch.int32), wv.view(torch.int32))


def test_offsets_beyond_32_bits(es):
    """A cache of more than 4 GiB: the last rows move."""
    import torch
    L, B, H, S, hd = 36, 2, 8, 65536, 64
    k = torch.zeros(L, B, H, S, hd, dtype=torch.bfloat16, device="cuda")
    assert k.numel() * 2 > 4 << 30
    k[-1, 1, -1, -2:] = 3.0
    k[-1, 0, -1, -2:] = 5.0
    v = torch.zeros_like(k)
    v[-1, 0, 0, -1] = 7.0
    layout = es.easyspec_kv_layout(L, B, H, S, hd, es.EASYSPEC_DTYPE_BF16)
    es.easyspec_kv_reorder(k, v, layout, torch.tensor([1, 0], dtype=torch.int32, device="cuda"), 2, S - 1, S, k, v, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert float(k[-1, 0, -1, -1, 9]) == 3.0 and float(k[-1, 1, -1, -1, 9]) == 5.0 and float(k[-1, 0, -1, -2, 9]) == 5.0
    assert float(v[-1, 1, 0, -1, 0]) == 7.0 and float(v[-1, 0, 0, -1, 0]) == 0.0
    assert float(k.float().abs().sum()) == 64 * 2 * 8.0
