"""The operators together, as a program uses them: tokens drafted by sampling on a context and accepted under the same filter; a context's
cache held in 4 bits, appended to, its blocks selected and attended to."""
import numpy as np
import pytest

import easyspec_synth as synth
import kvq_gpu as K
import kvq_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device; none is visible")
    import gpu_harness
    return gpu_harness


@pytest.mark.parametrize("setting", [(1.0, 50, 0.95, 0.0), (0.8, 0, 0.9, 0.02), (0.6, 8, 1.0, 0.0)])
def test_sampled_drafts_are_accepted_under_the_same_filter(gpu, oracle, setting):
    """Three users, four drafted tokens each; nothing is looked at on the host until all is done."""
    import torch
    es, B, gamma = gpu.es, 3, 4
    cfg = synth.model_shape("tiny")
    g = gpu.GpuDrafter(cfg, synth.make_weights(cfg, 5), max_batch=B, max_ctx=64)
    g.set_groups([0, 1, 3, 4])
    V, T = cfg["vocab"], setting[0]
    rng = np.random.default_rng(17)
    first, _ = g.calibrate({b: rng.integers(0, V, 5 + b).tolist() for b in range(B)})
    u = torch.from_numpy(rng.random((gamma, B), dtype=np.float32)).cuda()
    r, u_bonus = (torch.from_numpy(rng.random(s, dtype=np.float32)).cuda() for s in ((B, gamma), (B,)))
    noise = torch.from_numpy(rng.normal(0, 0.5, (B, gamma + 1, V)).astype(np.float32)).cuda()
    tok = torch.tensor([first[b] for b in range(B)], dtype=torch.int32, device="cuda")
    draft = torch.zeros(gamma, B, dtype=torch.int32, device="cuda")
    raw, kept = (torch.zeros(gamma, B, V, device="cuda") for _ in range(2))
    argmax = torch.zeros(B, dtype=torch.int32, device="cuda")
    ws = torch.empty(es.easyspec_sample_workspace_bytes(B * (gamma + 1), V) // 4 + 4, device="cuda")
    stream = K.stream()
    for i in range(gamma):
        es.easyspec_draft_step(g.ctx, tok if i == 0 else draft[i - 1], argmax, raw[i])
        raw[i] *= 40.0                                   # a random model's logits hardly differ
        es.easyspec_sample(raw[i], u[i], B, V, *setting, draft[i], kept[i], ws, stream)
    target = (raw.transpose(0, 1)[:, [0, 1, 2, 3, 3]] + noise).contiguous()
    target_kept = torch.empty_like(target)
    es.easyspec_sample(target, None, B * (gamma + 1), V, *setting, None, target_kept, ws, stream)
    lens, bonus = (torch.full((B,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    aws = torch.empty(es.easyspec_accept_workspace_bytes(B, gamma, V) // 8, dtype=torch.float64, device="cuda")
    d, dl = draft.t().contiguous(), kept.transpose(0, 1).contiguous()
    es.easyspec_accept(d, dl, target_kept, r, u_bonus, B, gamma, V, T, lens, bonus, aws, stream)
    torch.cuda.synchronize()
    raw, kept, draft = raw.cpu().numpy(), kept.cpu().numpy(), draft.cpu().numpy()
    for i in range(gamma):
        for b in range(B):
            token, left = ref.sample(raw[i, b], float(u[i, b]), *setting)
            assert draft[i, b] == token and np.array_equal(kept[i, b], left)
    for b in range(B):
        left = np.stack([ref.sample(target[b, i].cpu().numpy(), None, *setting)[1] for i in range(gamma + 1)])
        assert np.array_equal(target_kept[b].cpu().numpy(), left)
        m, token = oracle.accept(draft[:, b], kept[:, b], left, r[b].cpu().numpy(), float(u_bonus[b]), T)[:2]
        assert (int(lens[b]), int(bonus[b])) == (m, token)
        assert left[m, token] > -np.inf                  # what is drawn is what the filter leaves
    g.close()


@pytest.mark.parametrize("name", ["tiny", "tiny_qwen"])
def test_a_contexts_cache_in_four_bits(gpu, name):
    """A prompt's cache is exported and held in 4 bits, grows by the tokens of three calibrations, and is read by blocks and whole."""
    import torch
    es = gpu.es
    cfg = synth.model_shape(name)
    g = gpu.GpuDrafter(cfg, synth.make_weights(cfg, 9), max_ctx=256)
    L, H, Hq, hd, S = cfg["n_layers"], cfg["n_kv_heads"], cfg["n_q_heads"], cfg["head_dim"], 200
    rng = np.random.default_rng(3)
    g.prefill(0, rng.integers(0, cfg["vocab"], 150).tolist())
    cache = K.Cache(es, L, 1, H, S, hd, cfg["dtype"])
    dt = torch.float32 if cfg["dtype"] == "fp32" else torch.bfloat16

    def take(first, n):
        held = first + n
        k, v = (torch.zeros(L, H, held, hd, dtype=dt, device="cuda") for _ in range(2))
        es.easyspec_kv_export(g.ctx, 0, k, v, held)
        es.easyspec_kvq_store(k, v, cache.layout, held, [first], [n], [first], [held], cache.c, K.stream())
        torch.cuda.synchronize()
        return k.double().cpu().numpy(), v.double().cpu().numpy()
    take(0, 150)
    held = 150
    for n in (1, 6, 16):
        g.calibrate({0: rng.integers(0, cfg["vocab"], n).tolist()})
        k, v = take(held, n)
        held += n
        codes = cache.bytes()
        for got, want in zip(codes[:4], (*ref.encode(k), *ref.encode(v))):
            assert np.array_equal(got[:, 0, :, :held], want)
        q = K.dev(K.queries(held, L, n, Hq, hd))
        blocks = K.select(cache, q, [n], [held], 1, 1, 2)
        sparse = K.attend(cache, q, [n], [held], blocks)
        dense = K.attend(cache, q, [n], [held])
        torch.cuda.synchronize()
        bounds = np.stack([[ref.bounds_of(ref.decode(codes[0], codes[1])[layer, 0, h, j * 64:min(j * 64 + 64, held)]) for j in range((held + 63) // 64)]
                           for layer in range(L) for h in range(H)]).reshape(L, 1, H, -1, 2, hd)
        assert np.array_equal(cache.bounds.float().cpu().numpy()[:, :, :, :bounds.shape[3]], bounds)
        assert np.array_equal(blocks.cpu().numpy(), ref.select(q.double().cpu().numpy(), bounds, [n], [held], 1, 1, 2))
        values = cache.values()
        for out, lists in ((sparse, blocks.cpu().numpy()), (dense, None)):
            want, tol = ref.attention(q.double().cpu().numpy(), *values, [n], [held], lists)
            assert np.all(np.abs(out.double().cpu().numpy() - want) <= tol)
    g.close()
