"""A context's cache held in 4 bits and brought back: exported, stored, loaded, imported into another context, which goes on from it."""
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


@pytest.mark.parametrize("name,dtype", [("tiny", "fp32"), ("tiny", "bf16"), ("tiny_qwen", "fp32"), ("tiny_qwen", "bf16")])
@pytest.mark.parametrize("n", [1, 63, 150])
def test_a_context_goes_on_from_a_cache_of_four_bits(gpu, name, dtype, n):
    import torch
    es = gpu.es
    cfg = synth.model_shape(name, dtype=dtype)
    weights = synth.make_weights(cfg, 11)
    rng = np.random.default_rng(n)
    tokens = rng.integers(0, cfg["vocab"], n + 7).tolist()
    L, H, hd = cfg["n_layers"], cfg["n_kv_heads"], cfg["head_dim"]
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    first = gpu.GpuDrafter(cfg, weights, max_ctx=256)
    first.prefill(0, tokens[:n])
    k, v = (torch.zeros(L, H, n, hd, dtype=dt, device="cuda") for _ in range(2))
    es.easyspec_kv_export(first.ctx, 0, k, v, n)
    first.close()
    cache = K.Cache(es, L, 1, H, 200, hd, dtype)
    k_out, v_out = (torch.full((L, H, n, hd), 7.0, dtype=dt, device="cuda") for _ in range(2))
    es.easyspec_kvq_store(k, v, cache.layout, n, [0], [n], [0], [n], cache.c, K.stream())
    es.easyspec_kvq_load(cache.c, cache.layout, [0], [n], n, [0], k_out, v_out, K.stream())
    torch.cuda.synchronize()
    held = [ref.decode(*ref.encode(x.double().cpu().numpy())) for x in (k, v)]
    for got, want in zip((k_out, v_out), held):
        assert np.array_equal(got.double().cpu().numpy(), want)
    results = []
    for k_in, v_in in ((k_out, v_out), [torch.from_numpy(x).to(dt) for x in held]):          # from the device; the same numbers from the host
        if not k_in.is_cuda:
            k_in, v_in = (x.view(torch.int16 if dtype == "bf16" else torch.int32).numpy() for x in (k_in, v_in))
        g = gpu.GpuDrafter(cfg, weights, max_ctx=256)
        g.import_kv(0, k_in, v_in) if isinstance(k_in, np.ndarray) else es.easyspec_kv_import(g.ctx, 0, k_in, v_in, n)
        back = g.export_kv(0, n)
        for got, want in zip(back, held):
            assert np.array_equal(got.astype(np.float64), want)
        assert [int(x[0]) for x in g.lens()] == [n, 0]
        nxt, logits = g.calibrate({0: tokens[n:]})
        drafted, drafted_logits = g.draft_step({0: nxt[0]})
        results.append((nxt[0], logits[0], drafted, drafted_logits))
        assert np.isfinite(logits[0]).all() and np.isfinite(drafted_logits).all()
        g.close()
    for a, b in zip(*results):
        assert np.array_equal(a, b)
