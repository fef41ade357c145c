"""easyspec_track_attention on a device without room for one of its arrays: the context stays what it was and holds nothing more."""
import numpy as np
import pytest

import easyspec_synth as synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_call_that_cannot_allocate_leaves_the_context_as_it_was(dtype):
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device; none is visible")
    import gpu_harness
    es = gpu_harness.es
    cfg = synth.model_shape("tiny", dtype=dtype)
    w = synth.make_weights(cfg, 51)
    toks = [int(t) for t in synth.make_tokens(52, 40, cfg["vocab"])]

    def run(fails):
        g = gpu_harness.GpuDrafter(cfg, w, max_batch=16, max_ctx=4096)       # weights and list of slots: 2 MiB each, table 128 MiB
        out = []
        try:
            for i in range(4 if fails else 0):                              # weights, list of slots, workspace, rotary table
                torch.cuda.synchronize()
                free = torch.cuda.mem_get_info()[0]
                es.easyspec_deny_allocation(g.ctx, i)
                with pytest.raises(es.EasySpecError) as e:
                    es.easyspec_track_attention(g.ctx, 1 << 19)
                assert e.value.code == es.EASYSPEC_EHIP
                assert torch.cuda.mem_get_info()[0] == free, i
                with pytest.raises(es.EasySpecError) as e:
                    es.easyspec_evict(g.ctx, [4] * 16, 1)
                assert e.value.code == es.EASYSPEC_ESTATE
                es.easyspec_poison_workspaces(g.ctx)                        # none of them is gone
                out.append(g.calibrate({0: toks[4 * i: 4 * i + 4]})[1][0])  # and no pass reports the failure again
                out.append(g.draft_step({0: 7})[1][0])
                es.easyspec_truncate(g.ctx, 0, 0)
            es.easyspec_track_attention(g.ctx, 1 << 19)
            g.calibrate({0: toks[:16]})
            weights = np.full((cfg["n_layers"], cfg["n_kv_heads"], 16), np.nan, np.float32)
            es.easyspec_get_attn_weights(g.ctx, 0, weights, 16)
            es.easyspec_evict(g.ctx, [9] + [-1] * 15, 3)
            out.append(g.draft_step({0: 5})[1][0])
            return out, weights
        finally:
            g.close()

    run(False)                                                              # what a process's first context leaves in the allocator
    (_, want), (tail, got) = run(False), run(True)
    assert np.array_equal(want, got) and np.all(np.isfinite(got))
    assert all(np.all(np.isfinite(x)) for x in tail)
    plain = gpu_harness.GpuDrafter(cfg, w, max_batch=16, max_ctx=4096)
    try:
        for i in range(4):
            assert np.array_equal(plain.calibrate({0: toks[4 * i: 4 * i + 4]})[1][0], tail[2 * i])
            assert np.array_equal(plain.draft_step({0: 7})[1][0], tail[2 * i + 1])
            es.easyspec_truncate(plain.ctx, 0, 0)
    finally:
        plain.close()
