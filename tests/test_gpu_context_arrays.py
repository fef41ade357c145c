"""Host arrays with an entry per sequence, on contexts: a list that is too short is refused before anything reads it."""
import pytest

import easyspec_synth as synth

pytestmark = pytest.mark.gpu


def test_lists_of_another_length_than_max_batch():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device; none is visible")
    import gpu_harness
    es = gpu_harness.es
    cfg = synth.model_shape("tiny")
    g = gpu_harness.GpuDrafter(cfg, synth.make_weights(cfg, 41), max_batch=3, max_ctx=64)
    try:
        es.easyspec_track_attention(g.ctx, 64)
        g.calibrate({b: [1, 2, 3, 4, 5, 6] for b in range(3)})
        for call in (lambda: es.easyspec_evict(g.ctx, [3, 3], 1), lambda: es.easyspec_evict(g.ctx, [3] * 4, 1),
                     lambda: es.easyspec_get_evicted(g.ctx, 2)):
            with pytest.raises(es.EasySpecError) as e:
                call()
            assert e.value.code == es.EASYSPEC_EINVAL
        assert list(g.lens()[0]) == [6, 6, 6]
        es.easyspec_evict(g.ctx, [3, -1, 3], 1)
        assert list(g.lens()[0]) == [3, 6, 3] and list(es.easyspec_get_evicted(g.ctx, 3)) == [3, 0, 3]
    finally:
        g.close()
