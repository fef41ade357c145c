"""Per-kernel timing of calibrations whose attention weights are tracked: the kernels that make the weights are launches of the pass."""
import numpy as np
import pytest

import easyspec_synth as synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device; none is visible")
    import gpu_harness
    return gpu_harness


def profiled(gpu, cfg, w, track, calibs, op, **kw):
    """[(launches' classes)] of every calibration, and all their logits."""
    g = gpu.GpuDrafter(cfg, w, **kw)
    try:
        if track:
            gpu.es.easyspec_track_attention(g.ctx, kw["max_ctx"])
        out, logits = [], []
        for toks in calibs:
            per, ops = np.zeros(4096, np.float32), np.full(4096, -1, np.int32)
            gpu.es.easyspec_profile_begin(g.ctx, op, 4096)
            _, lg = g.calibrate(toks)
            n, total = gpu.es.easyspec_profile_end(g.ctx, per, ops)
            assert abs(float(per[:n].sum()) - total) < 1e-3 * total + 1e-6 and (op != gpu.es.EASYSPEC_OP_ALL or np.all(per[:n] > 0.0005))
            out.append(list(ops[:n]))
            logits.append(lg)
        return out, logits
    finally:
        g.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_every_launch_of_a_tracked_calibration_is_timed(gpu, dtype):
    """One pass (short contexts: one kernel of weights a layer; from 257 slots on in bf16, 129 in fp32: two) and passes of 16 columns and
    more: a wide one in bf16, two at a time in fp32, each with weights of its own.  The others' launches stay what they were."""
    es = gpu.es
    cfg = synth.model_shape("tiny", dtype=dtype)
    w = synth.make_weights(cfg, 42)
    toks = [int(t) for t in synth.make_tokens(43, 300, cfg["vocab"])]
    long = [{0: toks[i:i + 16]} for i in range(0, 288, 16)]
    both = [{0: toks[:16], 1: toks[16:32]}]
    kw = dict(max_batch=2, max_ctx=320)
    for calibs, extra in ((long + [{0: toks[288:294]}], None), (both, 1 if dtype == "bf16" else 2)):
        tracked, a = profiled(gpu, cfg, w, True, calibs, es.EASYSPEC_OP_ALL, **kw)
        plain, b = profiled(gpu, cfg, w, False, calibs, es.EASYSPEC_OP_ALL, **kw)
        slots = 0
        for i, (t, p) in enumerate(zip(tracked, plain)):
            slots += len(calibs[i][0])
            want = extra if extra else 1 if slots <= (256 if dtype == "bf16" else 128) else 2
            assert t.count(es.EASYSPEC_OP_ALL) - p.count(es.EASYSPEC_OP_ALL) == want * cfg["n_layers"], (i, slots)
            assert [x for x in t if x != es.EASYSPEC_OP_ALL] == [x for x in p if x != es.EASYSPEC_OP_ALL]
        for x, y in zip(a, b):
            for s in x:
                assert np.array_equal(x[s], y[s])           # tracking changes no logit
    attn = profiled(gpu, cfg, w, True, both, es.EASYSPEC_OP_ATTN, **kw)[0]
    assert attn == profiled(gpu, cfg, w, False, both, es.EASYSPEC_OP_ATTN, **kw)[0]
