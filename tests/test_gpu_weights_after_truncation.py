"""Tracked attention weights of a sequence that is cut back and goes on with other tokens: slots that stay keep what the tokens cut off
gave them, slots that are filled again start from zero."""
import numpy as np
import pytest

import easyspec_synth as synth
from plain_decoder import Decoder
from tolerances import PLAIN_TOL, TOL

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name,dtype,batch", [("tiny", "fp32", 1), ("tiny_qwen", "bf16", 1), ("tiny", "bf16", 2)])
def test_cut_back_and_on(name, dtype, batch):
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device; none is visible")
    import gpu_harness as gpu
    es = gpu.es
    cfg = synth.model_shape(name, dtype=dtype)
    w = synth.make_weights(cfg, 61)
    tol = TOL["fp32"] if dtype == "fp32" else PLAIN_TOL
    g, d = gpu.GpuDrafter(cfg, w, max_batch=batch, max_ctx=96), Decoder(cfg, w)
    V, cut, at = cfg["vocab"], 19, 0
    toks = [int(t) for t in synth.make_tokens(62, 60, V)]
    try:
        es.easyspec_track_attention(g.ctx, 96)

        def feed(n):
            nonlocal at
            t, at = toks[at:at + n], at + n
            _, logits = g.calibrate({b: t for b in range(batch)})
            want = d.calibrate(t)
            for b in range(batch):
                gpu.assert_close(logits[b], want, tol, "logits")

        def check():
            for b in range(batch):
                got = np.full((cfg["n_layers"], cfg["n_kv_heads"], d.precise), np.nan, np.float32)
                es.easyspec_get_attn_weights(g.ctx, b, got, d.precise)
                gpu.assert_close(got, np.array(d.weight), tol, f"weights of sequence {b}")
            return got

        feed(16)
        feed(9)
        before = check()
        for b in range(batch):
            es.easyspec_truncate(g.ctx, b, cut)
        d.thin([[np.arange(cut)] * cfg["n_kv_heads"]] * cfg["n_layers"])
        d.pos = cut
        kept = check()
        assert np.array_equal(kept, before[:, :, :cut])
        feed(7)
        feed(1)
        got = check()
        # every row gives one in all: 25 tokens' rows, less what the six cut off gave to their own slots, and eight tokens' more
        rows = cfg["n_q_heads"] // cfg["n_kv_heads"]
        want = 33 * rows - before[:, :, cut:].astype(np.float64).sum(-1)
        assert np.all(np.abs(got.astype(np.float64).sum(-1) - want) < want * 1e-4)
        es.easyspec_evict(g.ctx, [12] + [-1] * (batch - 1), 4)
        assert list(es.easyspec_get_evicted(g.ctx, batch))[0] == 15
    finally:
        g.close()
