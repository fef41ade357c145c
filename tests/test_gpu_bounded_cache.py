"""Tracked attention weights, eviction and beams on a context (easyspec_track_attention, _evict, _beam_fork, _beam_reorder and their
readers), against a plain float64 decoder whose cache is thinned and copied alike."""
import numpy as np
import pytest

import easyspec_synth as synth
import operator_ref as ref
from plain_decoder import Decoder
from tolerances import PLAIN_TOL, TOL

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device; none is visible")
    import gpu_harness
    return gpu_harness


def tol(cfg):
    return TOL["fp32"] if cfg["dtype"] == "fp32" else PLAIN_TOL


def model(gpu, name, seed, track=0, **over):
    kw = {k: over.pop(k) for k in ("max_batch", "max_ctx", "max_calib") if k in over}
    cfg = synth.model_shape(name, **over)
    w = synth.make_weights(cfg, seed)
    g = gpu.GpuDrafter(cfg, w, **kw)
    if track:
        gpu.es.easyspec_track_attention(g.ctx, track)
    return g, Decoder(cfg, w)


def weights_of(gpu, g, b, n):
    c = g.cfg
    out = np.full((c["n_layers"], c["n_kv_heads"], n), np.nan, np.float32)
    gpu.es.easyspec_get_attn_weights(g.ctx, b, out, n)
    return out


def assert_weights(gpu, g, b, d):
    got = weights_of(gpu, g, b, d.precise)
    gpu.assert_close(got, np.array([[x for x in layer] for layer in d.weight]), tol(g.cfg), f"weights of sequence {b}")
    # every row gives one in all
    return got


def evict(gpu, g, decoders, keep, recent):
    """decoders {b: Decoder}; the reference keeps the slots that the library's own weights name."""
    k = np.full(g.B, -1, np.int32)
    kept = {}
    for b, n in keep.items():
        k[b] = n
        d = decoders[b]
        w = weights_of(gpu, g, b, d.precise)
        kept[b] = [[ref.kept_slots(w[i, j], d.precise, n, recent) for j in range(g.cfg["n_kv_heads"])] for i in range(g.cfg["n_layers"])]
    before = {b: g.export_kv(b, decoders[b].precise) for b in decoders}
    gpu.es.easyspec_evict(g.ctx, k, recent)
    for b, d in decoders.items():
        if b not in kept:
            continue
        if keep[b] < d.precise:
            d.thin(kept[b])
        for got, was in zip(g.export_kv(b, d.precise), before[b]):
            for i in range(g.cfg["n_layers"]):
                for j in range(g.cfg["n_kv_heads"]):
                    assert np.array_equal(got[i, j], was[i, j][kept[b][i][j]]), (b, i, j)


SHAPES = [("tiny", {}), ("tiny_qwen", {}), ("tiny", dict(dtype="bf16")), ("tiny_qwen", dict(dtype="bf16"))]


@pytest.mark.parametrize("name,over", SHAPES)
def test_tracked_weights(gpu, name, over):
    """Narrow, paired and wide passes; ragged chunks; a sequence that waits; fuzzy steps in between leave no trace."""
    g, d0 = model(gpu, name, 31, track=128, max_batch=3, max_ctx=128, **over)
    try:
        V = g.cfg["vocab"]
        ds = {b: d0.clone() for b in range(3)}
        rng = np.random.default_rng(5)
        for sizes in ((16, 16, 16), (5, 0, 16), (1, 3, 0), (6, 16, 2), (0, 1, 0)):
            toks = {b: list(rng.integers(0, V, n)) for b, n in enumerate(sizes) if n}
            _, logits = g.calibrate(toks)
            for b, t in toks.items():
                gpu.assert_close(logits[b], ds[b].calibrate(t), tol(g.cfg), "logits")
            g.draft_step({b: 3 for b in range(3)})
        for b in range(3):
            got = assert_weights(gpu, g, b, ds[b])
            rows = ds[b].precise * g.cfg["n_q_heads"] // g.cfg["n_kv_heads"]
            assert np.all(np.abs(got.astype(np.float64).sum(-1) - rows) < rows * 1e-4)
    finally:
        g.close()


@pytest.mark.parametrize("name,over", SHAPES)
def test_eviction_and_what_follows(gpu, route, name, over):
    import torch
    g, d0 = model(gpu, name, 32, track=300, max_batch=2, max_ctx=80, **over)
    es = gpu.es
    try:
        cfg, V = g.cfg, g.cfg["vocab"]
        bounds = es.easyspec_default_groups(cfg["n_layers"], 2, es.EASYSPEC_POLICY_PACKED)
        g.set_groups(bounds)
        ds = {0: d0.clone(), 1: d0.clone()}
        rng = np.random.default_rng(6)

        def feed(sizes):
            toks = {b: list(rng.integers(0, V, n)) for b, n in sizes.items()}
            _, logits = g.calibrate(toks)
            for b, t in toks.items():
                gpu.assert_close(logits[b], ds[b].calibrate(t), tol(cfg), "logits")

        def draft(n):
            for _ in range(n):
                t = {b: int(rng.integers(0, V)) for b in ds}
                _, logits = g.draft_step(t)
                for b in ds:
                    gpu.assert_close(logits[b], ds[b].draft(t[b], bounds), tol(cfg), "fuzzy logits")

        for _ in range(4):
            feed({0: 16, 1: 13})
        draft(2)
        evict(gpu, g, ds, {0: 20, 1: 100}, 6)           # the second keeps what it has, its fuzzy slots too
        p, f = g.lens()
        assert list(p) == [20, 52] and list(f) == [0, 2]
        assert list(es.easyspec_get_evicted(g.ctx, 2)) == [44, 0]
        draft(3)
        feed({0: 5, 1: 1})
        for b in ds:
            assert_weights(gpu, g, b, ds[b])
        for i in range(14):                             # on and on: far more tokens than slots
            feed({0: 11, 1: 7})
            evict(gpu, g, ds, {b: 24 - b for b in ds if ds[b].precise > 40}, 9)
            draft(1)
        assert ds[0].pos > 2 * 80
        got = es.easyspec_get_evicted(g.ctx, 2)
        p, f = g.lens()
        for b in ds:
            assert p[b] + f[b] + got[b] == ds[b].pos
            assert_weights(gpu, g, b, ds[b])
        # a token tree after an eviction: its nodes' positions go on too
        g.calibrate({0: [1]}), ds[0].calibrate([1])
        _, logits = g.draft_tree_step({0: ([5, 7], [-1, -1])})
        _, deeper = g.draft_tree_step({0: ([9], [1])})
        one, two = ds[0].clone(), ds[0].clone()
        gpu.assert_close(logits[0][0], one.draft(5, bounds), tol(cfg), "tree")
        gpu.assert_close(logits[0][1], two.draft(7, bounds), tol(cfg), "tree")
        gpu.assert_close(deeper[0][0], two.draft(9, bounds), tol(cfg), "tree")
        torch.cuda.synchronize()
    finally:
        g.close()


def test_positions_run_out(gpu):
    g, _ = model(gpu, "tiny", 33, track=40, max_batch=1, max_ctx=32)
    es = gpu.es
    try:
        g.calibrate({0: list(range(16))})
        g.calibrate({0: list(range(14))})
        es.easyspec_evict(g.ctx, [10], 4)
        g.calibrate({0: list(range(9))})                # positions 30 .. 38
        g.draft_step({0: 1})                            # 39, the last
        for call in (lambda: g.draft_step({0: 1}), lambda: g.calibrate({0: [1, 2]}),):
            with pytest.raises(es.EasySpecError) as e:
                call()
            assert e.value.code == es.EASYSPEC_ECAPACITY
        g.calibrate({0: [1]})                           # the fuzzy slot is dropped: one position is left
        with pytest.raises(es.EasySpecError) as e:
            g.draft_tree_step({0: ([1], [-1])})
        assert e.value.code == es.EASYSPEC_ECAPACITY
        assert list(g.lens()[0]) == [20]
    finally:
        g.close()


def test_refusals(gpu):
    import torch
    es = gpu.es
    g, _ = model(gpu, "tiny", 34, max_batch=3, max_ctx=64)
    par = torch.zeros(3, dtype=torch.int32, device="cuda")

    def refused(code, f, *a):
        with pytest.raises(es.EasySpecError) as e:
            f(*a)
        assert e.value.code == code, str(e.value)

    try:
        buf = np.zeros((4, 2, 8), np.float32)
        refused(es.EASYSPEC_ESTATE, es.easyspec_evict, g.ctx, [4, 4, 4], 1)
        refused(es.EASYSPEC_ESTATE, es.easyspec_get_attn_weights, g.ctx, 0, buf, 1)
        refused(es.EASYSPEC_ESTATE, es.easyspec_beam_fork, g.ctx, 0, 0, 2)
        refused(es.EASYSPEC_ESTATE, es.easyspec_beam_reorder, g.ctx, 0, 2, par, 0)
        for n in (63, 0, -1, (1 << 20) + 1):
            refused(es.EASYSPEC_EINVAL, es.easyspec_track_attention, g.ctx, n)
        es.easyspec_track_attention(g.ctx, 64)
        refused(es.EASYSPEC_ESTATE, es.easyspec_track_attention, g.ctx, 64)
        g.calibrate({0: [1, 2, 3, 4, 5, 6, 7, 8], 1: [4, 5]})
        for a in ((3, 0, 1), (-1, 0, 1), (0, -1, 1), (0, 0, 0), (0, 1, 3), (0, 3, 1)):
            refused(es.EASYSPEC_EINVAL, es.easyspec_beam_fork, g.ctx, *a)
        refused(es.EASYSPEC_ESTATE, es.easyspec_beam_fork, g.ctx, 2, 0, 2)
        refused(es.EASYSPEC_ESTATE, es.easyspec_beam_reorder, g.ctx, 0, 2, par, 0)     # of two lengths
        refused(es.EASYSPEC_ESTATE, es.easyspec_beam_reorder, g.ctx, 0, 3, par, 0)
        refused(es.EASYSPEC_EINVAL, es.easyspec_beam_reorder, g.ctx, 0, 1, par, 9)
        refused(es.EASYSPEC_EINVAL, es.easyspec_beam_reorder, g.ctx, 0, 1, par, -1)
        refused(es.EASYSPEC_EINVAL, es.easyspec_beam_reorder, g.ctx, 0, 1, None, 0)
        refused(es.EASYSPEC_EINVAL, es.easyspec_beam_reorder, g.ctx, 2, 2, par, 0)
        refused(es.EASYSPEC_EINVAL, es.easyspec_evict, g.ctx, [4, -1, -1], -1)
        refused(es.EASYSPEC_EINVAL, es.easyspec_evict, g.ctx, [0, -1, -1], 1)
        refused(es.EASYSPEC_EINVAL, es.easyspec_get_attn_weights, g.ctx, 3, buf, 1)
        refused(es.EASYSPEC_EINVAL, es.easyspec_get_attn_weights, g.ctx, 0, buf, 9)
        g.draft_tree_step({0: ([1], [-1])})
        refused(es.EASYSPEC_ESTATE, es.easyspec_beam_reorder, g.ctx, 0, 1, par, 0)
        assert [list(x) for x in g.lens()] == [[8, 2, 0], [1, 0, 0]]                  # nothing of that changed anything
        es.easyspec_evict(g.ctx, [6, -1, -1], 2)
        assert [list(x) for x in g.lens()] == [[6, 2, 0], [0, 0, 0]]
        refused(es.EASYSPEC_ESTATE, es.easyspec_truncate, g.ctx, 0, 3)
        es.easyspec_truncate(g.ctx, 0, 4)
        es.easyspec_truncate(g.ctx, 0, 0)
        assert list(es.easyspec_get_evicted(g.ctx, 3)) == [0, 0, 0]
        g.calibrate({0: [1, 2, 3]})
        es.easyspec_truncate(g.ctx, 0, 1)
    finally:
        g.close()


def test_import_forgets_and_truncation_follows(gpu):
    """Imported slots have no weight; a sequence cut back takes up at the position that it was cut to."""
    g, d = model(gpu, "tiny", 35, track=200, max_batch=1, max_ctx=96)
    es = gpu.es
    try:
        bounds = list(range(g.cfg["n_layers"] + 1))
        rng = np.random.default_rng(7)
        for _ in range(3):
            t = list(rng.integers(0, g.cfg["vocab"], 16))
            g.calibrate({0: t}), d.calibrate(t)
        evict(gpu, g, {0: d}, {0: 30}, 10)
        es.easyspec_truncate(g.ctx, 0, 25)
        d.thin([[np.arange(25)] * g.cfg["n_kv_heads"]] * g.cfg["n_layers"])
        d.pos -= 5
        _, lg = g.draft_step({0: 4})
        gpu.assert_close(lg[0], d.draft(4, bounds), tol(g.cfg), "after truncation")
        k, v = g.export_kv(0, 25)
        g.import_kv(0, k, v)
        assert np.all(weights_of(gpu, g, 0, 25) == 0.0) and list(es.easyspec_get_evicted(g.ctx, 1)) == [0]
        d.drop_fuzzy()
        d.pos = 25                                       # an imported cache starts at position 0
        d.weight = [[np.zeros(25) for _ in layer] for layer in d.weight]
        _, lg = g.calibrate({0: [3, 1, 2]})
        gpu.assert_close(lg[0], d.calibrate([3, 1, 2]), tol(g.cfg), "after import")
        assert_weights(gpu, g, 0, d)
    finally:
        g.close()


@pytest.mark.parametrize("name,over", [("tiny", {}), ("tiny_qwen", {})])
def test_prompt_eviction_beams_and_calibration(gpu, route, name, over):
    """A run of all of them, as a program makes it, without a look at the host between draft step, selection and reordering."""
    import torch
    W, steps = 4, 4
    g, d = model(gpu, name, 36, track=256, max_batch=5, max_ctx=96, **over)
    es = gpu.es
    try:
        cfg, V, dev = g.cfg, g.cfg["vocab"], g.dev
        bounds = es.easyspec_default_groups(cfg["n_layers"], 2, es.EASYSPEC_POLICY_PACKED)
        g.set_groups(bounds)
        prompt = synth.make_tokens(77, 60, V)
        for i in range(0, 60, 16):
            _, lg = g.calibrate({1: list(prompt[i: i + 16])})
            want = d.calibrate(list(prompt[i: i + 16]))
        gpu.assert_close(lg[1], want, tol(cfg), "prompt")
        evict(gpu, g, {1: d}, {1: 33}, 12)
        es.easyspec_beam_fork(g.ctx, 1, 1, W)            # sequences 1 .. 4; 0 stays idle
        assert list(g.lens()[0]) == [0, 33, 33, 33, 33]
        first = torch.from_numpy(want[-1].astype(np.float32)).to(dev)
        logits = torch.zeros(5, V, device=dev)
        logits[1:] = first
        scores = torch.full((1, W), -float("inf"), device=dev)
        scores[0, 0] = 0.0
        tok = torch.zeros(steps, 5, dtype=torch.int32, device=dev)
        par = torch.zeros(steps, W, dtype=torch.int32, device=dev)
        kept_scores = torch.zeros(steps, W, device=dev)
        seen = torch.zeros(steps, W, V, device=dev)
        nxt = torch.zeros(5, dtype=torch.int32, device=dev)
        ws = torch.zeros(es.easyspec_beam_select_workspace_bytes(1, W, V, W) // 8 + 1, dtype=torch.float64, device=dev)
        st = torch.cuda.current_stream().cuda_stream
        torch.cuda.synchronize()
        for s in range(steps):
            seen[s].copy_(logits[1:])
            es.easyspec_beam_select(logits[1:], scores, None, 1, W, V, W, 1.0, 0, tok[s, 1:], par[s], scores, ws, st)
            kept_scores[s].copy_(scores[0])
            if s + 1 < steps:
                es.easyspec_beam_reorder(g.ctx, 1, W, par[s], 33)
                es.easyspec_draft_step(g.ctx, tok[s], nxt, logits)
        torch.cuda.synchronize()
        # every selection is the best of the logits it saw, and these are those of copies of the decoder that follow it
        beams, before, picks = [d.clone() for _ in range(W)], np.array([0.0] + [-np.inf] * 3, np.float32), []
        for s in range(steps):
            lg = seen[s].cpu().numpy()
            gpu.assert_close(lg, want[-1][None].repeat(W, 0) if s == 0 else np.array([x.draft(int(t), bounds) for x, t in zip(beams, picks[-1][0])]),
                             tol(cfg), "logits of the beams")
            t, p, sc = ref.beam_select(lg, before, None, W, 1.0, 0)
            assert np.array_equal(tok[s, 1:].cpu().numpy(), t) and np.array_equal(par[s].cpu().numpy(), p), s
            before = kept_scores[s].cpu().numpy()
            assert np.all(np.abs(before - sc) <= np.abs(sc) * 2.0 ** -24 * 1.001 + 1e-11)
            beams = [beams[j].clone() for j in p]
            picks.append((t, p))
        # the best line is accepted, and the other beams with it: calibrate one, fork the rest
        line, at = [], 0
        for s in reversed(range(steps)):
            line.append(int(picks[s][0][at]))
            at = int(picks[s][1][at])
        line.reverse()
        _, lg = g.calibrate({1: line})
        gpu.assert_close(lg[1], d.calibrate(line), tol(cfg), "calibration after beams")
        assert_weights(gpu, g, 1, d)
        es.easyspec_beam_fork(g.ctx, 1, 2, 3)
        _, lg = g.draft_step({1: 3, 2: 3, 3: 3, 4: 9})
        a, b = d.clone(), d.clone()
        x, y = a.draft(3, bounds), b.draft(9, bounds)
        for i in (1, 2, 3):
            gpu.assert_close(lg[i], x, tol(cfg), "forked")
        gpu.assert_close(lg[4], y, tol(cfg), "forked")
    finally:
        g.close()


def test_reorder_moves_drafted_slots_of_one_group_alone(gpu):
    import torch
    es = gpu.es
    g, _ = model(gpu, "tiny", 37, track=64, max_batch=6, max_ctx=64)
    try:
        g.calibrate({b: [b + 1, 2, 3, 4 * b, 9] for b in range(6)})
        for s in range(3):
            g.draft_step({b: 17 * b + s for b in range(6)})
        was = {b: g.export_kv(b, 8) for b in range(6)}
        ws = {b: weights_of(gpu, g, b, 5) for b in range(6)}
        es.easyspec_beam_reorder(g.ctx, 1, 4, torch.tensor([3, -1, 0, 0], dtype=torch.int32, device="cuda"), 3)
        torch.cuda.synchronize()
        for b, src in enumerate([0, 4, 2, 1, 1, 5]):
            for got, own, other in zip(g.export_kv(b, 8), was[b], was[src]):
                assert np.array_equal(got[:, :, :3], own[:, :, :3]) and np.array_equal(got[:, :, 3:], other[:, :, 3:]), b
            w = weights_of(gpu, g, b, 5)
            assert np.array_equal(w[:, :, :3], ws[b][:, :, :3]) and np.array_equal(w[:, :, 3:], ws[src][:, :, 3:]), b
    finally:
        g.close()


@pytest.mark.parametrize("name,over", SHAPES)
def test_weights_take_nothing_from_workspaces(gpu, name, over):
    """The same calibrations with every workspace filled with NaNs in front of each: the same bits."""
    def run(poison):
        g, _ = model(gpu, name, 36, track=400, max_batch=3, max_ctx=400, **over)
        try:
            rng = np.random.default_rng(9)
            for sizes in ((16, 16, 16),) * 20 + ((6, 1, 0), (0, 16, 3), (1, 1, 1)):
                if poison:
                    gpu.es.easyspec_poison_workspaces(g.ctx)
                g.calibrate({b: list(rng.integers(0, g.cfg["vocab"], n)) for b, n in enumerate(sizes) if n})
            return [weights_of(gpu, g, b, 320) for b in range(3)]
        finally:
            g.close()
    for a, b in zip(run(False), run(True)):
        assert np.array_equal(a, b) and np.all(np.isfinite(a))
