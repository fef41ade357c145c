"""Selection over beams and vocabulary (easyspec_beam_select) against a 64-bit evaluation: tokens and parents equal, scores to half a
step of fp32 (2^-24 of the value; both sides form them in 64 bits)."""
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


def call(es, logits, scores, ended, n_select, T=1.0, end_token=0, stream=None, alias=False):
    import torch
    G, W, V = logits.shape
    dev = torch.device("cuda:0")
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)
    d_l, d_s = t(logits), t(scores)
    d_e = None if ended is None else t(ended.astype(np.int32))
    tok = torch.full((G, n_select), -7, dtype=torch.int32, device=dev)
    par = torch.full((G, n_select), -7, dtype=torch.int32, device=dev)
    out = d_s if alias else torch.full((G, n_select), 7.0, device=dev)
    ws = torch.full((es.easyspec_beam_select_workspace_bytes(G, W, V, n_select) // 8 + 1,), float("nan"), dtype=torch.float64, device=dev)
    torch.cuda.synchronize()
    handle = torch.cuda.current_stream().cuda_stream if stream is None else stream.cuda_stream
    es.easyspec_beam_select(d_l, d_s, d_e, G, W, V, n_select, T, end_token, tok, par, out, ws, handle)
    torch.cuda.synchronize()
    return tok.cpu().numpy(), par.cpu().numpy(), out.cpu().numpy()


def check(es, logits, scores, ended=None, n_select=4, T=1.0, end_token=0, **more):
    tok, par, out = call(es, logits, scores, ended, n_select, T, end_token, **more)
    for g in range(logits.shape[0]):
        w_tok, w_par, w_out = ref.beam_select(logits[g], scores[g], None if ended is None else ended[g], n_select, float(np.float32(T)), end_token)
        assert np.array_equal(tok[g], w_tok), (g, tok[g], w_tok)
        assert np.array_equal(par[g], w_par), (g, par[g], w_par)
        none = w_tok < 0
        assert np.all(out[g][none] == -np.inf)
        err = np.abs(out[g][~none] - w_out[~none])
        assert np.all(err <= np.abs(w_out[~none]) * 2.0 ** -24 * 1.001 + 1e-11), err.max()


def rows(seed, G, W, V, std=2.0):
    rng = np.random.default_rng(seed)
    return rng.normal(0, std, (G, W, V)).astype(np.float32), (-6 * rng.random((G, W))).astype(np.float32)


@pytest.mark.parametrize("G,W,V,K,T", [
    (1, 1, 1, 1, 1.0), (1, 1, 1, 3, 1.0), (1, 2, 1, 4, 0.7), (2, 1, 5, 2, 1.0), (1, 4, 1000, 4, 1.0), (3, 3, 63, 64, 1.3),
    (1, 7, 513, 7, 0.8), (2, 16, 4095, 16, 0.8), (1, 5, 4096, 5, 1.0), (1, 5, 4097, 33, 1.0), (1, 64, 300, 64, 1.0),
    (5, 9, 8193, 17, 0.5), (1, 16, 128256, 16, 1.0), (2, 3, 152064, 64, 0.8), (40, 4, 1031, 8, 1.0), (1, 1, 128256, 1, 1.0),
    (1, 2, 1048576, 8, 1.0),
])
def test_sizes(es, G, W, V, K, T):
    logits, scores = rows(G * 1000 + W + V, G, W, V)
    check(es, logits, scores, None, K, T)


@pytest.mark.parametrize("G,W,V", [(1025, 63, 17), (65535, 1, 40)])
def test_many_groups(es, G, W, V):
    logits, scores = rows(7, G, W, V)
    tok, par, out = call(es, logits, scores, None, 3)
    for g in list(range(0, G, 997)) + [G - 1]:
        w_tok, w_par, _ = ref.beam_select(logits[g], scores[g], None, 3, 1.0, 0)
        assert np.array_equal(tok[g], w_tok) and np.array_equal(par[g], w_par)


def test_dead_and_ended_beams(es):
    logits, scores = rows(3, 6, 5, 2000)
    ended = np.zeros((6, 5), np.int32)
    scores[0, 1:] = -np.inf                      # the first step of a search: one beam
    scores[1] = -np.inf                          # nothing at all
    scores[2, 2] = np.nan
    ended[3] = 1                                 # every beam has ended
    ended[4, 1] = 3
    scores[4, 1] = 0.0                           # the best of its group
    ended[5, 4], scores[5, 4] = 1, -np.inf       # ended, and dropped
    logits[0, 1:] = np.nan                       # what is not read may hold anything
    logits[3] = np.inf
    check(es, logits, scores, ended, 8, 0.8, 1999)


def test_equal_logits_and_equal_beams(es):
    logits, scores = rows(4, 1, 6, 9000)
    logits[0, 0] = 0.5                           # all equal: the lowest tokens
    logits[0, 1] = np.round(logits[0, 1])        # many equal ones
    logits[0, 3] = logits[0, 2]                  # two beams alike, with equal scores: the lower first, token by token
    scores[0, 3] = scores[0, 2]
    logits[0, 4] = np.where(np.arange(9000) % 2 == 0, np.float32(0.0), np.float32(-0.0))   # one logit, two signs
    for k in (1, 5, 64):
        check(es, logits, scores, None, k)
    same = np.zeros((2, 16, 5000), np.float32)
    check(es, same, np.zeros((2, 16), np.float32), None, 64)


def test_masked_logits(es):
    logits, scores = rows(5, 8, 3, 12345)
    logits[0, :, 100:] = -np.inf                 # a few allowed tokens, of which too few for n_select
    logits[0, :, 7:] = -np.inf
    logits[1, 0] = -np.inf                       # a beam with none
    logits[2] = -np.inf                          # a group with none
    logits[3, 1, 17] = np.nan
    logits[4, 2, 4000] = np.inf                  # no distribution: the beam offers nothing
    logits[5] = np.float32(-3.4028235e38)        # a mask of the type's lowest value
    logits[5, :, 50:53] = 1.0
    logits[6] = np.where((np.arange(12345) % 512) < 480, logits[6], -np.inf)
    logits[7] = np.where((np.arange(12345) % 4096) < 40, logits[7], -np.inf)
    for k in (3, 40):
        check(es, logits, scores, None, k)


def test_sorted_vocabularies(es):
    V = 20000
    up = np.linspace(-5, 5, V, dtype=np.float32)
    logits = np.stack([np.stack([up, up[::-1]]), np.stack([np.roll(up, 777), -np.abs(up)])]).copy()
    check(es, logits, np.array([[-1.0, -1.25], [-3.0, -0.5]], np.float32), None, 64)


@pytest.mark.parametrize("scale", [1e-30, 1e4, 3e38])
def test_range_of_logits(es, scale):
    rng = np.random.default_rng(9)
    logits = (rng.random((1, 3, 3001)) * 2 - 1).astype(np.float32) * np.float32(scale)
    scores = np.array([[-1.0, -2.0, -4.0]], np.float32)
    check(es, logits, scores, None, 10, 0.5)


def test_scores_out_may_be_scores_other_stream_and_graph(es):
    import torch
    logits, scores = rows(11, 2, 8, 30001)
    check(es, logits, scores.copy(), None, 8, alias=True)
    check(es, logits, scores, None, 8, stream=torch.cuda.Stream())
    dev = torch.device("cuda:0")
    G, W, V, K = 2, 8, 30001, 8
    d_l, d_s = torch.from_numpy(logits).to(dev), torch.from_numpy(scores).to(dev)
    tok, par = (torch.zeros(G, K, dtype=torch.int32, device=dev) for _ in range(2))
    out = torch.zeros(G, K, device=dev)
    ws = torch.zeros(es.easyspec_beam_select_workspace_bytes(G, W, V, K) // 8 + 1, dtype=torch.float64, device=dev)
    run = lambda: es.easyspec_beam_select(d_l, d_s, None, G, W, V, K, 1.0, 0, tok, par, out, ws, torch.cuda.current_stream().cuda_stream)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for seed in range(3):
        fresh, s = rows(100 + seed, G, W, V)
        d_l.copy_(torch.from_numpy(fresh))
        d_s.copy_(torch.from_numpy(s))
        graph.replay()
        torch.cuda.synchronize()
        for g in range(G):
            w_tok, w_par, _ = ref.beam_select(fresh[g], s[g], None, K, 1.0, 0)
            assert np.array_equal(tok[g].cpu().numpy(), w_tok) and np.array_equal(par[g].cpu().numpy(), w_par)


@pytest.mark.parametrize("live,K", [(1, 64), (1, 16), (3, 64), (16, 1)])
def test_few_live_beams_of_many(es, live, K):
    """The first step of a search, and a level of few nodes in rows for sixteen; whatever the dead rows hold."""
    logits, scores = rows(live * K, 2, 16, 40000)
    scores[:, live:] = -np.inf
    scores[1] = np.roll(scores[1], 5)
    logits[scores == -np.inf] = np.nan
    check(es, logits, scores, None, K)


def test_more_lists_than_threads(es):
    logits, scores = rows(21, 1, 64, 80000)
    check(es, logits, scores, None, 64)
    logits[0, :, ::7] = 9.0                      # thousands of equal logits, in equal beams
    logits[0, 1:] = logits[0, :1]
    check(es, logits, np.zeros((1, 64), np.float32), None, 64)


def test_stays_inside_its_workspace_and_outputs(es):
    import torch
    dev = torch.device("cuda:0")
    for G, W, V, K in ((1, 4, 1000, 4), (3, 5, 9001, 64), (2, 16, 30000, 16)):
        logits, scores = rows(G + V, G, W, V)
        n = es.easyspec_beam_select_workspace_bytes(G, W, V, K)
        ws = torch.full((n + 4096,), 0xA5, dtype=torch.uint8, device=dev)
        out = [torch.full((G * K + 64,), 77, dtype=t, device=dev) for t in (torch.int32, torch.int32, torch.float32)]
        es.easyspec_beam_select(torch.from_numpy(logits).to(dev), torch.from_numpy(scores).to(dev), None, G, W, V, K, 1.0, 0, *out, ws,
                                torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert bool((ws[n:] == 0xA5).all()) and all(bool((o[G * K:] == 77).all()) for o in out)
        for g in range(G):
            assert np.array_equal(out[0][g * K: g * K + K].cpu().numpy(), ref.beam_select(logits[g], scores[g], None, K, 1.0, 0)[0])


def test_offsets_beyond_32_bits(es):
    """More than 2^31 logits: two beams of the last group alone are live, the others' logits and lists are not read."""
    import torch
    dev = torch.device("cuda:0")
    G, W, V, K = 33, 64, 1 << 20, 64
    logits, scores = rows(22, 1, 2, V)
    d_l = torch.full((G, W, V), float("nan"), device=dev)
    assert d_l.numel() > 1 << 31
    d_s = torch.full((G, W), -float("inf"), device=dev)
    d_l[-1, 62:], d_s[-1, 62:] = torch.from_numpy(logits[0]).to(dev), torch.from_numpy(scores[0]).to(dev)
    n = es.easyspec_beam_select_workspace_bytes(G, W, V, K)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=dev)
    tok, par = (torch.full((G, K), -7, dtype=torch.int32, device=dev) for _ in range(2))
    out = torch.full((G, K), 7.0, device=dev)
    torch.cuda.synchronize()
    es.easyspec_beam_select(d_l, d_s, None, G, W, V, K, 1.0, 0, tok, par, out, ws, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    w_tok, w_par, w_out = ref.beam_select(logits[0], scores[0], None, K, 1.0, 0)
    assert np.array_equal(tok[-1].cpu().numpy(), w_tok) and np.array_equal(par[-1].cpu().numpy(), w_par + 62)
    assert np.all(np.abs(out[-1].cpu().numpy() - w_out) <= np.abs(w_out) * 2.0 ** -24 * 1.001 + 1e-11)
    assert torch.all(tok[:-1] == -1) and torch.all(par[:-1] == -1) and torch.all(out[:-1] == -float("inf"))


def test_two_calls_at_once(es):
    """Two streams, each with its own workspace: the same results as one after the other."""
    import torch
    dev = torch.device("cuda:0")
    sets = []
    for seed, (G, W, V, K) in ((23, (1, 16, 128256, 16)), (24, (7, 5, 50000, 9))):
        logits, scores = rows(seed, G, W, V)
        t = [torch.from_numpy(x).to(dev) for x in (logits, scores)]
        outs = [[torch.zeros((G, K), dtype=d, device=dev) for d in (torch.int32, torch.int32, torch.float32)] for _ in range(2)]
        ws = torch.zeros(es.easyspec_beam_select_workspace_bytes(G, W, V, K), dtype=torch.uint8, device=dev)
        sets.append((t, outs, ws, (G, W, V, K), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for (l, s), outs, ws, size, _ in sets:
        es.easyspec_beam_select(l, s, None, *size, 0.9, 0, *outs[0], ws, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for _ in range(50):
        for (l, s), outs, ws, size, st in sets:
            es.easyspec_beam_select(l, s, None, *size, 0.9, 0, *outs[1], ws, st.cuda_stream)
    torch.cuda.synchronize()
    for _, (a, b), _, _, _ in sets:
        assert all(torch.equal(x, y) for x, y in zip(a, b))
