"""Sampling under top-k, top-p and min-p (easyspec_sample) against the definition in 64 bits: equal tokens, equal kept logits."""
import math

import numpy as np
import pytest

import kvq_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def es():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device; none is visible")
    import paper_2502_02493_amd as es
    return es


def call(es, logits, u, T, top_k, top_p, min_p, filtered=True, in_place=False, on=None):
    """numpy logits [rows, V], u [rows] or None -> (tokens or None, kept or None)"""
    import torch
    R, V = logits.shape
    x = torch.from_numpy(logits).cuda()
    uu = None if u is None else torch.from_numpy(np.asarray(u, np.float32)).cuda()
    tokens = None if u is None else torch.full((R + 4,), -7, dtype=torch.int32, device="cuda")
    out = None if not filtered else x if in_place else torch.full((R * V + 64,), 5.0, device="cuda")
    need = es.easyspec_sample_workspace_bytes(R, V)
    ws = torch.full((need + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    es.easyspec_sample(x, uu, R, V, T, top_k, top_p, min_p, tokens, out, ws, (on or torch.cuda.current_stream()).cuda_stream)
    torch.cuda.synchronize()
    assert bool((ws[need:] == 0xA5).all())
    if tokens is not None:
        assert bool((tokens[R:] == -7).all())
    if filtered and not in_place:
        assert bool((out[R * V:] == 5).all())
        out = out[:R * V].reshape(R, V)
    if not in_place:
        assert np.array_equal(x.cpu().numpy(), logits, equal_nan=True)
    return None if tokens is None else tokens[:R].cpu().numpy(), None if out is None else out.cpu().numpy()


def check(es, logits, u, T, top_k, top_p, min_p, **more):
    tokens, left = call(es, logits, u, T, top_k, top_p, min_p, **more)
    for r in range(len(logits)):
        token, kept = ref.sample(logits[r], None if u is None else np.float32(u[r]), T, top_k, top_p, min_p)
        if tokens is not None:
            assert tokens[r] == token, (r, tokens[r], token)
        if left is not None:
            assert np.array_equal(left[r], kept), (r, np.argwhere(left[r] != kept)[:5].tolist(), int((left[r] > -np.inf).sum()), int((kept > -np.inf).sum()))
    return tokens, left


def normal(seed, R, V, std=2.0):
    g = np.random.default_rng(seed)
    return g.normal(0, std, (R, V)).astype(np.float32), g.random(R).astype(np.float32)


SETTINGS = [(1.0, 0, 1.0, 0.0), (0.8, 40, 1.0, 0.0), (0.8, 0, 0.9, 0.0), (1.3, 0, 1.0, 0.05), (0.7, 50, 0.95, 0.02), (0.3, 1, 0.5, 0.5), (1.5, 2000, 0.99, 0.0), (0.05, 20, 0.999, 0.0)]


@pytest.mark.parametrize("setting", SETTINGS)
@pytest.mark.parametrize("R,V", [(1, 1), (3, 2), (2, 63), (5, 64), (1, 1000), (4, 1025), (2, 4096), (3, 8191), (1, 20000), (2, 50257), (1, 128256), (3, 152064)])
def test_sizes_and_settings(es, R, V, setting):
    logits, u = normal(V + R, R, V)
    check(es, logits, u, *setting)


@pytest.mark.parametrize("V", [1000, 40000, 1 << 20])
@pytest.mark.parametrize("T", [0.01, 1.0, 30.0])
def test_flat_and_sharp(es, V, T):
    logits, u = normal(V, 1, V, std=4.0)
    for k, p, m in ((0, 0.7, 0.0), (300, 1.0, 0.0), (V // 2, 0.9, 0.0), (0, 1.0, 0.3)):
        check(es, logits, u, T, k, p, m)


def test_filter_alone_and_draw_alone(es):
    logits, u = normal(3, 5, 30001)
    for setting in SETTINGS:
        check(es, logits, None, *setting)
        check(es, logits, u, *setting, filtered=False)
        check(es, logits, u, *setting, in_place=True)


@pytest.mark.parametrize("V", [16, 5000, 70000])
def test_equal_logits(es, V):
    """All of them, and steps: of equal ones the lowest tokens stay."""
    u = np.array([0.0, 0.25, 0.5, 0.999], np.float32)
    flat = np.full((4, V), 1.5, np.float32)
    for k, p in ((0, 1.0), (7, 1.0), (0, 0.5), (10, 0.35), (0, 1.0 / 3)):
        tokens, left = call(es, flat, u, 1.0, k, p, 0.0)
        n = min(k or V, V)
        n = n if p == 1 else math.ceil(np.float32(p) * np.float64(n))
        assert (left[:, :n] == 1.5).all() and np.isneginf(left[:, n:]).all()
        assert tokens.tolist() == [min(n - 1, int(np.float64(x) * n)) for x in u]
    g = np.random.default_rng(V)
    steps = (g.integers(0, 40, (4, V)) / 8).astype(np.float32)
    for k, p, m in ((0, 0.8, 0.0), (V // 3, 1.0, 0.0), (0, 1.0, 0.1), (V // 2, 0.6, 0.05)):
        check(es, steps, u, 0.9, k, p, m)
    check(es, np.where(g.random((4, V)) < 0.5, np.float32(0.0), np.float32(-0.0)), u, 1.0, V // 3, 1.0, 0.0)      # the two zeros are one number


@pytest.mark.parametrize("V", [700, 6000, 90000])
def test_nearly_equal_logits_in_place(es, V):
    """More words near a border than are sorted, or in one bucket, where the logits are overwritten: every filter, alone and with the others."""
    g = np.random.default_rng(V)
    logits = np.empty((4, V), np.float32)
    logits[0] = 2.0 + g.integers(0, 3, V) * np.float32(2.0 ** -22)
    logits[1] = g.integers(0, 6, V) / 4
    logits[2] = np.where(g.random(V) < 0.7, np.float32(-1.0), np.float32(3.0))
    logits[3] = g.normal(0, 1e-6, V)
    logits[3, 5] = -1e30                                   # so that all others lie in the first bin
    u = np.array([0.3, 0.99, 0.02, 0.6], np.float32)
    for k, p, m in ((V // 3, 1.0, 0.0), (0, 0.6, 0.0), (0, 1.0, 0.4), (V // 2, 0.7, 0.0), (V // 2, 0.9, 0.3), (0, 0.95, 0.8), (0, 1.0, 0.0)):
        check(es, logits, u, 0.9, k, p, m, in_place=True)
        check(es, logits, u, 0.9, k, p, m, filtered=False)
    check(es, logits, None, 0.9, V // 2, 0.7, 0.3, in_place=True)


def test_words_that_are_none(es):
    V = 9000
    logits, u = normal(8, 8, V)
    g = np.random.default_rng(1)
    logits[0, g.random(V) < 0.9] = -np.inf
    logits[1, g.random(V) < 0.5] = np.nan
    logits[2] = -np.inf
    logits[3] = np.nan
    logits[4, 77] = np.inf
    logits[5] = -np.inf
    logits[5, 4321] = -3.0
    logits[6] = np.float32(-3.4e38)
    logits[6, 5] = np.float32(3.4e38)
    logits[7, :] = np.finfo(np.float32).min
    for setting in SETTINGS:
        tokens, left = check(es, logits, u, *setting)
        assert tokens[2] == tokens[3] == tokens[4] == -1 and tokens[5] == 4321
        assert np.isneginf(left[2:5]).all()


@pytest.mark.parametrize("V", [500, 60000])
def test_the_ends_of_u(es, V):
    logits, _ = normal(V, 6, V)
    logits[:] = logits[0]
    u = np.array([0.0, np.nextafter(np.float32(1), np.float32(0)), 1.0, 2.0, np.nan, -1.0], np.float32)
    for T, k, p, m in ((0.8, 30, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (1.0, 0, 1.0, 0.1)):
        tokens, left = call(es, logits, u, T, k, p, m)
        order = np.argsort(-logits[0], kind="stable")
        n = int((left[0] > -np.inf).sum())
        assert tokens[0] == tokens[5] == order[0] and tokens[2] == tokens[3] == tokens[4] == order[n - 1]
        assert tokens[1] in order[:n]


@pytest.mark.parametrize("V", [50, 20000])
def test_the_share_of_every_word(es, V):
    """u at the middles of 4096 equal parts: every word is drawn as often as its share says, to one."""
    n = 4096
    logits = np.broadcast_to(normal(2, 1, V)[0], (n, V)).copy()
    tokens, _ = call(es, logits, (np.arange(n) + 0.5) / n, 0.9, 30, 0.95, 0.01, filtered=False)
    kept = ref.sample(logits[0], None, 0.9, 30, 0.95, 0.01)[1].astype(np.float64)
    p = np.exp((kept - kept.max()) / np.float64(np.float32(0.9)))
    p /= p.sum()
    assert np.abs(np.bincount(tokens, minlength=V) - n * p).max() <= 1.0 + 1e-6


def test_min_p_of_one_and_top_p_of_nearly_nothing(es):
    logits, u = normal(4, 3, 12345)
    logits[0, [7, 9000]] = 11.0
    tokens, left = check(es, logits, u, 1.0, 0, 1.0, 1.0)
    assert (left[0] > -np.inf).sum() == 2 and (left[1] > -np.inf).sum() == 1
    _, left = check(es, logits, u, 1.0, 0, 1e-30, 0.0)
    assert ((left > -np.inf).sum(1) == 1).all() and left[0, 7] == 11.0


def test_many_rows(es):
    logits, u = normal(6, 300, 700)
    check(es, logits, u, 0.8, 40, 0.9, 0.01)
    logits, u = normal(7, 70, 30000)
    check(es, logits, u, 0.8, 0, 0.9, 0.0)


@pytest.mark.parametrize("R,V", [(2, 256), (2, 257), (2, 513), (3, 1025), (2, 2049), (2, 4096), (2, 4097), (3, 8192), (3, 8193), (300, 9001), (1024, 8200), (1025, 8200)])
def test_where_the_ways_of_cutting_rows_change(es, R, V):
    logits, u = normal(R + V, R, V)
    logits[-1] = np.round(logits[-1] * 2) / 2              # thousands of equal ones
    check(es, logits, u, 0.9, 0, 0.85, 0.0)
    check(es, logits, u, 0.8, 60, 0.95, 0.01)


def test_streams_and_graphs(es):
    """Captured calls with their own workspaces, replayed between eager ones: bits do not change."""
    import torch
    R, V = 3, 50000
    logits, u = normal(12, R, V)
    check(es, logits, u, 0.8, 40, 0.95, 0.0, on=torch.cuda.Stream())
    x, uu = torch.from_numpy(logits).cuda(), torch.from_numpy(u).cuda()
    graphs, tokens, outs, spaces = [], [], [], []
    settings = ((0.8, 40, 0.95, 0.0), (1.2, 0, 0.9, 0.01))
    torch.cuda.synchronize()
    for s in settings:
        tokens.append(torch.zeros(R, dtype=torch.int32, device="cuda"))
        outs.append(torch.zeros(R, V, device="cuda"))
        spaces.append(torch.empty(es.easyspec_sample_workspace_bytes(R, V) // 4 + 4, device="cuda"))
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            es.easyspec_sample(x, uu, R, V, *s, tokens[-1], outs[-1], spaces[-1], torch.cuda.current_stream().cuda_stream)
    for turn in range(4):
        x.normal_(0, 2)
        uu.uniform_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for s, t, o in zip(settings, tokens, outs):
            want, left = call(es, x.cpu().numpy(), uu.cpu().numpy(), *s)
            assert np.array_equal(t.cpu().numpy(), want) and np.array_equal(o.cpu().numpy(), left)
            for r in range(R):
                assert want[r] == ref.sample(x[r].cpu().numpy(), float(uu[r]), *s)[0]


def test_offsets_beyond_32_bits(es):
    """Logits of 4.3 GB: the last row, in place."""
    import torch
    R, V = 1030, 1 << 20
    x = torch.zeros(R, V, device="cuda")
    row, u = normal(1, 1, V)
    x[-1] = torch.from_numpy(row[0]).cuda()
    uu = torch.from_numpy(np.repeat(u, R)).cuda()
    tokens = torch.zeros(R, dtype=torch.int32, device="cuda")
    ws = torch.empty(es.easyspec_sample_workspace_bytes(R, V) // 4 + 4, device="cuda")
    es.easyspec_sample(x, uu, R, V, 0.8, 50, 0.9, 0.0, tokens, x, ws, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    token, kept = ref.sample(row[0], u[0], 0.8, 50, 0.9, 0.0)
    assert int(tokens[-1]) == token and np.array_equal(x[-1].cpu().numpy(), kept)
    n = math.ceil(50 * np.float64(np.float32(0.9)))          # of equal words the first 45 or 46
    assert (tokens[:-1] == int(np.float64(u[0]) * n)).all() and bool((x[:-1, :n] == 0).all()) and bool(torch.isneginf(x[:-1, n:]).all())
