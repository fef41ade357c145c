"""What the operators on beams and on bounded caches are measured on: the calls a drafting program makes of them, at the
sizes it makes them, and the same results in plain torch operations.

A case is one of
  beam     selection over beams and vocabulary (easyspec_beam_select): the `select` best continuations of every group
  reorder  the beams' caches put in the order of the chosen parents (easyspec_kv_reorder)
  weigh    the attention weight that the cached slots receive from new tokens, added up (easyspec_attn_weights)
  evict    the lightest slots dropped from the caches of a model, the rest moved together (easyspec_kv_evict)
Head counts, head sizes, layers and vocabularies are those of the repository's model shapes.  Caches hold N(0, 1) values,
accumulated weights are spread over orders of magnitude, and some slots have none at all.
"""
import math

import numpy as np
import torch

own = False  # True: the framework's operators instead of the plain forms

DEV = "cuda:0"

#        layers, query heads, KV heads, head size, vocabulary, type
MODELS = {
    "tiny": (4, 4, 2, 64, 1024, "fp32"),
    "tiny_qwen": (5, 7, 1, 64, 1000, "fp32"),
    "llama3_8b": (32, 32, 8, 128, 128256, "bf16"),
    "qwen2_7b": (28, 28, 4, 128, 152064, "bf16"),
}


# ----------------------------------------------------------------------------------------------------------------
# the cases
# ----------------------------------------------------------------------------------------------------------------

def _beam(groups, beams, vocab, select, temperature=1.0, live=0, ended=0):
    return dict(kind="beam", groups=groups, beams=beams, vocab=vocab, select=select, temperature=temperature,
                live=live or beams, ended=ended)


def _cache(kind, model, layers=0, dtype=None, **more):
    n_layers, hq, hkv, hd, _, t = MODELS[model]
    c = dict(kind=kind, layers=layers or n_layers, q_heads=hq, kv_heads=hkv, head_dim=hd, dtype=dtype or t)
    for name, value in more.items():
        c[name] = ",".join(str(x) for x in value) if isinstance(value, list) else value
    return c


def _ints(text):
    return [int(n) for n in str(text).split(",")]


def listed():
    return [
        # the smallest drafter's beams: launches and latency
        dict(_beam(1, 4, 1000, 4), name="beam_tiny"),
        # one level of a wide token tree of the 8B drafter: sixteen nodes, the sixteen best children
        dict(_beam(1, 16, 128256, 16), name="beam_8b_level"),
        # sixteen users, four beams each, eight continuations looked at, at the paper's second temperature; one beam has ended
        dict(_beam(16, 4, 152064, 8, temperature=0.8, ended=1), name="beam_7b_users"),
        # after a drafted run: only the five drafted slots of eight beams differ
        dict(_cache("reorder", "llama3_8b", beams=4, seqs=8, slots=320, first=300, last=305, survivors=2), name="reorder_drafted"),
        # beams that share no prefix: whole caches move
        dict(_cache("reorder", "llama3_8b", beams=4, seqs=4, slots=2048, first=0, last=2048, survivors=3), name="reorder_whole"),
        # one new token of the smallest drafter in a short context
        dict(_cache("weigh", "tiny", layers=1, tokens=[1], lens=[128], slots=256), name="weigh_tiny_1"),
        # the calibration of one bonus token after a 2048-token context, one layer
        dict(_cache("weigh", "llama3_8b", layers=1, tokens=[1], lens=[2048], slots=2112), name="weigh_8b_1"),
        # a calibration of four users at long contexts, one layer
        dict(_cache("weigh", "llama3_8b", layers=1, tokens=[6, 6, 6, 6], lens=[4096, 8192, 16384, 32768], slots=32832),
             name="weigh_8b_batch4_long"),
        # sixteen users prefill a full chunk each, seven query heads per KV head, one layer
        dict(_cache("weigh", "qwen2_7b", layers=1, tokens=[16] * 16, lens=[512 + 37 * i for i in range(16)], slots=1152),
             name="weigh_7b_16x16"),
        # the smallest drafter's cache thinned
        dict(_cache("evict", "tiny_qwen", lens=[61], keep=[24], recent=8, slots=125, slots_out=32), name="evict_tiny"),
        # half of a 2048-token context of the 8B drafter dropped
        dict(_cache("evict", "llama3_8b", lens=[2048], keep=[1024], recent=128, slots=2112, slots_out=1024), name="evict_8b"),
        # four long contexts brought down to 4096 slots or less, a quarter of the layers
        dict(_cache("evict", "llama3_8b", layers=8, lens=[4096, 8192, 16384, 32768], keep=[2048, 4096, 4096, 4096], recent=512,
                    slots=32832, slots_out=4160), name="evict_8b_batch4_long"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["beam", "reorder", "weigh", "weigh", "evict"])
    if kind == "beam":
        beams = _log_int(rng, 1, 16)
        vocab = _log_int(rng, 500, 152064)
        groups = _log_int(rng, 1, max(1, min(16, 9_700_000 // (beams * vocab))))
        return _beam(groups, beams, vocab, rng.choice([1, beams, min(64, 2 * beams), _log_int(rng, 1, 64)]),
                     temperature=round(rng.uniform(0.5, 1.3), 2), live=rng.choice([1, beams, beams, rng.randint(1, beams)]),
                     ended=rng.choice([0, 0, min(1, beams - 1)]))
    heads = rng.choice([(4, 2, 64), (7, 1, 64), (32, 8, 128), (32, 8, 128), (28, 4, 128), (8, 8, 64), (8, 1, 128)])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    c = dict(kind=kind, q_heads=heads[0], kv_heads=heads[1], head_dim=heads[2], dtype=dtype)
    if kind == "reorder":
        beams = rng.choice([2, 3, 4, 5, 8, 16])
        seqs = beams * rng.randint(1, 16 // beams)
        slots = _log_int(rng, 20, 1500)
        layers = max(1, min(rng.randint(2, 32), 500_000 // (seqs * heads[1] * slots)))
        first = rng.choice([0, rng.randint(0, slots - 1), max(0, slots - rng.randint(1, 16))])
        c.update(layers=layers, beams=beams, seqs=seqs, slots=slots, first=first, last=rng.randint(first + 1, slots),
                 survivors=rng.randint(1, beams))
        return c
    batch = rng.choice([1, 1, 2, 3, 4, 7, 16])
    lens = [_log_int(rng, 24, 24000 // batch) for _ in range(batch)]
    if kind == "weigh":
        t = rng.randint(1, 16)
        c.update(layers=rng.choice([1, 1, 2]), tokens=",".join(str(rng.randint(1, t)) for _ in lens))
        c.update(lens=",".join(map(str, lens)), slots=max(lens) + rng.randint(0, 70))
        return c
    keep = [max(8, int(n * rng.uniform(0.1, 1.1))) for n in lens]
    layers = max(1, min(rng.randint(2, 32), 1_000_000 // (sum(lens) * heads[1])))
    c.update(layers=layers, lens=",".join(map(str, lens)), keep=",".join(map(str, keep)), recent=rng.randint(1, min(keep)),
             slots=max(lens) + rng.randint(0, 70), slots_out=max(keep) + rng.randint(0, 70))
    return c


# ----------------------------------------------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------------------------------------------

def _gen(seed, salt):
    return torch.Generator(device=DEV).manual_seed(1000003 * int(seed) + salt)


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _normal(gen, *shape, std=1.0, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=gen)


def _weights(gen, middle, *shape):
    """Accumulated weights: a few heavy slots, many light ones (half of them below `middle`), one in sixteen without any."""
    w = torch.exp(_normal(gen, *shape, std=2.0)) * middle
    return torch.where(torch.rand(shape, device=DEV, generator=gen) < 0.0625, torch.zeros((), device=DEV), w)


def prepare(case, seed):
    kind, st = case["kind"], dict(case=case)
    if kind == "beam":
        G, W, V, K = case["groups"], case["beams"], case["vocab"], case["select"]
        scores = -torch.rand(G, W, device=DEV, generator=_gen(seed, 2)) * 6.0
        ended = torch.zeros(G, W, dtype=torch.int32, device=DEV)
        scores[:, case["live"]:] = -math.inf                     # beams not in use yet
        ended[:, W - case["ended"]:] = 1
        st.update(logits=_normal(_gen(seed, 1), G, W, V, std=2.0), scores=scores, ended=ended, end_token=V // 2,
                  out=(torch.zeros(G, K, dtype=torch.int32, device=DEV), torch.zeros(G, K, dtype=torch.int32, device=DEV),
                       torch.zeros(G, K, device=DEV)))
        return st
    L, H, D = case["layers"], case["kv_heads"], case["head_dim"]
    if kind == "reorder":
        B, W = case["seqs"], case["beams"]
        shape = (L, B, H, case["slots"], D)
        st.update({n: _normal(_gen(seed, 10 + i), *shape, dtype=_type(case)) for i, n in enumerate(("k", "v"))})
        st.update(k_out=st["k"].clone(), v_out=st["v"].clone())  # the caches that the next step works on, up to date but for these slots
        chosen = torch.rand(B // W, W, device=DEV, generator=_gen(seed, 12)).argsort(-1)[:, : case["survivors"]]
        more = torch.randint(0, case["survivors"], (B // W, W), device=DEV, generator=_gen(seed, 13))
        more[:, : case["survivors"]] = torch.arange(case["survivors"], device=DEV)
        st["parents"] = chosen.gather(1, more).reshape(B).to(torch.int32).contiguous()
        return st
    lens = _ints(case["lens"])
    B, S = len(lens), case["slots"]
    st.update(lens=np.array(lens, np.int32), lens_dev=torch.tensor(lens, device=DEV),
              k=_normal(_gen(seed, 20), L, B, H, S, D, dtype=_type(case)),
              weights=_weights(_gen(seed, 22), case["q_heads"] / H / max(lens), L, B, H, S))  # a few calibrations' worth
    if kind == "weigh":
        n = _ints(case["tokens"])
        st.update(tokens=np.array(n, np.int32), tokens_dev=torch.tensor(n, device=DEV),
                  token_seq=torch.tensor([b for b in range(B) for _ in range(n[b])], device=DEV),
                  token_row=torch.tensor([t for b in range(B) for t in range(n[b])], device=DEV),
                  q=_normal(_gen(seed, 21), L, sum(n), case["q_heads"], D, std=1.5),
                  weights_out=torch.zeros(L, B, H, S, device=DEV))
        return st
    keep, So = _ints(case["keep"]), case["slots_out"]
    st.update(keep=np.array(keep, np.int32), keep_dev=torch.tensor(keep, device=DEV),
              v=_normal(_gen(seed, 23), L, B, H, S, D, dtype=_type(case)))
    st.update(out=(torch.zeros(L, B, H, So, D, dtype=_type(case), device=DEV), torch.zeros(L, B, H, So, D, dtype=_type(case), device=DEV),
                   torch.zeros(L, B, H, So, device=DEV), torch.zeros(L, B, H, So, dtype=torch.int32, device=DEV)))
    return st


# ----------------------------------------------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------------------------------------------

def run(st):
    return {"beam": _run_beam, "reorder": _run_reorder, "weigh": _run_weigh, "evict": _run_evict}[st["case"]["kind"]](st)


def _workspace(st, n_bytes):
    """The workspace that a program keeps from its first call on."""
    if "ws" not in st:
        st["ws"] = torch.empty((n_bytes + 15) // 8, dtype=torch.float64, device=DEV)
    return st["ws"]


def _run_beam(st):
    case = st["case"]
    G, W, V, K, T = case["groups"], case["beams"], case["vocab"], case["select"], case["temperature"]
    if own:
        import paper_2502_02493_amd as es
        ws = _workspace(st, 0 if "ws" in st else es.easyspec_beam_select_workspace_bytes(G, W, V, K))
        tokens, parents, scores = st["out"]
        es.easyspec_beam_select(st["logits"], st["scores"], st["ended"], G, W, V, K, T, st["end_token"], tokens, parents, scores, ws,
                                torch.cuda.current_stream().cuda_stream)
        return dict(tokens=tokens, parents=parents, scores=scores)
    # in 64 bits: candidates of different beams are compared, and the sums run over a vocabulary
    z = st["logits"].double()
    z = (z - z.amax(-1, keepdim=True)) / T
    z = z - torch.log(torch.exp(z).sum(-1, keepdim=True))
    start = st["scores"].double().unsqueeze(-1)
    only_end = torch.where(torch.arange(V, device=DEV) == st["end_token"], start, -math.inf)
    z = torch.where((st["ended"] != 0).unsqueeze(-1), only_end, start + z).reshape(G, W * V)
    # a stable sort: of equal scores the lowest beam and token comes first
    best, at = torch.sort(z, dim=-1, descending=True, stable=True)
    if W * V < K:
        best, at = (torch.nn.functional.pad(x, (0, K - W * V), value=f) for x, f in ((best, -math.inf), (at, 0)))
    best, at = best[:, :K], at[:, :K]
    none = best == -math.inf
    return dict(tokens=torch.where(none, -1, at % V).to(torch.int32), parents=torch.where(none, -1, at // V).to(torch.int32),
                scores=best.float())


def _run_reorder(st):
    case = st["case"]
    B, W, first, last = case["seqs"], case["beams"], case["first"], case["last"]
    if own:
        import paper_2502_02493_amd as es
        layout = es.easyspec_kv_layout(case["layers"], B, case["kv_heads"], case["slots"], case["head_dim"],
                                       es.EASYSPEC_DTYPE_BF16 if case["dtype"] == "bf16" else es.EASYSPEC_DTYPE_F32)
        es.easyspec_kv_reorder(st["k"], st["v"], layout, st["parents"], W, first, last, st["k_out"], st["v_out"],
                               torch.cuda.current_stream().cuda_stream)
        return dict(k=st["k_out"], v=st["v_out"])
    src = torch.arange(B, device=DEV) // W * W + st["parents"]
    st["k_out"][:, :, :, first:last] = st["k"][:, src, :, first:last]
    st["v_out"][:, :, :, first:last] = st["v"][:, src, :, first:last]
    return dict(k=st["k_out"], v=st["v_out"])


def _run_weigh(st):
    case = st["case"]
    L, Hq, H, D, S = case["layers"], case["q_heads"], case["kv_heads"], case["head_dim"], case["slots"]
    B, G = len(st["lens"]), Hq // H
    if own:
        import paper_2502_02493_amd as es
        layout = es.easyspec_kv_layout(L, B, H, S, D, es.EASYSPEC_DTYPE_BF16 if case["dtype"] == "bf16" else es.EASYSPEC_DTYPE_F32)
        ws = _workspace(st, 0 if "ws" in st else es.easyspec_attn_weights_workspace_bytes(layout, st["tokens"], st["lens"], Hq))
        es.easyspec_attn_weights(st["q"], st["k"], layout, st["tokens"], st["lens"], Hq, st["weights"], st["weights_out"], ws,
                                 torch.cuda.current_stream().cuda_stream)
        return st["weights_out"]
    M = int(st["tokens"].max())
    q = torch.zeros(L, B, M, H, G, D, device=DEV)
    q[:, st["token_seq"], st["token_row"]] = st["q"].reshape(L, -1, H, G, D)
    q = q.permute(0, 1, 3, 2, 4, 5).reshape(L, B, H, M * G, D)
    s = torch.matmul(q, st["k"].float().transpose(-1, -2)) * (1.0 / math.sqrt(D))
    slot, row = torch.arange(S, device=DEV), torch.arange(M, device=DEV)
    old = (st["lens_dev"] - st["tokens_dev"])[:, None, None]
    seen = (slot <= old + row[:, None]) & (row[:, None] < st["tokens_dev"][:, None, None])   # [B, M, S]
    seen = seen.repeat_interleave(G, dim=1)[None, :, None]
    s = torch.where(seen, s, -math.inf)
    p = torch.where(seen, torch.exp(s - s.amax(-1, keepdim=True).clamp_min(-1e30)), 0.0)
    p = (p / p.sum(-1, keepdim=True).clamp_min(1e-30)).sum(-2)
    before = torch.where((slot < old[:, 0])[None, :, None], st["weights"], 0.0)   # the new tokens' slots start from nothing
    return torch.where((slot < st["lens_dev"][:, None])[None, :, None], before + p, 0.0)


def _run_evict(st):
    case = st["case"]
    L, H, D, S, So, R = case["layers"], case["kv_heads"], case["head_dim"], case["slots"], case["slots_out"], case["recent"]
    k_out, v_out, w_out, at_out = st["out"]
    if own:
        import paper_2502_02493_amd as es
        layout = es.easyspec_kv_layout(L, len(st["lens"]), H, S, D, es.EASYSPEC_DTYPE_BF16 if case["dtype"] == "bf16" else es.EASYSPEC_DTYPE_F32)
        es.easyspec_kv_evict(st["k"], st["v"], st["weights"], layout, st["lens"], st["keep"], R, So, k_out, v_out, w_out, at_out,
                             torch.cuda.current_stream().cuda_stream)
        return dict(k=k_out, v=v_out, weights=w_out, slots=at_out)
    n, keep = st["lens_dev"][:, None, None], st["keep_dev"][:, None, None]
    slot = torch.arange(S, device=DEV)
    key = torch.where(slot >= n, -1.0, torch.where(slot >= n - torch.clamp(keep, max=R), math.inf, st["weights"]))
    order = torch.sort(key, dim=-1, descending=True, stable=True)[1]     # of equal weights the lowest slot first
    left = torch.minimum(n, keep)
    kept = torch.where(slot < left, order, S)                           # [L, B, H, S]
    kept = torch.sort(kept, dim=-1)[0][..., :So]
    if So > S:
        kept = torch.nn.functional.pad(kept, (0, So - S), value=S)
    there = kept < S
    kept = kept.clamp_max(S - 1)
    rows = kept.unsqueeze(-1).expand(-1, -1, -1, -1, D)
    return dict(k=torch.where(there.unsqueeze(-1), st["k"].gather(3, rows), k_out), v=torch.where(there.unsqueeze(-1), st["v"].gather(3, rows), v_out),
                weights=torch.where(there, st["weights"].gather(3, kept), w_out), slots=torch.where(there, kept.to(torch.int32), at_out))


# ----------------------------------------------------------------------------------------------------------------
# the work
# ----------------------------------------------------------------------------------------------------------------

def work(case):
    if case["kind"] == "beam":
        read = case["groups"] * max(1, min(case["live"], case["beams"] - case["ended"]))     # rows whose logits count
        return dict(bytes=4 * read * case["vocab"] + 12 * case["groups"] * case["select"], flops=4 * read * case["vocab"])
    H, D, L = case["kv_heads"], case["head_dim"], case["layers"]
    row = D * (2 if case["dtype"] == "bf16" else 4)
    if case["kind"] == "reorder":
        moved = 2 * L * H * (case["last"] - case["first"]) * row
        return dict(bytes=moved * (case["seqs"] + case["seqs"] // case["beams"] * case["survivors"]), flops=0)
    lens = _ints(case["lens"])
    if case["kind"] == "weigh":
        n = _ints(case["tokens"])
        seen = sum(n[b] * lens[b] - n[b] * (n[b] - 1) // 2 for b in range(len(n)))
        return dict(bytes=L * (H * sum(lens) * (row + 8) + 4 * sum(n) * case["q_heads"] * D), flops=2 * L * case["q_heads"] * D * seen)
    kept = sum(min(a, b) for a, b in zip(lens, _ints(case["keep"])))
    return dict(bytes=L * H * (4 * sum(lens) + kept * (4 * row + 8)), flops=L * H * sum(lens))


# ----------------------------------------------------------------------------------------------------------------
# the definition, in 64 bits
# ----------------------------------------------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "beam":
        return _exact_beam(st)
    if case["kind"] == "reorder":
        B, W, a, z = case["seqs"], case["beams"], case["first"], case["last"]
        parents = st["parents"].tolist()
        k, v = st["k"].clone(), st["v"].clone()
        for i in range(B):
            for to, src in ((k, st["k"]), (v, st["v"])):
                to[:, i, :, a:z] = src[:, i - i % W + parents[i], :, a:z]
        return dict(k=k, v=v)
    if case["kind"] == "weigh":
        return _exact_weigh(st)
    return _exact_evict(st)


def _exact_beam(st):
    case = st["case"]
    G, W, V, K, T = case["groups"], case["beams"], case["vocab"], case["select"], case["temperature"]
    cum, ended = st["scores"].double().cpu().numpy(), st["ended"].cpu().numpy()
    tokens, parents, scores = np.full((G, K), -1, np.int32), np.full((G, K), -1, np.int32), np.full((G, K), -np.inf)
    for g in range(G):
        found = []
        for w in range(W):
            if cum[g, w] == -np.inf:
                continue
            if ended[g, w]:
                found.append((-cum[g, w], w, st["end_token"]))
                continue
            x = st["logits"][g, w].cpu().numpy().astype(np.float64) / T
            top = x.max()
            norm = top + math.log(math.fsum(np.exp(x - top)))
            for v in np.argsort(-x, kind="stable")[:K]:
                found.append((-(cum[g, w] + x[v] - norm), w, int(v)))
        for i, (s, w, v) in enumerate(sorted(found)[:K]):
            tokens[g, i], parents[g, i], scores[g, i] = v, w, -s
    return dict(tokens=tokens, parents=parents, scores=scores)


def _exact_weigh(st):
    case = st["case"]
    Hq, H, D = case["q_heads"], case["kv_heads"], case["head_dim"]
    out = torch.zeros(st["weights"].shape, dtype=torch.float64, device=DEV)
    first = 0
    for b, (n, length) in enumerate(zip(st["tokens"].tolist(), st["lens"].tolist())):
        for layer in range(case["layers"]):
            keys = st["k"][layer, b, :, :length].double()
            out[layer, b, :, : length - n] = st["weights"][layer, b, :, : length - n].double()
            for t in range(n):
                seen = length - n + t + 1
                for j in range(Hq):
                    h = j // (Hq // H)
                    s = keys[h, :seen].mv(st["q"][layer, first + t, j].double()) / math.sqrt(D)
                    out[layer, b, h, :seen] += torch.softmax(s, 0)
        first += n
    return out


def _exact_evict(st):
    case = st["case"]
    k, v, w, at = (t.cpu().clone() for t in st["out"])
    heavy = st["weights"].cpu().numpy()
    for b, (n, keep) in enumerate(zip(st["lens"].tolist(), st["keep"].tolist())):
        recent = min(case["recent"], keep)
        for layer in range(case["layers"]):
            for h in range(case["kv_heads"]):
                if keep >= n:
                    kept = np.arange(n)
                else:
                    by_weight = np.argsort(-heavy[layer, b, h, : n - recent], kind="stable")[: keep - recent]
                    kept = np.concatenate([np.sort(by_weight), np.arange(n - recent, n)])
                at[layer, b, h, : len(kept)] = torch.from_numpy(kept.astype(np.int32))
                w[layer, b, h, : len(kept)] = torch.from_numpy(heavy[layer, b, h][kept])
                rows = torch.from_numpy(kept).to(DEV)
                k[layer, b, h, : len(kept)] = st["k"][layer, b, h].index_select(0, rows).cpu()
                v[layer, b, h, : len(kept)] = st["v"][layer, b, h].index_select(0, rows).cpu()
    return dict(k=k, v=v, weights=w, slots=at)
