"""What the operators of drafting by sampling over long contexts are measured on: the calls a drafting program makes of them, at the
sizes it makes them, and the same results in plain torch operations.

A case is one of
  hold    slots of K and V brought into a cache held in 4 bits and read back as the values they stand for (easyspec_kvq_store, _load)
  attend  attention of new tokens over a whole cache held in 4 bits (easyspec_kvq_attention)
  sparse  the blocks of such a cache that matter to a token selected, and attention over these (easyspec_kvq_select, _attention)
  sample  logits filtered by top-k, top-p and min-p and a token drawn from what stays (easyspec_sample)
Head counts, head sizes, layers and vocabularies are those of the repository's model shapes.

A cache in 4 bits: codes, uint8 [layer][sequence][KV head][slot][head size / 2], channel 2 i in the low half of byte i: a sign and one of
0, 0.5, 1, 1.5, 2, 3, 4, 6; scales, uint8 [..][slot][head size / 32]: 2^(scale - 127) for 32 channels; bounds, bf16
[..][blocks of 64 slots][2][head size]: every channel's lowest and highest key of the block.
"""
import math

import numpy as np
import torch

own = False  # True: the framework's operators instead of the plain forms

DEV = "cuda:0"
BLOCK = 64

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

def _cache(kind, model, layers=0, **more):
    n_layers, hq, hkv, hd, _, t = MODELS[model]
    c = dict(kind=kind, layers=layers or n_layers, q_heads=hq, kv_heads=hkv, head_dim=hd, dtype=t)
    for name, value in more.items():
        c[name] = ",".join(str(x) for x in value) if isinstance(value, list) else value
    return c


def _sample(rows, vocab, temperature, top_k=0, top_p=1.0, min_p=0.0, draw=True, filtered=True):
    return dict(kind="sample", rows=rows, vocab=vocab, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p, draw=draw,
                filtered=filtered)


def _ints(text):
    return [int(n) for n in str(text).split(",")]


def listed():
    return [
        # one drafted token of sixteen users enters a layer's cache: launches and latency
        dict(_cache("hold", "llama3_8b", layers=1, new=[1] * 16, to=[400 + 97 * i for i in range(16)], slots=2048), name="hold_8b_append"),
        # a calibrated prompt of 2048 tokens, all layers, goes over into 4 bits
        dict(_cache("hold", "llama3_8b", new=[2048], to=[0], slots=2112), name="hold_8b_prompt"),
        # one new token of the smallest drafter in a short context
        dict(_cache("attend", "tiny", layers=1, tokens=[1], lens=[128], slots=256), name="attend_tiny_1"),
        # a drafted token after a 2048-token context, one layer
        dict(_cache("attend", "llama3_8b", layers=1, tokens=[1], lens=[2048], slots=2112), name="attend_8b_1"),
        # four users at long contexts, five drafted tokens and the bonus token of each, one layer
        dict(_cache("attend", "llama3_8b", layers=1, tokens=[6, 6, 6, 6], lens=[4096, 8192, 16384, 32768], slots=32832),
             name="attend_8b_batch4_long"),
        # sixteen users prefill a full chunk each, seven query heads per KV head, one layer
        dict(_cache("attend", "qwen2_7b", layers=1, tokens=[16] * 16, lens=[512 + 37 * i for i in range(16)], slots=1152),
             name="attend_7b_16x16"),
        # a drafted token that reads 32 of the 512 blocks of a long context, one layer
        dict(_cache("sparse", "llama3_8b", layers=1, tokens=[1], lens=[32768], slots=32832, select=32, first=1, last=2), name="sparse_8b_1"),
        # sixteen users' drafted tokens at contexts of 4000 to 16000 slots, one layer
        dict(_cache("sparse", "qwen2_7b", layers=1, tokens=[1] * 16, lens=[4000 + 800 * i for i in range(16)], slots=16064, select=24,
                    first=1, last=2), name="sparse_7b_users"),
        # the smallest drafter's token, the usual settings
        dict(_sample(1, 1000, 1.0, top_k=50, top_p=0.95), name="sample_tiny"),
        # one drafted token at the paper's second temperature, and the distribution that it was drawn from
        dict(_sample(1, 128256, 0.8, top_p=0.9), name="sample_8b"),
        # sixteen users' drafted tokens, all three filters
        dict(_sample(16, 152064, 0.8, top_k=40, top_p=0.95, min_p=0.02), name="sample_7b_users"),
        # the target's logits at six positions of sixteen users, filtered alike for the acceptance; no token is drawn
        dict(_sample(96, 152064, 0.8, top_p=0.95, draw=False), name="sample_7b_target"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["hold", "attend", "attend", "sparse", "sample", "sample"])
    if kind == "sample":
        vocab = _log_int(rng, 500, 152064)
        drawn = rng.random() < 0.8
        return _sample(_log_int(rng, 1, 96), vocab, round(rng.uniform(0.3, 1.5), 2), top_k=rng.choice([0, 0, 1, _log_int(rng, 2, 2000)]),
                       top_p=rng.choice([1.0, round(rng.uniform(0.3, 0.99), 3)]), min_p=rng.choice([0.0, 0.0, round(rng.uniform(0.005, 0.3), 4)]),
                       draw=drawn, filtered=not drawn or rng.random() < 0.6)
    heads = rng.choice([(4, 2, 64), (7, 1, 64), (32, 8, 128), (32, 8, 128), (28, 4, 128), (8, 8, 64), (8, 1, 128)])
    c = dict(kind=kind, q_heads=heads[0], kv_heads=heads[1], head_dim=heads[2], dtype=rng.choice(["bf16", "bf16", "fp32"]))
    batch = rng.choice([1, 1, 2, 3, 4, 7, 16])
    if kind == "hold":
        most = rng.choice([1, 1, 6, 16, 1500 // batch])
        new = [rng.randint(1, most) for _ in range(batch)]
        to = [rng.choice([0, _log_int(rng, 1, 3000)]) for _ in range(batch)]
        slots = max(a + b for a, b in zip(new, to)) + rng.randint(0, 70)
        c.update(layers=max(1, min(rng.randint(1, 32), 8_000_000 // (batch * heads[1] * slots))))
        c.update(new=",".join(map(str, new)), to=",".join(map(str, to)), slots=slots)
        return c
    lens = [_log_int(rng, 24, 24000 // batch) for _ in range(batch)]
    c.update(layers=rng.choice([1, 1, 2]), lens=",".join(map(str, lens)), slots=max(lens) + rng.randint(0, 70))
    t = rng.randint(1, 4 if kind == "sparse" else 6 if sum(lens) > 6000 else 16)
    c.update(tokens=",".join(str(rng.randint(1, t)) for _ in lens))
    if kind == "sparse":
        first, last = rng.randint(0, 2), rng.randint(1, 3)
        c.update(select=first + last + _log_int(rng, 1, 60), first=first, last=last)
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


def _held(gen, L, B, H, S, D, drift):
    """Codes and scales of a cache: channels of unequal size, and a part that slots have in common with their neighbours."""
    size = torch.exp(_normal(gen, H, 1, D, std=0.5))
    codes = torch.empty(L, B, H, S, D // 2, dtype=torch.uint8, device=DEV)
    scales = torch.empty(L, B, H, S, D // 32, dtype=torch.uint8, device=DEV)
    for layer in range(L):
        for b in range(B):
            common = _normal(gen, H, S // 48 + 1, D, std=drift).repeat_interleave(48, 1)[:, :S]
            codes[layer, b], scales[layer, b] = _quantise(size * (_normal(gen, H, S, D) + common))
    return codes, scales


def prepare(case, seed):
    kind, st = case["kind"], dict(case=case)
    if kind == "sample":
        R, V = case["rows"], case["vocab"]
        st.update(logits=_normal(_gen(seed, 1), R, V, std=2.0), u=torch.rand(R, device=DEV, generator=_gen(seed, 2)),
                  tokens=torch.zeros(R, dtype=torch.int32, device=DEV) if case["draw"] else None,
                  logits_out=torch.zeros(R, V, device=DEV) if case["filtered"] else None)
        return st
    L, H, D, S = case["layers"], case["kv_heads"], case["head_dim"], case["slots"]
    N = (S + BLOCK - 1) // BLOCK
    if kind == "hold":
        new, to = _ints(case["new"]), _ints(case["to"])
        B, n = len(new), max(new)
        gen = _gen(seed, 11)
        for name in ("k", "v"):   # what the cache holds already, and room for what comes
            st[name + "_codes"] = torch.randint(0, 256, (L, B, H, S, D // 2), dtype=torch.uint8, device=DEV, generator=gen)
            st[name + "_scales"] = torch.randint(124, 127, (L, B, H, S, D // 32), dtype=torch.uint8, device=DEV, generator=gen)
            st[name] = _normal(gen, L, B, H, n, D, dtype=_type(case))
            st[name + "_out"] = torch.zeros(L, B, H, n, D, dtype=_type(case), device=DEV)
        touched = [(b, j) for b in range(B) for j in range(to[b] // BLOCK, (to[b] + new[b] - 1) // BLOCK + 1)]
        st.update(bounds=_normal(gen, L, B, H, N, 2, D, dtype=torch.bfloat16), new=np.array(new, np.int32), to=np.array(to, np.int32),
                  lens=np.array([a + b for a, b in zip(new, to)], np.int32), zeros=np.zeros(B, np.int32),
                  seq=torch.tensor([b for b in range(B) for _ in range(new[b])], device=DEV),
                  src=torch.tensor([i for b in range(B) for i in range(new[b])], device=DEV),
                  dst=torch.tensor([to[b] + i for b in range(B) for i in range(new[b])], device=DEV),
                  block_seq=torch.tensor([b for b, _ in touched], device=DEV), block=torch.tensor([j for _, j in touched], device=DEV),
                  block_len=torch.tensor([to[b] + new[b] for b, _ in touched], device=DEV))
        return st
    lens, n = _ints(case["lens"]), _ints(case["tokens"])
    B = len(lens)
    drift = 0.7 if kind == "sparse" else 0.0
    st["k_codes"], st["k_scales"] = _held(_gen(seed, 20), L, B, H, S, D, drift)
    st["v_codes"], st["v_scales"] = _held(_gen(seed, 21), L, B, H, S, D, 0.0)
    st.update(q=_normal(_gen(seed, 22), L, sum(n), case["q_heads"], D, std=1.5), out=torch.zeros(L, sum(n), case["q_heads"], D, device=DEV),
              tokens=np.array(n, np.int32), lens=np.array(lens, np.int32), lens_dev=torch.tensor(lens, device=DEV),
              tokens_dev=torch.tensor(n, device=DEV), token_seq=torch.tensor([b for b in range(B) for _ in range(n[b])], device=DEV),
              token_row=torch.tensor([t for b in range(B) for t in range(n[b])], device=DEV),
              seen=torch.tensor([lens[b] - n[b] + t + 1 for b in range(B) for t in range(n[b])], device=DEV), bounds=None)
    if kind == "sparse":
        st["bounds"] = _bounds(st["k_codes"], st["k_scales"], st["lens_dev"])
        st["blocks"] = torch.zeros(L, sum(n), H, case["select"], dtype=torch.int32, device=DEV)
    return st


# ----------------------------------------------------------------------------------------------------------------
# a cache in 4 bits, in plain operations
# ----------------------------------------------------------------------------------------------------------------

def _quantise(x):
    """Values [..][D] as codes [..][D / 2] and scales [..][D / 32].  All of it is exact but the rounding to a code, which goes to the
    nearest and, half-way, to the even one."""
    x = x.float().unflatten(-1, (-1, 32))
    top = x.abs().amax(-1, keepdim=True)
    power = (torch.frexp(top)[1] - 3).clamp_min(-120)                 # floor(log2(top)) - 2: the largest lies in 4 .. 8
    power = torch.where(top > 0, power, -120)
    a = torch.ldexp(x.abs(), -power)
    code = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    code = (code + (x < 0) * 8).to(torch.uint8).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), (power.squeeze(-1) + 127).to(torch.uint8)


def _values(codes, scales):
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=codes.device)
    x = table[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    return (x.unflatten(-1, (-1, 32)) * torch.exp2(scales.float() - 127.0).unsqueeze(-1)).flatten(-2)


def _bounds(codes, scales, lens):
    """Every block's lowest and highest value of a channel, of the sequences' slots alone."""
    L, B, H, S, _ = codes.shape
    N = (S + BLOCK - 1) // BLOCK
    k = _values(codes, scales)
    there = (torch.arange(S, device=DEV) < lens[:, None])[None, :, None, :, None]
    pad = (0, 0, 0, N * BLOCK - S)
    lo = torch.nn.functional.pad(torch.where(there, k, math.inf), pad, value=math.inf).unflatten(3, (N, BLOCK)).amin(4)
    hi = torch.nn.functional.pad(torch.where(there, k, -math.inf), pad, value=-math.inf).unflatten(3, (N, BLOCK)).amax(4)
    return torch.stack((lo, hi), 4).to(torch.bfloat16)


# ----------------------------------------------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------------------------------------------

def run(st):
    return {"hold": _run_hold, "attend": _run_attend, "sparse": _run_sparse, "sample": _run_sample}[st["case"]["kind"]](st)


def _workspace(st, name, n_bytes):
    """The workspace that a program keeps from its first call on."""
    if name not in st:
        st[name] = torch.empty((n_bytes + 15) // 8, dtype=torch.float64, device=DEV)
    return st[name]


def _layout(es, case, n_seqs):
    return es.easyspec_kv_layout(case["layers"], n_seqs, case["kv_heads"], case["slots"], case["head_dim"],
                                 es.EASYSPEC_DTYPE_BF16 if case["dtype"] == "bf16" else es.EASYSPEC_DTYPE_F32)


def _run_hold(st):
    case = st["case"]
    if own:
        import paper_2502_02493_amd as es
        layout, stream = _layout(es, case, len(st["new"])), torch.cuda.current_stream().cuda_stream
        cache = es.make_kvq(st["k_codes"], st["k_scales"], st["v_codes"], st["v_scales"], st["bounds"])
        n = st["k"].shape[3]
        es.easyspec_kvq_store(st["k"], st["v"], layout, n, st["zeros"], st["new"], st["to"], st["lens"], cache, stream)
        es.easyspec_kvq_load(cache, layout, st["to"], st["new"], n, st["zeros"], st["k_out"], st["v_out"], stream)
        return dict(k=st["k_out"], v=st["v_out"], bounds=st["bounds"])
    seq, src, dst = st["seq"], st["src"], st["dst"]
    for name in ("k", "v"):
        codes, scales = _quantise(st[name])
        st[name + "_codes"][:, seq, :, dst] = codes[:, seq, :, src]
        st[name + "_scales"][:, seq, :, dst] = scales[:, seq, :, src]
        st[name + "_out"][:, seq, :, src] = _values(st[name + "_codes"][:, seq, :, dst], st[name + "_scales"][:, seq, :, dst]).to(_type(case))
    # every block that received a slot: its keys from its first slot on
    at = st["block"][:, None] * BLOCK + torch.arange(BLOCK, device=DEV)
    there = (at < st["block_len"][:, None])[:, :, None, None, None]
    at = at.clamp_max(case["slots"] - 1)
    k = _values(st["k_codes"][:, st["block_seq"][:, None], :, at], st["k_scales"][:, st["block_seq"][:, None], :, at])   # [blocks][64][L][H][D]
    lo, hi = torch.where(there, k, math.inf).amin(1), torch.where(there, k, -math.inf).amax(1)
    st["bounds"][:, st["block_seq"], :, st["block"]] = torch.stack((lo, hi), 3).to(torch.bfloat16)
    return dict(k=st["k_out"], v=st["v_out"], bounds=st["bounds"])


def _own_attention(st, blocks, n_blocks):
    import paper_2502_02493_amd as es
    case = st["case"]
    layout, stream = _layout(es, case, len(st["lens"])), torch.cuda.current_stream().cuda_stream
    cache = es.make_kvq(st["k_codes"], st["k_scales"], st["v_codes"], st["v_scales"], st["bounds"])
    ws = _workspace(st, "ws", 0 if "ws" in st else es.easyspec_kvq_attention_workspace_bytes(layout, st["tokens"], st["lens"], case["q_heads"], n_blocks))
    es.easyspec_kvq_attention(st["q"], cache, layout, st["tokens"], st["lens"], case["q_heads"], blocks, n_blocks, st["out"], ws, stream)
    return st["out"]


def _run_attend(st):
    if own:
        return _own_attention(st, None, 0)
    case = st["case"]
    L, Hq, H, D, S = case["layers"], case["q_heads"], case["kv_heads"], case["head_dim"], case["slots"]
    B, G, M = len(st["lens"]), Hq // H, int(st["tokens"].max())
    k, v = _values(st["k_codes"], st["k_scales"]), _values(st["v_codes"], st["v_scales"])
    q = torch.zeros(L, B, M, H, G, D, device=DEV)
    q[:, st["token_seq"], st["token_row"]] = st["q"].reshape(L, -1, H, G, D)
    q = q.permute(0, 1, 3, 2, 4, 5).reshape(L, B, H, M * G, D)
    s = torch.matmul(q, k.transpose(-1, -2)) * (1.0 / math.sqrt(D))
    slot, row = torch.arange(S, device=DEV), torch.arange(M, device=DEV)
    old = (st["lens_dev"] - st["tokens_dev"])[:, None, None]
    seen = (slot <= old + row[:, None]) & (row[:, None] < st["tokens_dev"][:, None, None])   # [B, M, S]
    seen = seen.repeat_interleave(G, dim=1)[None, :, None]
    s = torch.where(seen, s, -math.inf)
    p = torch.where(seen, torch.exp(s - s.amax(-1, keepdim=True).clamp_min(-1e30)), 0.0)
    p = p / p.sum(-1, keepdim=True).clamp_min(1e-30)
    out = torch.matmul(p, v).reshape(L, B, H, M, G, D).permute(0, 1, 3, 2, 4, 5)
    st["out"].copy_(out[:, st["token_seq"], st["token_row"]].reshape(L, -1, Hq, D))
    return st["out"]


def _run_sparse(st):
    case = st["case"]
    L, Hq, H, D, S, K = case["layers"], case["q_heads"], case["kv_heads"], case["head_dim"], case["slots"], case["select"]
    B, G, T = len(st["lens"]), Hq // H, st["q"].shape[1]
    if own:
        import paper_2502_02493_amd as es
        layout, stream = _layout(es, case, B), torch.cuda.current_stream().cuda_stream
        ws = _workspace(st, "ws_select", 0 if "ws_select" in st else es.easyspec_kvq_select_workspace_bytes(layout, st["tokens"], st["lens"], Hq, K))
        es.easyspec_kvq_select(st["q"], st["bounds"], layout, st["tokens"], st["lens"], Hq, case["first"], case["last"], K, st["blocks"], ws, stream)
        return dict(blocks=st["blocks"], out=_own_attention(st, st["blocks"], K))
    # scores in 64 bits: blocks are compared
    N = st["bounds"].shape[3]
    q = st["q"].reshape(L, T, H, G, 1, D).double()
    b = st["bounds"][:, st["token_seq"]].double().unsqueeze(3)                                  # [L, T, H, 1, N, 2, D]
    score = torch.maximum(q * b[..., 0, :], q * b[..., 1, :]).sum(-1).amax(3)                   # [L, T, H, N]
    j, held = torch.arange(N, device=DEV), ((st["seen"] + BLOCK - 1) // BLOCK)[:, None, None]
    score = torch.where((j < case["first"]) | (j >= held - case["last"]), math.inf, score)
    score = torch.where(j < held, score, -math.inf)
    order = torch.sort(score, dim=-1, descending=True, stable=True)[1]                          # of equal scores the lowest block first
    order = torch.where(j < held, order, N)[..., :K]
    order = torch.nn.functional.pad(torch.sort(order, dim=-1)[0], (0, max(0, K - N)), value=N)
    st["blocks"].copy_(torch.where(order < N, order, -1))
    # attention over the slots of these blocks
    at = (order[..., None] * BLOCK + torch.arange(BLOCK, device=DEV)).flatten(-2)               # [L, T, H, K * 64]
    seen = (at < st["seen"][:, None, None]).unsqueeze(3)
    at = at.clamp_max(S - 1)
    where = (torch.arange(L, device=DEV)[:, None, None, None], st["token_seq"][:, None, None], torch.arange(H, device=DEV)[:, None], at)
    k, v = _values(st["k_codes"][where], st["k_scales"][where]), _values(st["v_codes"][where], st["v_scales"][where])
    s = torch.matmul(st["q"].reshape(L, T, H, G, D), k.transpose(-1, -2)) * (1.0 / math.sqrt(D))
    s = torch.where(seen, s, -math.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    st["out"].copy_(torch.matmul(p, v).reshape(L, T, Hq, D))
    return dict(blocks=st["blocks"], out=st["out"])


def _settings(case):
    """Temperature, top-p and min-p as the calls take them: numbers of 32 bits."""
    return tuple(float(np.float32(case[name])) for name in ("temperature", "top_p", "min_p"))


def _run_sample(st):
    case = st["case"]
    R, V, K = case["rows"], case["vocab"], case["top_k"]
    T, top_p, min_p = _settings(case)
    if own:
        import paper_2502_02493_amd as es
        ws = _workspace(st, "ws", 0 if "ws" in st else es.easyspec_sample_workspace_bytes(R, V))
        es.easyspec_sample(st["logits"], st["u"] if case["draw"] else None, R, V, T, K, top_p, min_p, st["tokens"], st["logits_out"], ws,
                           torch.cuda.current_stream().cuda_stream)
        return {name: st[name] for name in ("tokens", "logits_out") if st[name] is not None}
    # in 64 bits: the sums run over a vocabulary, and who stays is decided by them
    x, order = torch.sort(st["logits"], dim=-1, descending=True, stable=True)   # of equal logits the lowest token first
    z = x.double()
    z = z - z[:, :1]
    w = torch.exp(z / T)
    stays = torch.arange(V, device=DEV) < (K or V)
    w = torch.where(stays, w, 0.0)
    before = torch.cumsum(w, -1) - w
    if top_p < 1:
        stays = stays & (before < top_p * w.sum(-1, keepdim=True))
    if min_p > 0:
        stays = stays & (z >= T * math.log(min_p))
    if st["tokens"] is not None:
        w = torch.where(stays, w, 0.0)
        passed = torch.cumsum(w, -1) <= st["u"].double()[:, None] * w.sum(-1, keepdim=True)
        st["tokens"].copy_(order.gather(1, passed.sum(-1, keepdim=True).clamp_max(V - 1)).squeeze(1))
    if st["logits_out"] is not None:
        st["logits_out"].scatter_(1, order, torch.where(stays, x, -math.inf))
    return {name: st[name] for name in ("tokens", "logits_out") if st[name] is not None}


# ----------------------------------------------------------------------------------------------------------------
# the work
# ----------------------------------------------------------------------------------------------------------------

def work(case):
    if case["kind"] == "sample":
        n = case["rows"] * case["vocab"]
        return dict(bytes=4 * n * (2 if case["filtered"] else 1), flops=4 * n)
    H, D, L = case["kv_heads"], case["head_dim"], case["layers"]
    slot = 2 * (D // 2 + D // 32)     # K and V of a slot
    if case["kind"] == "hold":
        n = sum(_ints(case["new"])) * L * H
        return dict(bytes=n * (2 * slot + 4 * D * (2 if case["dtype"] == "bf16" else 4)), flops=4 * n * D)
    n, lens = _ints(case["tokens"]), _ints(case["lens"])
    rows = 8 * sum(n) * case["q_heads"] * D     # queries and results
    if case["kind"] == "attend":
        seen = sum(n[b] * lens[b] - n[b] * (n[b] - 1) // 2 for b in range(len(n)))
        return dict(bytes=L * (H * sum(lens) * slot + rows), flops=4 * L * case["q_heads"] * D * seen)
    blocks = [(m + BLOCK - 1) // BLOCK for m in lens]
    read = sum(n[b] * min(case["select"] * BLOCK, lens[b]) for b in range(len(n)))
    # every block's bounds once, the selected blocks of every token and KV head
    return dict(bytes=L * (H * (sum(blocks) * 4 * D + read * slot) + rows),
                flops=L * case["q_heads"] * D * (4 * read + 3 * sum(n[b] * blocks[b] for b in range(len(n)))))


# ----------------------------------------------------------------------------------------------------------------
# the definition, in 64 bits
# ----------------------------------------------------------------------------------------------------------------

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def exact(case, seed):
    st = prepare(case, seed)
    return {"hold": _exact_hold, "attend": _exact_attend, "sparse": _exact_sparse, "sample": _exact_sample}[case["kind"]](st)


def _held_values(codes, scales):
    """numpy codes [..][D / 2], scales [..][D / 32] -> float64 [..][D]"""
    x = np.empty(codes.shape[:-1] + (2 * codes.shape[-1],))
    for half in range(2):
        c = (codes >> (4 * half)) & 15
        x[..., half::2] = np.where(c >= 8, -1.0, 1.0) * E2M1[c & 7]
    return x * np.repeat(np.ldexp(1.0, scales.astype(np.int64) - 127), 32, -1)


def _nearest(x):
    """float64 [..][D] -> the nearest values of 4 bits, by distance; half-way to the one with the even code"""
    g = x.reshape(x.shape[:-1] + (-1, 32))
    top = np.abs(g).max(-1, keepdims=True)
    with np.errstate(divide="ignore"):
        power = np.where(top > 0, np.maximum(np.floor(np.log2(top)) - 2, -120), -120)
    unit = np.exp2(power)
    a = np.minimum(np.abs(g) / unit, 6.0)
    best, far = np.zeros(a.shape), np.full(a.shape, np.inf)
    for c in (0, 2, 4, 6, 1, 3, 5, 7):         # an odd code only where it is nearer
        d = np.abs(a - E2M1[c])
        best, far = np.where(d < far, E2M1[c], best), np.minimum(d, far)
    return (np.sign(g) * best * unit).reshape(x.shape)


def _exact_hold(st):
    if st["k"].numel() > 30_000_000:
        return None
    case = st["case"]
    out = {name: st[name + "_out"].double().cpu().numpy() for name in ("k", "v")}
    bounds = st["bounds"].double().cpu().numpy()
    codes, scales = st["k_codes"].cpu().numpy(), st["k_scales"].cpu().numpy()
    new = {name: st[name].double().cpu().numpy() for name in ("k", "v")}
    for b, (n, to) in enumerate(zip(st["new"].tolist(), st["to"].tolist())):
        for name in ("k", "v"):
            out[name][:, b, :, :n] = _nearest(new[name][:, b, :, :n])
        for j in range(to // BLOCK, (to + n - 1) // BLOCK + 1):
            first, end = j * BLOCK, min(j * BLOCK + BLOCK, to + n)
            keys = [_held_values(codes[:, b, :, s], scales[:, b, :, s]) if s < to else out["k"][:, b, :, s - to] for s in range(first, end)]
            bounds[:, b, :, j, 0], bounds[:, b, :, j, 1] = np.min(keys, 0), np.max(keys, 0)
    return dict(k=torch.from_numpy(out["k"]), v=torch.from_numpy(out["v"]), bounds=torch.from_numpy(bounds))


def _exact_slots(st, name, layer, b, h, slots):
    rows = [st[name + part][layer, b, h].index_select(0, slots).cpu().numpy() for part in ("_codes", "_scales")]
    return torch.from_numpy(_held_values(*rows)).to(DEV)


def _attention_of(q, k, v):
    s = k.mv(q.double()) / math.sqrt(k.shape[1])
    return v.t().contiguous().mv(torch.softmax(s, 0))


def _exact_attend(st):
    case = st["case"]
    Hq, H = case["q_heads"], case["kv_heads"]
    if case["layers"] * H * int(st["lens"].sum()) * case["head_dim"] > 150_000_000:
        return None
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device=DEV)
    first = 0
    for b, (n, length) in enumerate(zip(st["tokens"].tolist(), st["lens"].tolist())):
        for layer in range(case["layers"]):
            for h in range(H):
                k, v = (_exact_slots(st, x, layer, b, h, torch.arange(length, device=DEV)) for x in "kv")
                for t in range(n):
                    seen = length - n + t + 1
                    for i in range(h * (Hq // H), (h + 1) * (Hq // H)):
                        out[layer, first + t, i] = _attention_of(st["q"][layer, first + t, i], k[:seen], v[:seen])
        first += n
    return out


def _exact_sparse(st):
    case = st["case"]
    Hq, H, K, G = case["q_heads"], case["kv_heads"], case["select"], case["q_heads"] // case["kv_heads"]
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device=DEV)
    blocks = np.full(st["blocks"].shape, -1, np.int32)
    bounds, q = st["bounds"].double().cpu().numpy(), st["q"].double().cpu().numpy()
    first = 0
    for b, (n, length) in enumerate(zip(st["tokens"].tolist(), st["lens"].tolist())):
        for t in range(first, first + n):
            seen = length - n + (t - first) + 1
            held = (seen + BLOCK - 1) // BLOCK
            for layer in range(case["layers"]):
                for h in range(H):
                    heads = range(h * G, (h + 1) * G)
                    lo, hi = bounds[layer, b, h, :held, 0], bounds[layer, b, h, :held, 1]
                    score = np.max([np.maximum(lo * q[layer, t, i], hi * q[layer, t, i]).sum(-1) for i in heads], 0)
                    forced = [j for j in range(held) if j < case["first"] or j >= held - case["last"]]
                    others = sorted(set(range(held)) - set(forced), key=lambda j: (-score[j], j))
                    chosen = np.array(sorted((forced + others)[:K]), np.int64)
                    blocks[layer, t, h, :len(chosen)] = chosen
                    slots = (chosen[:, None] * BLOCK + np.arange(BLOCK)).reshape(-1)
                    slots = torch.from_numpy(slots[slots < seen]).to(DEV)
                    k, v = (_exact_slots(st, x, layer, b, h, slots) for x in "kv")
                    for i in heads:
                        out[layer, t, i] = _attention_of(st["q"][layer, t, i], k, v)
        first += n
    return dict(blocks=blocks, out=out)


def _exact_sample(st):
    case = st["case"]
    R, V = case["rows"], case["vocab"]
    T, top_p, min_p = _settings(case)
    logits, u = st["logits"].cpu().numpy(), st["u"].cpu().numpy().astype(np.float64)
    tokens, left = np.zeros(R, np.int32), np.full((R, V), -np.inf, np.float32)
    for r in range(R):
        order = np.argsort(-logits[r], kind="stable")[: case["top_k"] or V]
        x = logits[r][order].astype(np.float64)
        mass = np.exp((x - x[0]) / T)
        sums = np.cumsum(mass)
        n = len(order)
        if top_p < 1:     # as many as have a sum in front that is below
            n = int(np.searchsorted(np.concatenate([[0.0], sums[:-1]]), top_p * sums[-1], side="left"))
        if min_p > 0:
            n = min(n, int((x - x[0] >= T * math.log(min_p)).sum()))
        n = max(n, 1)
        tokens[r] = order[min(n - 1, int(np.searchsorted(sums[:n], u[r] * sums[n - 1], side="right")))]
        left[r, order[:n]] = logits[r, order[:n]]
    found = {}
    if st["tokens"] is not None:
        found["tokens"] = tokens
    if st["logits_out"] is not None:
        found["logits_out"] = torch.from_numpy(left)
    return found
