"""ctypes binding of libeasyspec.so: one Python function per C entry point of
include/easyspec.h and include/easyspec_instrument.h, same names, argument marshalling only.  Nothing is computed here and there
is no fallback: if the library is missing or no GPU is usable the calls raise."""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libeasyspec.so")

EASYSPEC_OK, EASYSPEC_EINVAL, EASYSPEC_ECAPACITY, EASYSPEC_ESTATE, EASYSPEC_EHIP = 0, -1, -2, -3, -4
EASYSPEC_DTYPE_F32, EASYSPEC_DTYPE_BF16 = 0, 1
EASYSPEC_POLICY_ALIGNED, EASYSPEC_POLICY_PACKED = 0, 1
EASYSPEC_MAX_BATCH, EASYSPEC_MAX_CALIB_TOKENS, EASYSPEC_MAX_SET = 16, 16, 8
EASYSPEC_MAX_TREE_WIDTH, EASYSPEC_MAX_TREE_NODES = 16, 64
EASYSPEC_MAX_CHUNKS = 64
EASYSPEC_PARALLEL_ATTENTION, EASYSPEC_PARALLEL_FULL_LAYER = 0, 1
EASYSPEC_MAX_BEAMS, EASYSPEC_MAX_SELECT, EASYSPEC_MAX_BEAM_VOCAB = 64, 64, 1048576
EASYSPEC_MAX_POSITIONS, EASYSPEC_MAX_CACHE_ROWS = 1048576, 4194304
EASYSPEC_KVQ_BLOCK, EASYSPEC_MAX_KVQ_SELECT, EASYSPEC_MAX_SAMPLE_VOCAB = 64, 1024, 1048576

EXPORTS = ["easyspec_create", "easyspec_destroy", "easyspec_load_weights", "easyspec_set_groups",
           "easyspec_default_groups", "easyspec_draft_step", "easyspec_calibrate", "easyspec_greedy_accept", "easyspec_greedy_accept_host",
           "easyspec_accept", "easyspec_accept_give_up", "easyspec_accept_workspace_bytes", "easyspec_accept_static", "easyspec_accept_static_max_bytes", "easyspec_draft_tree_step", "easyspec_set_parallel_mode", "easyspec_stream_read", "easyspec_stream_read_sink_floats", "easyspec_attention_cut", "easyspec_attention_route", "easyspec_weight_walk", "easyspec_wide_walk", "easyspec_attention_stage_walk",
           "easyspec_get_lens", "easyspec_truncate", "easyspec_kv_import", "easyspec_kv_export",
           "easyspec_get_hidden", "easyspec_poison_workspaces", "easyspec_force_give_up", "easyspec_deny_allocation", "easyspec_step_bytes", "easyspec_profile_begin", "easyspec_profile_end",
           "easyspec_beam_select", "easyspec_beam_select_workspace_bytes", "easyspec_kv_reorder",
           "easyspec_attn_weights", "easyspec_attn_weights_workspace_bytes", "easyspec_kv_evict",
           "easyspec_beam_fork", "easyspec_beam_reorder", "easyspec_track_attention", "easyspec_evict", "easyspec_get_evicted",
           "easyspec_get_attn_weights",
           "easyspec_kvq_store", "easyspec_kvq_load", "easyspec_kvq_attention", "easyspec_kvq_attention_workspace_bytes", "easyspec_kvq_attention_workspace_limit",
           "easyspec_kvq_select", "easyspec_kvq_select_workspace_bytes", "easyspec_sample", "easyspec_sample_workspace_bytes",
           "easyspec_last_error"]
EASYSPEC_OP_QKV, EASYSPEC_OP_ATTN, EASYSPEC_OP_OPROJ, EASYSPEC_OP_GATEUP, EASYSPEC_OP_DOWN, EASYSPEC_OP_HEAD, EASYSPEC_OP_ALL = range(7)


class EasySpecError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"easyspec error {code}: {msg}")
        self.code = code


class easyspec_config(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("d_ffn", C.c_int32), ("vocab", C.c_int32), ("rms_eps", C.c_float),
                ("rope_theta", C.c_float), ("qkv_bias", C.c_int32), ("dtype", C.c_int32), ("max_batch", C.c_int32),
                ("max_ctx", C.c_int32), ("max_calib_tokens", C.c_int32)]


class easyspec_layer_weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("wq", "wk", "wv", "wo", "wg", "wu", "wd", "bq", "bk", "bv", "g_attn", "g_mlp")]


class easyspec_weights(C.Structure):
    _fields_ = [("layers", C.POINTER(easyspec_layer_weights)), ("embed", C.c_void_p), ("lm_head", C.c_void_p),
                ("g_final", C.c_void_p)]


class easyspec_kv_layout(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "n_seqs", "n_kv_heads", "max_slots", "head_dim", "dtype")]


class easyspec_kvq(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k_codes", "v_codes", "k_scales", "v_scales", "k_bounds")]


_lib = None


def load_library():
    """Load libeasyspec.so (built by paper_2502_02493_amd.build).  Raises if it is not there."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} is not built; run `python -m paper_2502_02493_amd.build`")
        L = C.CDLL(LIB_PATH)
        vp, i32 = C.c_void_p, C.c_int32
        L.easyspec_create.argtypes = [C.POINTER(easyspec_config), vp, C.POINTER(vp)]
        L.easyspec_destroy.argtypes = [vp]
        L.easyspec_destroy.restype = None
        L.easyspec_load_weights.argtypes = [vp, C.POINTER(easyspec_weights)]
        L.easyspec_set_groups.argtypes = [vp, vp, i32]
        L.easyspec_default_groups.argtypes = [i32, i32, i32, vp, C.POINTER(i32)]
        L.easyspec_draft_step.argtypes = [vp, vp, vp, vp]
        L.easyspec_set_parallel_mode.argtypes = [vp, i32]
        L.easyspec_calibrate.argtypes = [vp, vp, vp, vp, vp, i32]
        L.easyspec_draft_tree_step.argtypes = [vp, vp, vp, vp, vp, vp]
        L.easyspec_greedy_accept.argtypes = [vp, vp, i32, i32, vp, vp, vp]
        L.easyspec_greedy_accept_host.argtypes = [vp, vp, i32, i32, vp, vp]
        L.easyspec_accept.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, C.c_float, vp, vp, vp, vp]
        L.easyspec_accept_give_up.argtypes = L.easyspec_accept.argtypes
        L.easyspec_accept_static.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, C.c_float, vp, vp, vp]
        L.easyspec_accept_static_max_bytes.argtypes = []
        L.easyspec_accept_static_max_bytes.restype = C.c_int64
        L.easyspec_accept_workspace_bytes.argtypes = [i32, i32, i32]
        L.easyspec_accept_workspace_bytes.restype = C.c_int64
        kvl = C.POINTER(easyspec_kv_layout)
        L.easyspec_beam_select.argtypes = [vp, vp, vp, i32, i32, i32, i32, C.c_float, i32, vp, vp, vp, vp, vp]
        L.easyspec_beam_select_workspace_bytes.argtypes = [i32, i32, i32, i32]
        L.easyspec_beam_select_workspace_bytes.restype = C.c_int64
        L.easyspec_kv_reorder.argtypes = [vp, vp, kvl, vp, i32, i32, i32, vp, vp, vp]
        L.easyspec_attn_weights.argtypes = [vp, vp, kvl, vp, vp, i32, vp, vp, vp, vp]
        L.easyspec_attn_weights_workspace_bytes.argtypes = [kvl, vp, vp, i32]
        L.easyspec_attn_weights_workspace_bytes.restype = C.c_int64
        L.easyspec_kv_evict.argtypes = [vp, vp, vp, kvl, vp, vp, i32, i32, vp, vp, vp, vp, vp]
        kvq = C.POINTER(easyspec_kvq)
        L.easyspec_kvq_store.argtypes = [vp, vp, kvl, i32, vp, vp, vp, vp, kvq, vp]
        L.easyspec_kvq_load.argtypes = [kvq, kvl, vp, vp, i32, vp, vp, vp, vp]
        L.easyspec_kvq_attention.argtypes = [vp, kvq, kvl, vp, vp, i32, vp, i32, vp, vp, vp]
        L.easyspec_kvq_attention_workspace_bytes.argtypes = [kvl, vp, vp, i32, i32]
        L.easyspec_kvq_attention_workspace_bytes.restype = C.c_int64
        L.easyspec_kvq_attention_workspace_limit.argtypes = [kvl, i32, i32, i32]
        L.easyspec_kvq_attention_workspace_limit.restype = C.c_int64
        L.easyspec_kvq_select.argtypes = [vp, vp, kvl, vp, vp, i32, i32, i32, i32, vp, vp, vp]
        L.easyspec_kvq_select_workspace_bytes.argtypes = [kvl, vp, vp, i32, i32]
        L.easyspec_kvq_select_workspace_bytes.restype = C.c_int64
        L.easyspec_sample.argtypes = [vp, vp, i32, i32, C.c_float, i32, C.c_float, C.c_float, vp, vp, vp, vp]
        L.easyspec_sample_workspace_bytes.argtypes = [i32, i32]
        L.easyspec_sample_workspace_bytes.restype = C.c_int64
        L.easyspec_beam_fork.argtypes = [vp, i32, i32, i32]
        L.easyspec_beam_reorder.argtypes = [vp, i32, i32, vp, i32]
        L.easyspec_track_attention.argtypes = [vp, i32]
        L.easyspec_evict.argtypes = [vp, vp, i32]
        L.easyspec_get_evicted.argtypes = [vp, vp]
        L.easyspec_get_attn_weights.argtypes = [vp, i32, vp, i32]
        L.easyspec_get_lens.argtypes = [vp, vp, vp]
        L.easyspec_truncate.argtypes = [vp, i32, i32]
        L.easyspec_kv_import.argtypes = [vp, i32, vp, vp, i32]
        L.easyspec_kv_export.argtypes = [vp, i32, vp, vp, i32]
        L.easyspec_get_hidden.argtypes = [vp, vp, i32, C.POINTER(i32)]
        L.easyspec_step_bytes.argtypes = [vp]
        L.easyspec_poison_workspaces.argtypes = [vp]
        L.easyspec_force_give_up.argtypes = [vp, i32]
        L.easyspec_deny_allocation.argtypes = [vp, i32]
        L.easyspec_stream_read.argtypes = [vp, C.c_int64, vp, vp]
        L.easyspec_stream_read_sink_floats.argtypes = []
        L.easyspec_attention_cut.argtypes = [C.POINTER(easyspec_config), vp, i32, i32, vp, vp]
        L.easyspec_attention_route.argtypes = [C.POINTER(easyspec_config), vp, vp, i32, i32, vp]
        L.easyspec_step_bytes.restype = C.c_int64
        L.easyspec_weight_walk.argtypes = [C.POINTER(easyspec_config), i32, i32, i32, i32, vp]
        L.easyspec_wide_walk.argtypes = [C.POINTER(easyspec_config), i32, i32, vp]
        L.easyspec_attention_stage_walk.argtypes = [i32, vp]
        L.easyspec_profile_begin.argtypes = [vp, i32, i32]
        L.easyspec_profile_end.argtypes = [vp, C.POINTER(i32), C.POINTER(C.c_float), vp, vp]
        L.easyspec_last_error.argtypes = [vp]
        L.easyspec_last_error.restype = C.c_char_p
        _lib = L
    return _lib


def _ptr(x):
    """Address of a torch tensor, numpy array, raw int or None."""
    if x is None or type(x) is int:
        return x
    if type(x) is np.ndarray:
        assert x.flags["C_CONTIGUOUS"]
        return x.__array_interface__["data"][0]  # x.ctypes.data, at a third of its time
    try:  # a tensor, of which most calls have five to ten: asking for its kind first takes as long as its address
        assert x.is_contiguous()
        return x.data_ptr()
    except AttributeError:
        pass
    if isinstance(x, np.ndarray):
        return _ptr(x.view(np.ndarray))
    if isinstance(x, int):
        return x
    raise TypeError(type(x))


def _check(rc, ctx):
    if rc != EASYSPEC_OK:
        raise EasySpecError(rc, easyspec_last_error(ctx))


def easyspec_last_error(ctx=None) -> str:
    return load_library().easyspec_last_error(ctx).decode()


class _Context(C.c_void_p):
    """The handle that easyspec_create returns, with the length of the host arrays that hold an entry per sequence."""
    max_batch = None


def easyspec_create(cfg: easyspec_config, hip_stream=None):
    h = _Context()
    _check(load_library().easyspec_create(C.byref(cfg), _ptr(hip_stream), C.byref(h)), None)
    h.max_batch = int(cfg.max_batch)
    return h


def easyspec_destroy(ctx):
    load_library().easyspec_destroy(ctx)


def easyspec_load_weights(ctx, weights: dict):
    """weights: the dict layout of easyspec_synth.make_weights; values are numpy arrays (host) or
    torch tensors (host or device)."""
    keep = []

    def p(a):
        if a is None:
            return None
        if isinstance(a, np.ndarray):
            a = np.ascontiguousarray(a)
        keep.append(a)
        return _ptr(a)

    n = len(weights["layers"])
    arr = (easyspec_layer_weights * n)()
    for i, lw in enumerate(weights["layers"]):
        for name in ("wq", "wk", "wv", "wo", "wg", "wu", "wd", "g_attn", "g_mlp"):
            setattr(arr[i], name, p(lw[name]))
        for name in ("bq", "bk", "bv"):
            setattr(arr[i], name, p(lw.get(name)))
    w = easyspec_weights(arr, p(weights["embed"]), p(weights["lm_head"]), p(weights["g_final"]))
    _check(load_library().easyspec_load_weights(ctx, C.byref(w)), ctx)


def easyspec_set_groups(ctx, bounds):
    b = np.ascontiguousarray(bounds, dtype=np.int32)
    _check(load_library().easyspec_set_groups(ctx, _ptr(b), b.size - 1), ctx)


def easyspec_default_groups(n_layers: int, N: int, policy: int) -> np.ndarray:
    b = np.zeros(max(n_layers, 0) + 2, dtype=np.int32)
    n = C.c_int32(0)
    _check(load_library().easyspec_default_groups(n_layers, N, policy, _ptr(b), C.byref(n)), None)
    return b[: n.value + 1].copy()


def easyspec_draft_step(ctx, tokens_in, tokens_out, logits_out=None):
    _check(load_library().easyspec_draft_step(ctx, _ptr(tokens_in), _ptr(tokens_out), _ptr(logits_out)), ctx)


def easyspec_calibrate(ctx, tokens, n_tokens, next_token_out, logits_out=None, logits_rows=0):
    n = np.ascontiguousarray(n_tokens, dtype=np.int32)
    _check(load_library().easyspec_calibrate(ctx, _ptr(tokens), _ptr(n), _ptr(next_token_out), _ptr(logits_out),
                                             int(logits_rows)), ctx)


def easyspec_set_parallel_mode(ctx, mode: int):
    _check(load_library().easyspec_set_parallel_mode(ctx, int(mode)), ctx)


def easyspec_draft_tree_step(ctx, tokens_in, n_nodes, parents, tokens_out, logits_out=None):
    n = np.ascontiguousarray(n_nodes, dtype=np.int32)
    p = np.ascontiguousarray(parents, dtype=np.int32)
    assert p.size == n.size * EASYSPEC_MAX_TREE_WIDTH
    _check(load_library().easyspec_draft_tree_step(ctx, _ptr(tokens_in), _ptr(n), _ptr(p), _ptr(tokens_out), _ptr(logits_out)), ctx)


def easyspec_greedy_accept(draft, target_argmax, batch, gamma, accept_len, bonus, hip_stream=None):
    _check(load_library().easyspec_greedy_accept(_ptr(draft), _ptr(target_argmax), batch, gamma, _ptr(accept_len),
                                                 _ptr(bonus), _ptr(hip_stream)), None)


def easyspec_greedy_accept_host(draft, target_argmax, batch, gamma, accept_len, bonus):
    _check(load_library().easyspec_greedy_accept_host(_ptr(draft), _ptr(target_argmax), batch, gamma, _ptr(accept_len),
                                                      _ptr(bonus)), None)


def easyspec_accept(draft, draft_logits, target_logits, r, u, batch, gamma, vocab, temperature, accept_len, bonus,
                    workspace, hip_stream=None):
    _check(load_library().easyspec_accept(_ptr(draft), _ptr(draft_logits), _ptr(target_logits), _ptr(r), _ptr(u), batch,
                                          gamma, vocab, float(temperature), _ptr(accept_len), _ptr(bonus), _ptr(workspace),
                                          _ptr(hip_stream)), None)


def easyspec_accept_give_up(draft, draft_logits, target_logits, r, u, batch, gamma, vocab, temperature, accept_len, bonus,
                            workspace, hip_stream=None):
    _check(load_library().easyspec_accept_give_up(_ptr(draft), _ptr(draft_logits), _ptr(target_logits), _ptr(r), _ptr(u), batch,
                                                  gamma, vocab, float(temperature), _ptr(accept_len), _ptr(bonus), _ptr(workspace),
                                                  _ptr(hip_stream)), None)


def easyspec_accept_static(draft, draft_logits, target_logits, r, u, batch, gamma, vocab, temperature, accept_len, bonus,
                           hip_stream=None):
    _check(load_library().easyspec_accept_static(_ptr(draft), _ptr(draft_logits), _ptr(target_logits), _ptr(r), _ptr(u), batch,
                                                 gamma, vocab, float(temperature), _ptr(accept_len), _ptr(bonus),
                                                 _ptr(hip_stream)), None)


def easyspec_accept_static_max_bytes() -> int:
    return int(load_library().easyspec_accept_static_max_bytes())


def easyspec_accept_workspace_bytes(batch: int, gamma: int, vocab: int) -> int:
    return int(load_library().easyspec_accept_workspace_bytes(batch, gamma, vocab))


def easyspec_beam_select(logits, scores, ended, groups, beams, vocab, n_select, temperature, end_token, tokens_out, parents_out,
                         scores_out, workspace, hip_stream=None):
    _check(load_library().easyspec_beam_select(_ptr(logits), _ptr(scores), _ptr(ended), groups, beams, vocab, n_select,
                                               float(temperature), end_token, _ptr(tokens_out), _ptr(parents_out), _ptr(scores_out),
                                               _ptr(workspace), _ptr(hip_stream)), None)


def easyspec_beam_select_workspace_bytes(groups: int, beams: int, vocab: int, n_select: int) -> int:
    return int(load_library().easyspec_beam_select_workspace_bytes(groups, beams, vocab, n_select))


_INT32 = np.dtype(np.int32)


def _host_ints(x, n):
    """An array of n host integers, all of which the library reads (n None: a handle that does not say how many)."""
    a = np.ascontiguousarray(x, _INT32)
    if n is not None and a.size != n:
        raise EasySpecError(EASYSPEC_EINVAL, f"an array of {a.size} entries where there are {n} sequences")
    return a


def easyspec_kv_reorder(k, v, layout: easyspec_kv_layout, parents, beams, from_slot, to_slot, k_out, v_out, hip_stream=None):
    _check(load_library().easyspec_kv_reorder(_ptr(k), _ptr(v), C.byref(layout), _ptr(parents), beams, from_slot, to_slot, _ptr(k_out),
                                              _ptr(v_out), _ptr(hip_stream)), None)


def easyspec_attn_weights(q, k, layout: easyspec_kv_layout, n_tokens, lens, n_q_heads, weights_in, weights_out, workspace, hip_stream=None):
    n, s = _host_ints(n_tokens, layout.n_seqs), _host_ints(lens, layout.n_seqs)
    _check(load_library().easyspec_attn_weights(_ptr(q), _ptr(k), C.byref(layout), _ptr(n), _ptr(s), n_q_heads, _ptr(weights_in),
                                                _ptr(weights_out), _ptr(workspace), _ptr(hip_stream)), None)


def easyspec_attn_weights_workspace_bytes(layout: easyspec_kv_layout, n_tokens, lens, n_q_heads) -> int:
    n, s = _host_ints(n_tokens, layout.n_seqs), _host_ints(lens, layout.n_seqs)
    return int(load_library().easyspec_attn_weights_workspace_bytes(C.byref(layout), _ptr(n), _ptr(s), n_q_heads))


def easyspec_kv_evict(k, v, weights, layout: easyspec_kv_layout, lens, keep, recent, out_slots, k_out, v_out, weights_out, slots_out,
                      hip_stream=None):
    n, s = _host_ints(lens, layout.n_seqs), _host_ints(keep, layout.n_seqs)
    _check(load_library().easyspec_kv_evict(_ptr(k), _ptr(v), _ptr(weights), C.byref(layout), _ptr(n), _ptr(s), recent, out_slots,
                                            _ptr(k_out), _ptr(v_out), _ptr(weights_out), _ptr(slots_out), _ptr(hip_stream)), None)


def make_kvq(k_codes, k_scales, v_codes, v_scales, k_bounds=None) -> easyspec_kvq:
    """easyspec_kvq of a cache's arrays (device tensors, which the caller keeps; raw addresses)."""
    return easyspec_kvq(_ptr(k_codes), _ptr(v_codes), _ptr(k_scales), _ptr(v_scales), _ptr(k_bounds))


def _int_bytes(x, n):
    """_host_ints for arrays that are only read during the call: bytes, which ctypes passes on as they are (an array's address takes 0.7 us to ask for)."""
    return _host_ints(x, n).tobytes()


def easyspec_kvq_store(k, v, layout: easyspec_kv_layout, src_slots, src_from, n_slots, to, lens, cache: easyspec_kvq, hip_stream=None):
    f, n, t, s = (_int_bytes(x, layout.n_seqs) for x in (src_from, n_slots, to, lens))
    _check(load_library().easyspec_kvq_store(_ptr(k), _ptr(v), C.byref(layout), src_slots, f, n, t, s, C.byref(cache),
                                             _ptr(hip_stream)), None)


def easyspec_kvq_load(cache: easyspec_kvq, layout: easyspec_kv_layout, from_, n_slots, out_slots, to, k_out, v_out, hip_stream=None):
    f, n, t = (_int_bytes(x, layout.n_seqs) for x in (from_, n_slots, to))
    _check(load_library().easyspec_kvq_load(C.byref(cache), C.byref(layout), f, n, out_slots, t, _ptr(k_out), _ptr(v_out),
                                            _ptr(hip_stream)), None)


def easyspec_kvq_attention(q, cache: easyspec_kvq, layout: easyspec_kv_layout, n_tokens, lens, n_q_heads, blocks, n_blocks, out, workspace,
                           hip_stream=None):
    n, s = _int_bytes(n_tokens, layout.n_seqs), _int_bytes(lens, layout.n_seqs)
    _check(load_library().easyspec_kvq_attention(_ptr(q), C.byref(cache), C.byref(layout), n, s, n_q_heads, _ptr(blocks), n_blocks,
                                                 _ptr(out), _ptr(workspace), _ptr(hip_stream)), None)


def easyspec_kvq_attention_workspace_bytes(layout: easyspec_kv_layout, n_tokens, lens, n_q_heads, n_blocks) -> int:
    n, s = _int_bytes(n_tokens, layout.n_seqs), _int_bytes(lens, layout.n_seqs)
    return int(load_library().easyspec_kvq_attention_workspace_bytes(C.byref(layout), n, s, n_q_heads, n_blocks))


def easyspec_kvq_attention_workspace_limit(layout: easyspec_kv_layout, max_tokens: int, n_q_heads: int, max_blocks: int) -> int:
    return int(load_library().easyspec_kvq_attention_workspace_limit(C.byref(layout), max_tokens, n_q_heads, max_blocks))


def easyspec_kvq_select(q, k_bounds, layout: easyspec_kv_layout, n_tokens, lens, n_q_heads, keep_first, keep_last, n_select, blocks_out, workspace,
                        hip_stream=None):
    n, s = _int_bytes(n_tokens, layout.n_seqs), _int_bytes(lens, layout.n_seqs)
    _check(load_library().easyspec_kvq_select(_ptr(q), _ptr(k_bounds), C.byref(layout), n, s, n_q_heads, keep_first, keep_last, n_select,
                                              _ptr(blocks_out), _ptr(workspace), _ptr(hip_stream)), None)


def easyspec_kvq_select_workspace_bytes(layout: easyspec_kv_layout, n_tokens, lens, n_q_heads, n_select) -> int:
    n, s = _int_bytes(n_tokens, layout.n_seqs), _int_bytes(lens, layout.n_seqs)
    return int(load_library().easyspec_kvq_select_workspace_bytes(C.byref(layout), n, s, n_q_heads, n_select))


def easyspec_sample(logits, u, rows, vocab, temperature, top_k, top_p, min_p, tokens_out, logits_out, workspace, hip_stream=None):
    _check(load_library().easyspec_sample(_ptr(logits), _ptr(u), rows, vocab, float(temperature), top_k, float(top_p), float(min_p), _ptr(tokens_out),
                                          _ptr(logits_out), _ptr(workspace), _ptr(hip_stream)), None)


def easyspec_sample_workspace_bytes(rows: int, vocab: int) -> int:
    return int(load_library().easyspec_sample_workspace_bytes(rows, vocab))


def easyspec_beam_fork(ctx, source: int, first: int, count: int):
    _check(load_library().easyspec_beam_fork(ctx, source, first, count), ctx)


def easyspec_beam_reorder(ctx, first: int, count: int, parents, from_slot: int):
    _check(load_library().easyspec_beam_reorder(ctx, first, count, _ptr(parents), from_slot), ctx)


def easyspec_track_attention(ctx, max_positions: int):
    _check(load_library().easyspec_track_attention(ctx, max_positions), ctx)


def easyspec_evict(ctx, keep, recent: int):
    k = _host_ints(keep, getattr(ctx, "max_batch", None))
    _check(load_library().easyspec_evict(ctx, _ptr(k), recent), ctx)


def easyspec_get_evicted(ctx, max_batch: int):
    n = _host_ints(np.zeros(max_batch, np.int32), getattr(ctx, "max_batch", None))
    _check(load_library().easyspec_get_evicted(ctx, _ptr(n)), ctx)
    return n


def easyspec_get_attn_weights(ctx, b: int, out, n_slots: int):
    _check(load_library().easyspec_get_attn_weights(ctx, b, _ptr(out), n_slots), ctx)


def easyspec_stream_read(buf, nbytes: int, sink, hip_stream=None):
    _check(load_library().easyspec_stream_read(_ptr(buf), int(nbytes), _ptr(sink), _ptr(hip_stream)), None)


def easyspec_stream_read_sink_floats() -> int:
    return int(load_library().easyspec_stream_read_sink_floats())


def easyspec_attention_cut(cfg: easyspec_config, ctx_lens, n_layers_in_set: int, with_ranges=True):
    """(waves per workgroup, n_chunks[n_cols], ranges[n_cols][EASYSPEC_MAX_CHUNKS][8][2] or None)."""
    lens = np.ascontiguousarray(ctx_lens, dtype=np.int32)
    n_chunks = np.zeros(len(lens), np.int32)
    ranges = np.zeros((len(lens), EASYSPEC_MAX_CHUNKS, 8, 2), np.int32) if with_ranges else None
    rc = load_library().easyspec_attention_cut(C.byref(cfg), _ptr(lens), len(lens), int(n_layers_in_set), _ptr(n_chunks),
                                               _ptr(ranges))
    if rc < 0:
        _check(rc, None)
    return rc, n_chunks, ranges


def easyspec_attention_route(cfg: easyspec_config, ctx_lens, seqs, n_layers_in_set: int):
    """(matrix cores, bf16 terms of a probability, tiles of 16 query rows per workgroup)."""
    lens, seqs = (np.ascontiguousarray(a, dtype=np.int32) for a in (ctx_lens, seqs))
    assert len(lens) == len(seqs)
    route = np.zeros(3, np.int32)
    _check(load_library().easyspec_attention_route(C.byref(cfg), _ptr(lens), _ptr(seqs), len(lens), int(n_layers_in_set),
                                                   _ptr(route)), None)
    return bool(route[0]), int(route[1]), int(route[2])


EASYSPEC_WALK_FIELDS = 16
WALK_NAMES = ("grid", "waves", "units_per_wg", "tile_rows", "fragments", "w_max", "w_pieces", "w_out_of_range", "x_max",
              "x_slot_elems", "x_out_of_range", "tiles", "missed_tiles", "repeated_tiles", "reread_tiles", "uncovered_pieces")


def easyspec_weight_walk(cfg: easyspec_config, op: int, n_cols: int, n_layers_in_set: int, full_layer: bool = False) -> dict:
    rep = np.zeros(EASYSPEC_WALK_FIELDS, np.int64)
    _check(load_library().easyspec_weight_walk(C.byref(cfg), int(op), int(n_cols), int(n_layers_in_set), int(bool(full_layer)),
                                               _ptr(rep)), None)
    return dict(zip(WALK_NAMES, (int(v) for v in rep)))


EASYSPEC_WIDE_FIELDS = 22
WIDE_NAMES = ("row_tiles", "col_tiles", "stage_tiles", "col_blocks", "row_blocks", "splits", "per_split", "grid", "kernel",
              "w_max", "w_pieces", "w_out_of_range", "x_max", "x_pieces", "x_out_of_range", "products", "missed", "repeated",
              "misplaced", "empty_splits", "out_max", "out_room")


def easyspec_wide_walk(cfg: easyspec_config, op: int, n_cols: int) -> dict:
    rep = np.zeros(EASYSPEC_WIDE_FIELDS, np.int64)
    _check(load_library().easyspec_wide_walk(C.byref(cfg), int(op), int(n_cols), _ptr(rep)), None)
    return dict(zip(WIDE_NAMES, (int(v) for v in rep)))


EASYSPEC_STAGE_FIELDS = 9
STAGE_NAMES = ("stored", "distinct_places", "highest_place", "places", "fetched", "wrong_piece", "unused_rows", "misplaced_scores",
               "bank_conflicts")


def easyspec_attention_stage_walk(n_loads: int) -> dict:
    rep = np.zeros(EASYSPEC_STAGE_FIELDS, np.int64)
    _check(load_library().easyspec_attention_stage_walk(int(n_loads), _ptr(rep)), None)
    return dict(zip(STAGE_NAMES, (int(v) for v in rep)))


def easyspec_get_lens(ctx, max_batch: int):
    p, f = np.zeros(max_batch, np.int32), np.zeros(max_batch, np.int32)
    _check(load_library().easyspec_get_lens(ctx, _ptr(p), _ptr(f)), ctx)
    return p, f


def easyspec_truncate(ctx, b: int, new_precise_len: int):
    _check(load_library().easyspec_truncate(ctx, b, new_precise_len), ctx)


def easyspec_kv_import(ctx, b: int, k, v, n_slots: int):
    _check(load_library().easyspec_kv_import(ctx, b, _ptr(k), _ptr(v), n_slots), ctx)


def easyspec_kv_export(ctx, b: int, k, v, n_slots: int):
    _check(load_library().easyspec_kv_export(ctx, b, _ptr(k), _ptr(v), n_slots), ctx)


def easyspec_get_hidden(ctx, out, max_rows: int) -> int:
    n = C.c_int32(0)
    _check(load_library().easyspec_get_hidden(ctx, _ptr(out), max_rows, C.byref(n)), ctx)
    return n.value


def easyspec_poison_workspaces(ctx):
    _check(load_library().easyspec_poison_workspaces(ctx), ctx)


def easyspec_deny_allocation(ctx, n: int):
    _check(load_library().easyspec_deny_allocation(ctx, int(n)), ctx)


def easyspec_force_give_up(ctx, on: bool):
    _check(load_library().easyspec_force_give_up(ctx, int(on)), ctx)


def easyspec_step_bytes(ctx) -> int:
    return int(load_library().easyspec_step_bytes(ctx))


def easyspec_profile_begin(ctx, op: int, max_launches: int):
    _check(load_library().easyspec_profile_begin(ctx, op, max_launches), ctx)


def easyspec_profile_end(ctx, per_launch=None, per_launch_op=None):
    """Returns (timed launches, total milliseconds); per_launch / per_launch_op: float32 / int32 numpy arrays of
    at least max_launches entries that receive each launch's milliseconds and kernel class."""
    n, ms = C.c_int32(0), C.c_float(0.0)
    assert per_launch is None or per_launch.dtype == np.float32
    assert per_launch_op is None or per_launch_op.dtype == np.int32
    _check(load_library().easyspec_profile_end(ctx, C.byref(n), C.byref(ms), _ptr(per_launch), _ptr(per_launch_op)), ctx)
    return n.value, ms.value


def make_config(shape: dict, max_batch: int, max_ctx: int, max_calib_tokens: int) -> easyspec_config:
    """easyspec_config from a model-shape dict (fields of easyspec_synth.model_shape)."""
    return easyspec_config(shape["n_layers"], shape["d_model"], shape["n_q_heads"], shape["n_kv_heads"],
                           shape["head_dim"], shape["d_ffn"], shape["vocab"], shape["rms_eps"], shape["rope_theta"],
                           int(shape["qkv_bias"]), EASYSPEC_DTYPE_BF16 if shape["dtype"] == "bf16" else EASYSPEC_DTYPE_F32,
                           max_batch, max_ctx, max_calib_tokens)
