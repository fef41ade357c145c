"""Device arrays and calls for the tests of the operators on caches held in 4 bits."""
import numpy as np

import kvq_ref as ref

BLOCK = 64


def stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Cache:
    """A cache in 4 bits on the device, its arrays filled with a byte that shows."""

    def __init__(self, es, L, B, H, S, hd, dtype="bf16", bounds=True, fill=0xA5):
        import torch
        self.es, self.shape = es, (L, B, H, S, hd)
        self.layout = es.easyspec_kv_layout(L, B, H, S, hd, es.EASYSPEC_DTYPE_BF16 if dtype == "bf16" else es.EASYSPEC_DTYPE_F32)
        full = lambda *s: torch.full(s, fill, dtype=torch.uint8, device="cuda")  # noqa: E731
        self.kc, self.vc = full(L, B, H, S, hd // 2), full(L, B, H, S, hd // 2)
        self.ks, self.vs = full(L, B, H, S, hd // 32), full(L, B, H, S, hd // 32)
        self.bounds = torch.full((L, B, H, -(-S // BLOCK), 2, hd), 77.0, dtype=torch.bfloat16, device="cuda") if bounds else None
        self.c = es.make_kvq(self.kc, self.ks, self.vc, self.vs, self.bounds)

    def put(self, k, v, slots=slice(None)):
        """Numbers k, v [L, B, H, n, hd] into slots, encoded on the host."""
        for codes, scales, x in ((self.kc, self.ks, k), (self.vc, self.vs, v)):
            c, s = ref.encode(x)
            codes[:, :, :, slots], scales[:, :, :, slots] = dev(c), dev(s)
        return self

    def values(self):
        return [ref.decode(c.cpu().numpy(), s.cpu().numpy()) for c, s in ((self.kc, self.ks), (self.vc, self.vs))]

    def bytes(self):
        return [x.cpu().numpy().copy() for x in (self.kc, self.ks, self.vc, self.vs)] + ([] if self.bounds is None else [self.bounds.float().cpu().numpy().copy()])


def random_cache(es, seed, L, B, H, S, hd, std=1.0):
    g = np.random.default_rng(seed)
    size = np.exp(g.normal(0, 0.5, hd))
    return Cache(es, L, B, H, S, hd).put(g.normal(0, std, (L, B, H, S, hd)) * size, g.normal(0, 1, (L, B, H, S, hd)))


def queries(seed, L, T, Hq, hd, std=1.5):
    return np.random.default_rng(seed + 1000).normal(0, std, (L, T, Hq, hd)).astype(np.float32)


def attend(cache, q, n, lens, blocks=None, ws=None, out=None, on=None):
    import torch
    es, (L, _, _, _, _) = cache.es, cache.shape
    Hq, n_blocks = q.shape[2], 0 if blocks is None else blocks.shape[-1]
    out = torch.full(tuple(q.shape), -3.0, device="cuda") if out is None else out
    need = es.easyspec_kvq_attention_workspace_bytes(cache.layout, n, lens, Hq, n_blocks)
    assert need >= 0
    ws = torch.full((need // 4 + 4,), float("nan"), device="cuda") if ws is None else ws
    es.easyspec_kvq_attention(q, cache.c, cache.layout, n, lens, Hq, blocks, n_blocks, out, ws, (on or torch.cuda.current_stream()).cuda_stream)
    return out


def select(cache, q, n, lens, keep_first, keep_last, n_select, out=None, ws=None):
    import torch
    es, Hq = cache.es, q.shape[2]
    out = torch.full((q.shape[0], q.shape[1], cache.shape[2], n_select), -7, dtype=torch.int32, device="cuda") if out is None else out
    need = es.easyspec_kvq_select_workspace_bytes(cache.layout, n, lens, Hq, n_select)
    assert need >= 0
    ws = torch.full((need // 4 + 4,), float("nan"), device="cuda") if ws is None else ws
    es.easyspec_kvq_select(q, cache.bounds, cache.layout, n, lens, Hq, keep_first, keep_last, n_select, out, ws, stream())
    return out


def check_attention(cache, q, n, lens, out, blocks=None):
    k, v = cache.values()
    want, tol = ref.attention(q.double().cpu().numpy(), k, v, n, lens, None if blocks is None else blocks.cpu().numpy())
    got = out.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    fine = ~np.isnan(want)
    err = np.abs(got - want)[fine]
    assert np.all(err <= tol[fine]), float((err / np.maximum(tol[fine], 1e-300)).max())
