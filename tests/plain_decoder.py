"""A plain float64 decoder whose cache can be thinned and copied: for tests of beams and bounded caches on a context.  Written from
the model function (pre-norm, RMSNorm, rotary pairs i, i + hd/2, grouped-query attention, SwiGLU), one token at a time."""
import copy
import math

import numpy as np

import easyspec_synth as synth


def plain(a, dtype):
    a = np.asarray(a)
    return (synth.bf16_bits_to_f32(a).reshape(a.shape) if a.dtype == np.uint16 else a).astype(np.float64)


class Decoder:
    def __init__(self, cfg, weights):
        self.c, t = cfg, cfg["dtype"]
        self.w = [{k: plain(v, t) for k, v in lw.items() if v is not None} for lw in weights["layers"]]
        self.embed, self.head, self.g = (plain(weights[k], t) for k in ("embed", "lm_head", "g_final"))
        n = cfg["n_layers"]
        self.k, self.v, self.weight = ([[np.zeros((0, cfg["head_dim"])) for _ in range(cfg["n_kv_heads"])] for _ in range(n)] for _ in range(3))
        self.weight = [[np.zeros(0) for _ in range(cfg["n_kv_heads"])] for _ in range(n)]
        self.pos = self.precise = 0   # position of the next token; precise slots

    def clone(self):
        d = copy.copy(self)
        d.k, d.v, d.weight = (copy.deepcopy(x) for x in (self.k, self.v, self.weight))
        return d

    def _norm(self, x, g):
        return x / math.sqrt(np.mean(x * x) + self.c["rms_eps"]) * g

    def _rope(self, x):
        half = self.c["head_dim"] // 2
        a = self.pos * self.c["rope_theta"] ** (-np.arange(half) / half)
        lo, hi = x[..., :half], x[..., half:]
        return np.concatenate([lo * np.cos(a) - hi * np.sin(a), hi * np.cos(a) + lo * np.sin(a)], -1)

    def _stored(self, x):
        if self.c["dtype"] != "bf16":
            return x.astype(np.float32).astype(np.float64)
        return synth.bf16_bits_to_f32(synth.f32_to_bf16_bits(x.astype(np.float32))).reshape(x.shape).astype(np.float64)

    def _attn(self, i, h, weigh):
        w, c = self.w[i], self.c
        hd, G = c["head_dim"], c["n_q_heads"] // c["n_kv_heads"]
        x = self._norm(h, w["g_attn"])
        q, k, v = (w[m] @ x + (w[b] if b in w else 0.0) for m, b in (("wq", "bq"), ("wk", "bk"), ("wv", "bv")))
        q, k, v = q.reshape(-1, hd), k.reshape(-1, hd), v.reshape(-1, hd)
        q, k = self._rope(q), self._stored(self._rope(k))
        v = self._stored(v)
        out = np.zeros_like(q)
        for j in range(c["n_kv_heads"]):
            self.k[i][j] = np.concatenate([self.k[i][j], k[j: j + 1]])
            self.v[i][j] = np.concatenate([self.v[i][j], v[j: j + 1]])
            if weigh:
                self.weight[i][j] = np.append(self.weight[i][j], 0.0)
            for m in range(j * G, j * G + G):
                s = self.k[i][j] @ q[m] / math.sqrt(hd)
                p = np.exp(s - s.max())
                p /= p.sum()
                out[m] = p @ self.v[i][j]
                if weigh:
                    self.weight[i][j] += p
        return w["wo"] @ out.ravel()

    def _mlp(self, i, h):
        w = self.w[i]
        y = self._norm(h, w["g_mlp"])
        z = w["wg"] @ y
        return w["wd"] @ (z / (1 + np.exp(-z)) * (w["wu"] @ y))

    def _token(self, token, bounds, weigh):
        h = self.embed[token].copy()
        for lo, hi in zip(bounds[:-1], bounds[1:]):
            a = [self._attn(i, h, weigh) for i in range(lo, hi)]
            for i in range(lo, hi):
                h = h + a[i - lo]
                h = h + self._mlp(i, h)
        self.pos += 1
        return self.head @ self._norm(h, self.g)

    def drop_fuzzy(self):
        self.pos -= len(self.k[0][0]) - self.precise
        for i in range(self.c["n_layers"]):
            for j in range(self.c["n_kv_heads"]):
                self.k[i][j], self.v[i][j] = self.k[i][j][: self.precise], self.v[i][j][: self.precise]

    def calibrate(self, tokens):
        """Logits after every token."""
        self.drop_fuzzy()
        rows = [self._token(t, range(self.c["n_layers"] + 1), True) for t in tokens]
        self.precise += len(tokens)
        return np.array(rows)

    def draft(self, token, bounds):
        return self._token(token, bounds, False)

    def thin(self, kept):
        """kept[layer][KV head]: the precise slots that stay."""
        self.drop_fuzzy()
        for i in range(self.c["n_layers"]):
            for j in range(self.c["n_kv_heads"]):
                for a in (self.k, self.v, self.weight):
                    a[i][j] = a[i][j][kept[i][j]]
        self.precise = len(kept[0][0])
