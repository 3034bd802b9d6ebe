"""A float64 decoder on the CPU: every layer is an ordinary causal block over a prefix of the columns, and what the cache holds can be
rounded as 8-bit pages round it."""
import numpy as np

import kv_reference as R


def logits(shape, w, tokens, depth, warmup=0, start=None, kv8=False, first=0):
    """tokens [B][N]; depth[t]: layers of column t.  Logits [N - first][B][V] of columns first .. N - 1, and K, V of every layer
    [B][columns][d] as the cache holds them."""
    B, N = tokens.shape
    d, H, dh = shape.d, shape.H, shape.d // shape.H
    start = np.zeros(B, dtype=int) if start is None else np.asarray(start)
    f8 = lambda a: np.asarray(a, dtype=np.float64)  # noqa: E731
    bf16 = lambda a: R_round(a)  # noqa: E731

    def norm(v, g, b):
        v = v - v.mean(-1, keepdims=True)
        return v / np.sqrt((v * v).mean(-1, keepdims=True) + 1e-5) * f8(g) + f8(b)

    pos = np.maximum(np.arange(N)[None] - start[:, None], 0)
    x = f8(w["tok_emb"])[tokens] + f8(w["pos_emb"])[pos]
    cache = []
    for l in range(shape.L):
        cols = sum(1 for t in range(N) if l < warmup or l >= shape.L - (depth[t] - warmup))
        y = x[:, :cols]
        qkv = norm(y, w["ln1_g"][l], w["ln1_b"][l]) @ f8(w["wqkv"][l]).T + f8(w["bqkv"][l])
        q, k, v = (a.reshape(B, cols, H, dh) for a in np.split(qkv, 3, axis=-1))
        if kv8:
            k, v = R.as_held(bf16(k), R.FP8), R.as_held(bf16(v), R.FP8)
        o = np.zeros((B, cols, H, dh))
        for b in range(B):
            s = np.einsum("ihd,jhd->hij", q[b], k[b]) / np.sqrt(dh)
            seen = (np.arange(cols)[None] <= np.arange(cols)[:, None]) & ((np.arange(cols)[None] >= start[b]) | (np.arange(cols)[:, None] < start[b]))
            s = np.where(seen[None], s, -np.inf)
            p = np.exp(s - s.max(-1, keepdims=True))
            o[b] = np.einsum("hij,jhd->ihd", p / p.sum(-1, keepdims=True), v[b])
        y = y + o.reshape(B, cols, d) @ f8(w["wo"][l]).T + f8(w["bo"][l])
        u = np.maximum(norm(y, w["ln2_g"][l], w["ln2_b"][l]) @ f8(w["w1"][l]).T + f8(w["b1"][l]), 0)
        x = x.copy()
        x[:, :cols] = y + u @ f8(w["w2"][l]).T + f8(w["b2"][l])
        cache.append((k.reshape(B, cols, d), v.reshape(B, cols, d)))
    z = norm(x[:, first:], w["lnf_g"], w["lnf_b"]) @ f8(w.get("lm_head", w["tok_emb"])).T
    return z.transpose(1, 0, 2), cache


def R_round(a):
    import torch
    return torch.from_numpy(np.asarray(a)).float().bfloat16().double().numpy()
