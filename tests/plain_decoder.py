"""A plain decoder in numpy, 64 bits: the layers of streaming.WindowedDecoder written from their definition, with a
given rounding of what enters the cache and a window with sinks."""
import numpy as np

import window_ref as W


def tensors(orc, m, seed):
    """Weights [layer][name] and (embed, lm_head, g_final) of the generated model."""
    H, F, d, V = m["hidden"], m["ffn"], m["head_dim"], m["vocab"]
    qd, kvd = m["n_heads"] * d, m["n_kv_heads"] * d

    def gen(shape, tid, kind=0):
        return orc.bf16_bits_to_f64(orc.gen_tensor(seed, tid, int(np.prod(shape)), kind)).reshape(shape)

    names = [("g_attn", (H,), 1), ("wq", (qd, H), 0), ("wk", (kvd, H), 0), ("wv", (kvd, H), 0), ("wo", (H, qd), 0),
             ("g_mlp", (H,), 1), ("wg", (F, H), 0), ("wu", (F, H), 0), ("wd", (H, F), 0)]
    layers = []
    for l in range(m["n_layers"]):
        w = {name: gen(shape, orc.tensor_id(l, i), kind) for i, (name, shape, kind) in enumerate(names)}
        for i, name in ((9, "g_q"), (10, "g_k")):
            w[name] = gen((d,), orc.tensor_id(l, i), 1) if m.get("qk_norm") else None
        layers.append(w)
    return layers, (gen((V, H), orc.tensor_id(-1, 0)), gen((V, H), orc.tensor_id(-1, 1)), gen((H,), orc.tensor_id(-1, 2), 1))


def norm(x, g, eps):
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * g


def forward(orc, m, seed, tokens, round_kv, window, sinks):
    """(hidden, logits) of every token; round_kv: what the cache makes of keys and values [n][Hkv][d]."""
    layers, (embed, lm_head, g_final) = tensors(orc, m, seed)
    Hq, Hkv, d, eps, n = m["n_heads"], m["n_kv_heads"], m["head_dim"], m.get("rms_eps", 1e-5), len(tokens)
    x = embed[np.asarray(tokens)].copy()
    pos = np.arange(n)
    sees = W.visible(pos[:, None], pos[None, :], window, sinks)
    for w in layers:
        y = norm(x, w["g_attn"], eps)
        rows = np.concatenate([y @ w["wq"].T, y @ w["wk"].T, y @ w["wv"].T], 1)
        q, k, v = (np.stack(a) for a in zip(*(W.append_row(rows[t], t, Hq, Hkv, d, w["g_q"], w["g_k"], eps,
                                                           m["rope_theta"])[:3] for t in range(n))))
        k, v = round_kv(k), round_kv(v)
        G = Hq // Hkv
        s = np.einsum("tgid,jgd->tgij", q.reshape(n, Hkv, G, d), k) / np.sqrt(d)
        s = np.where(sees[:, None, None, :], s, -np.inf)
        p = np.exp(s - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        x = x + np.einsum("tgij,jgd->tgid", p, v).reshape(n, Hq * d) @ w["wo"].T
        y = norm(x, w["g_mlp"], eps)
        gate = y @ w["wg"].T
        x = x + (gate / (1 + np.exp(-gate)) * (y @ w["wu"].T)) @ w["wd"].T
    z = norm(x, g_final, eps)
    return z, z @ lm_head.T
