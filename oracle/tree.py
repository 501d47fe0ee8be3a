"""Drafted tokens: trees of new tokens, normalised heads, rules on logits (test infrastructure).

A sequence's new tokens form a tree (`parents`: index of an earlier node, -1 below the cached prefix, -2 padding).  Node i
sits in the cache at position prefix + i, is rotated for position prefix + depth, and attends to the prefix, its ancestors and itself;
padding attends to nothing, has depth 0 and an attention output of zero.  Everything is dense and naive on purpose.
"""
import numpy as np

from . import head as _head
from . import layer as _layer

PAD = -2


def depths(parents):
    d = []
    for p in parents:
        d.append(d[p] + 1 if p >= 0 else 0)
    return np.array(d, dtype=np.int64)


def sees(parents):
    """[n][n] truth values: node i attends to node j."""
    n = len(parents)
    a = np.zeros((n, n), dtype=bool)
    for i in range(n):
        j = i
        while j >= 0 and parents[i] != PAD:
            a[i, j] = True
            j = parents[j]
    return a


def branch(parents, i):
    """Nodes from the prefix down to i."""
    out = []
    while i >= 0:
        out.append(i)
        i = parents[i]
    return out[::-1]


def norm_heads(u, gain, eps):
    """u [..][d]: every head on its own, u * gain / sqrt(mean(u^2) + eps)."""
    return u / np.sqrt(np.mean(u * u, axis=-1, keepdims=True) + u.dtype.type(eps)) * gain


def attention(q, k, v, prefix, parents):
    """q [n][n_q][d]; k, v [prefix + n][n_kv][d].  Returns (out [n][n_q][d], sum of the weights times |v|: what errors of the weights can do)."""
    n, n_q, d = q.shape
    group = n_q // k.shape[1]
    see = np.concatenate([np.repeat((np.asarray(parents) != PAD)[:, None], prefix, axis=1), sees(parents)], axis=1)
    out, spread = np.zeros_like(q), np.zeros_like(q)
    for i in range(n):
        at = np.flatnonzero(see[i])
        if not len(at):
            continue
        for h in range(n_q):
            s = k[at, h // group] @ q[i, h] / np.sqrt(d)
            w = np.exp(s - s.max())
            w /= w.sum()
            out[i, h] = w @ v[at, h // group]
            spread[i, h] = w @ np.abs(v[at, h // group])
    return out, spread


def apply_rules(logits, history, n_prompt, branch_tokens, repetition, frequency, presence, biases, allowed, dtype=np.float64):
    """One row [vocab].  history: token ids, the first n_prompt of them the prompt's; biases: (token, value) pairs, later ones replace earlier
    ones; allowed: truth values [vocab] or None.  Each operation is rounded to `dtype`."""
    f = dtype
    z = np.asarray(logits, dtype=f).copy()
    V = len(z)
    made = [t for t in list(history[n_prompt:]) + list(branch_tokens) if 0 <= t < V]
    seen = {t for t in history if 0 <= t < V} | set(made)
    for t in seen:
        z[t] = z[t] / f(repetition) if z[t] > 0 else z[t] * f(repetition)
    for t in set(made):
        z[t] = z[t] - f(f(frequency) * f(made.count(t)))
        z[t] = z[t] - f(presence)
    last = {}
    for t, b in biases:
        if 0 <= t < V:
            last[t] = b
    for t, b in last.items():
        z[t] = z[t] + f(b)
    if allowed is not None:
        z[~allowed] = -np.inf
    return z


def pick(z):
    """(index of the largest, the lowest among equal ones, or -1; its log-probability)."""
    ok = ~np.isnan(z)
    if not ok.any() or not np.max(z[ok]) > -np.inf:
        return -1, (np.nan if np.isnan(z).any() else -np.inf)
    best = np.max(z[ok])
    i = int(np.flatnonzero(z == best)[0])
    if np.isnan(z).any() or best == np.inf:
        return i, np.nan
    w = np.asarray(z, dtype=np.float64)
    return i, float(-np.log(np.sum(np.exp(w - best))))   # the maximum cancels: added and taken off again, a large one would swallow the logarithm


def verify(shape, head, layers, gains, seqs, parents, token_ids, pool, dtype=np.float32, bf16_activations=False):
    """Full-model step over trees.  seqs: layer.Seq; parents: one list a sequence; gains: per layer (g_q, g_k) or None; head, layers: float weights.
    Returns (logits [T][vocab], hidden [T][hidden]); keys and values are appended to the pool."""
    from . import bf16

    def stored(a):
        return bf16.round_trip(a.astype(np.float32)).astype(a.dtype) if bf16_activations else a

    nq, nkv, d = shape.n_q, shape.n_kv, shape.head_dim
    x = _head.embed(token_ids, head["embedding"].astype(dtype))
    T = len(x)
    pos = np.concatenate([s.kv_len - s.n_new + depths(p) for s, p in zip(seqs, parents)])
    for l, w in enumerate(layers):
        slot = l % pool.bits.shape[0]
        qkv = stored(_layer.rmsnorm(x, w["g_attn"].astype(dtype), shape.rms_eps)) @ w["w_qkv"].astype(dtype)
        q, k, v = (a.reshape(T, -1, d) for a in np.split(qkv, [nq * d, (nq + nkv) * d], axis=1))
        if gains[l] is not None:
            q, k = norm_heads(q, gains[l][0].astype(dtype), shape.rms_eps), norm_heads(k, gains[l][1].astype(dtype), shape.rms_eps)
        q, k = stored(_layer.rope(q, pos, shape.rope_base)), _layer.rope(k, pos, shape.rope_base)
        attn = np.zeros((T, nq, d), dtype=dtype)
        t0 = 0
        for s, par in zip(seqs, parents):
            t1 = t0 + s.n_new
            pool.write(slot, s.pages, s.kv_len - s.n_new, k[t0:t1].astype(np.float32), v[t0:t1].astype(np.float32))
            K, V = pool.gather(slot, s.pages, s.kv_len, dtype)
            attn[t0:t1] = attention(q[t0:t1], K, V, s.kv_len - s.n_new, par)[0]
            t0 = t1
        x1 = x + stored(attn).reshape(T, nq * d) @ w["w_o"].astype(dtype)
        xn2 = stored(_layer.rmsnorm(x1, w["g_ffn"].astype(dtype), shape.rms_eps))
        act = stored(_layer.silu(xn2 @ w["w_gate"].astype(dtype)) * (xn2 @ w["w_up"].astype(dtype)))
        x = x1 + act @ w["w_down"].astype(dtype)
    xn = stored(_layer.rmsnorm(x, head["g_final"].astype(dtype), shape.rms_eps))
    return xn @ head["w_out"].astype(dtype), x
