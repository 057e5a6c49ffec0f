"""A KV cache in 8 bits, stated in float64: what its blocks stand for, attention over it, the accumulated weights, eviction.

Tokens are arrays [n, heads, d] (or [n, d]); a block is 16 consecutive tokens of one head, K and V apart."""
import numpy as np

from . import layer_math as lm

BLOCK = 16


def quantise(block, fp32=False):
    """[16, d] values -> (whole numbers, largest magnitude).  `fp32`: the quotient is formed in 32 bits, as the definition has it
    for the evictions of fp32 models."""
    t = np.float32 if fp32 else np.float64
    b = np.asarray(block, dtype=t)
    if not np.all(np.isfinite(b)):
        return np.zeros(b.shape), np.nan
    a = np.max(np.abs(b))
    if a == 0:
        return np.zeros(b.shape), 0.0
    f = t(2.0 ** -8) if a > 1e36 else t(1)          # 127 times the value stays below the largest 32-bit number
    return np.rint(b * f * t(127) / (a * f)).astype(np.float64), float(a)


def units_head(x, fp32=False):
    """[n, d] of one head: 127 times what a cache of these tokens stands for: q * A in full blocks, 127 times the value in the open
    one.  Exact for values of up to 24 bits, so that a value on half a step of another block is seen to be there; `fp32`: rounded
    to 32 bits."""
    x = np.asarray(x, dtype=np.float64)
    u = x * 127
    for b in range(0, x.shape[0] // BLOCK * BLOCK, BLOCK):
        q, a = quantise(x[b:b + BLOCK])
        u[b:b + BLOCK] = q * a
    return u.astype(np.float32).astype(np.float64) if fp32 else u


def units(x, fp32=False):
    """The same for [n, heads, d]."""
    x = np.asarray(x, dtype=np.float64)
    return np.stack([units_head(x[:, g], fp32) for g in range(x.shape[1])], axis=1)


def held_head(x, fp32=False):
    x = np.array(x, dtype=np.float64)
    for b in range(0, x.shape[0] // BLOCK * BLOCK, BLOCK):
        q, a = quantise(x[b:b + BLOCK], fp32)
        x[b:b + BLOCK] = q * a / 127
    return x


def held(x, fp32=False):
    """What a cache of the tokens [n, heads, d] stands for."""
    x = np.asarray(x, dtype=np.float64)
    return np.stack([held_head(x[:, g], fp32) for g in range(x.shape[1])], axis=1)


def attention(q, k, v, first):
    """Causal attention of q [n, n_q, d], at cached positions first .. first + n - 1, over k, v [L, n_kv, d].  Returns the output, the
    same sum with the magnitudes of v (what rounded weights can move it by) and the weights [n, n_q, L]."""
    n, n_q, d = q.shape
    group = n_q // k.shape[1]
    out, mag, wts = np.zeros(q.shape), np.zeros(q.shape), np.zeros((n, n_q, k.shape[0]))
    hidden = np.arange(k.shape[0])[None, :] > first + np.arange(n)[:, None]
    for a in range(n_q):
        g = a // group
        s = np.where(hidden, -np.inf, q[:, a] @ k[:, g].T / np.sqrt(float(d)))
        wts[:, a] = lm.softmax_rows(s)
        out[:, a] = wts[:, a] @ v[:, g]
        mag[:, a] = wts[:, a] @ np.abs(v[:, g])
    return out, mag, wts


def kept_positions(w, keep, recent):
    """Positions of one head that stay, ascending: the newest `recent`, and of the others those of greatest weight, the earlier of
    equal ones.  NaN is greater than anything."""
    n = len(w)
    if n <= keep:
        return np.arange(n)
    recent = min(recent, keep)
    old = n - recent
    key = np.where(np.isnan(w[:old]), np.inf, w[:old])
    order = sorted(range(old), key=lambda i: (-int(np.isnan(w[i])), -key[i], i))
    return np.array(sorted(order[:keep - recent]) + list(range(old, n)))


def evict(k, v, w, keep, recent, store=lambda x: x, fp32=False):
    """k, v: units() of the cache, [n, heads, d]; w [heads, n].  Returns what the cut cache stands for and its weights; `store` rounds
    what ends in the open block to the model's type."""
    heads = k.shape[1]
    pos = [kept_positions(w[g], keep, recent) for g in range(heads)]
    if k.shape[0] <= keep:
        return k / 127, v / 127, w
    out = []
    for x in (k, v):
        y = np.stack([x[pos[g], g] for g in range(heads)], axis=1)
        full = keep // BLOCK * BLOCK
        out.append(np.concatenate([held(y[:full], fp32) / 127 if full else y[:0], store(y[full:] / 127)]))
    return out[0], out[1], np.stack([w[g][pos[g]] for g in range(heads)])


class LayerCache:
    """Keys and values of a layer, per sequence, as they came; read as the cache stands for them."""

    def __init__(self):
        self.data = {}

    def append(self, seq, before, k, v):
        old = self.data.get(seq)
        if old is not None and before:
            k, v = np.concatenate([old[0][:before], k]), np.concatenate([old[1][:before], v])
        self.data[seq] = (k, v)

    def read(self, seq):
        return tuple(held(x) for x in self.data[seq])


def attn_block(cfg, w, x, batch, cache, k=1, i=0, round_kv=None):
    """layer_math.attn_block over a cache in 8 bits (LayerCache of the shard)."""
    (q0, q1), (g0, g1), _ = lm.shard_ranges(cfg, k, i)
    d, T = cfg.head_dim, np.shape(x)[0]
    pos, spans = lm.batch_positions(batch)
    h = lm.rmsnorm(np.asarray(x, dtype=np.float64), w["g1"], cfg.rms_eps)
    q = lm.rope((h @ w["wq"][:, q0 * d:q1 * d]).reshape(T, q1 - q0, d), pos, cfg.rope_base)
    kk = lm.rope((h @ w["wk"][:, g0 * d:g1 * d]).reshape(T, g1 - g0, d), pos, cfg.rope_base)
    v = (h @ w["wv"][:, g0 * d:g1 * d]).reshape(T, g1 - g0, d)
    if round_kv is not None:
        kk, v = round_kv(kk), round_kv(v)
    out = np.zeros((T, q1 - q0, d))
    for (seq, _, before), (t0, t1) in zip(batch, spans):
        cache.append(seq, before, kk[t0:t1], v[t0:t1])
        out[t0:t1] = attention(q[t0:t1], *cache.read(seq), before)[0]
    return out.reshape(T, (q1 - q0) * d) @ w["wo"][q0 * d:q1 * d, :]
