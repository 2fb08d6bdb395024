"""Float64 NumPy oracle of the 4-bit K/V cache: what a row is held as, head
norms and rotation, causal attention with the weights that positions receive,
eviction by accumulated weight.  Written from the definitions (include/spade.h),
one request and head at a time."""

from __future__ import annotations

import numpy as np

from .decoder import Decoder, apply_rope, rms_norm, rope_tables, silu


def bf16(x: np.ndarray) -> np.ndarray:
    """The bfloat16 nearest to the float32 nearest to x (ties to even), as float64."""
    f = np.asarray(x, dtype=np.float32)
    u = f.view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> np.uint64(16)) & np.uint64(1))) & np.uint64(0xFFFF0000)).astype(np.uint32)
    out = r.view(np.float32).astype(np.float64)
    return np.where(np.isnan(f), np.nan, out)


def codes(x: np.ndarray):
    """(n, s, m) of rows x [..., hd]; rows that are not finite, or whose span
    max - m is not: s = m = NaN."""
    x = np.asarray(x, dtype=np.float32).astype(np.float64)
    bad = ~np.isfinite(x).all(-1, keepdims=True)
    x = np.where(bad, 0.0, x)
    m = bf16(x.min(-1, keepdims=True))
    with np.errstate(over="ignore"):
        d = (x.max(-1, keepdims=True) - m).astype(np.float32)
    bad = bad | ~np.isfinite(d)
    d = np.where(bad, np.float32(0), np.maximum(d, np.float32(0)))
    m = np.where(bad, 0.0, m)
    s = bf16(d * np.float32(1 / 15))
    with np.errstate(divide="ignore", invalid="ignore"):
        n = np.where(s > 0, np.clip(np.rint((x - m) / np.where(s > 0, s, 1.0)), 0, 15), 0.0)
    return np.where(bad, 0.0, n), np.where(bad, np.nan, s), np.where(bad, np.nan, m)


def held(x: np.ndarray) -> np.ndarray:
    """Rows x as the cache holds them (float64)."""
    n, s, m = codes(x)
    return m + n * s


def norm_rotate(x: np.ndarray, gain, eps: float, angles) -> np.ndarray:
    """x [heads, hd]: RMSNorm over each head (gain or None), rotation of
    feature i with i + hd/2 by angles [hd/2, 2] (cosine, sine; or None)."""
    x = np.asarray(x, dtype=np.float64)
    if gain is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(gain, np.float64)
    if angles is not None:
        h = x.shape[-1] // 2
        c, s = np.asarray(angles, np.float64).T
        a, b = x[:, :h], x[:, h:]
        x = np.concatenate([a * c - b * s, b * c + a * s], -1)
    return x


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray, L: int, scale: float):
    """q [R, H, hd], k and v [>= L + R, KVH, hd] (what the cache holds).
    Returns (out [R, H, hd], p [R, H, L + R])."""
    R, H, hd = q.shape
    KVH = k.shape[1]
    G = H // KVH
    out = np.zeros((R, H, hd))
    p = np.zeros((R, H, L + R))
    for i in range(R):
        n = L + i + 1
        for h in range(H):
            z = k[:n, h // G] @ q[i, h].astype(np.float64) * scale
            e = np.exp(z - z.max())
            p[i, h, :n] = e / e.sum()
            out[i, h] = p[i, h, :n] @ v[:n, h // G]
    return out, p


def keep(weights: np.ndarray, n: int, budget: int, recent: int) -> np.ndarray:
    """Kept positions (ascending) of n cached ones with these weights: the
    last `recent` and the heaviest others, ties to the lower position, NaN
    heavier than any number."""
    if n <= budget:
        return np.arange(n)
    w = weights[:n - recent].astype(np.float64)
    rank = np.where(np.isnan(w), np.inf, w)
    # NaN before +inf, then by weight, then by position
    order = np.lexsort((np.arange(len(w)), -rank, ~np.isnan(w)))
    old = np.sort(order[:budget - recent])
    return np.concatenate([old, np.arange(n - recent, n)])


class QuantDecoder(Decoder):
    """The verifier over 4-bit caches, with the head norms where gains are
    given.  A cache may have lost positions: ``shift`` of them (an attribute
    set on the cache) come before its rows, which only moves the angles.
    ``weights`` [layer][KV head, capacity], where set on the cache, gets the
    probabilities of the first ``count`` rows of every call (count None: all)."""

    def __init__(self, shape, get, gain_q=None, gain_k=None, eps: float = 1e-5, keep_f64: bool = False):
        super().__init__(shape, get, keep_f64)
        self.gain_q, self.gain_k, self.eps = gain_q, gain_k, eps
        self.count = None

    def stored(self, l, cache, k, v):
        """The rows [R, KV heads, hd] as the cache holds them."""
        return held(k), held(v)

    def block(self, l, W, cache, x):
        s = self.shape
        R, L, H, hd, KVH = x.shape[0], cache.length, s.n_heads, s.head_dim, s.kv_heads
        h = rms_norm(x, W("g_attn"), s.rms_eps)
        q, k, v = ((h @ W(n).T).reshape(R, m, hd) for n, m in (("wq", H), ("wk", KVH), ("wv", KVH)))
        cos, sin = rope_tables(np.arange(L, L + R) + getattr(cache, "shift", 0), hd, s.rope_theta)
        if self.gain_q is not None:
            q = q / np.sqrt((q * q).mean(-1, keepdims=True) + self.eps) * self.gain_q[l]
            k = k / np.sqrt((k * k).mean(-1, keepdims=True) + self.eps) * self.gain_k[l]
        q, k = apply_rope(q, cos, sin), apply_rope(k, cos, sin)
        kk, vv = self.stored(l, cache, k, v)
        cache.k[l][:, L:L + R] = kk.transpose(1, 0, 2)
        cache.v[l][:, L:L + R] = vv.transpose(1, 0, 2)
        o, p = attend(q, cache.k[l][:, :L + R].transpose(1, 0, 2).astype(np.float64),
                      cache.v[l][:, :L + R].transpose(1, 0, 2).astype(np.float64), L, 1.0 / np.sqrt(hd))
        if getattr(cache, "weights", None) is not None:
            w = cache.weights[l]
            w[:, L:L + R] = 0
            w[:, :L + R] += p[:R if self.count is None else self.count].reshape(-1, KVH, H // KVH, L + R).sum((0, 2))
        x = x + o.reshape(R, H * hd) @ W("wo").T
        h = rms_norm(x, W("g_ffn"), s.rms_eps)
        return x + (silu(h @ W("wg").T) * (h @ W("wu").T)) @ W("wd").T
