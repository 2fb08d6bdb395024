"""Oracle of tree verification and filtered sampling -- test infrastructure only.

Plain float64 statements of the calls for trees of drafts and of the sampler:
rotation by position, attention of a row to the context, its ancestors and
itself, the walk over the drawn tokens, and the tokens that temperature, top-k,
top-p and min-p leave.
"""

from __future__ import annotations

from typing import List, Optional, Tuple

import numpy as np

from .sampling import gumbel_noise, uniform_seed


def rotate(x: np.ndarray, angle: np.ndarray, interleaved: bool, amplitude: float = 1.0) -> np.ndarray:
    """Heads x [..., hd] turned by angle [pairs]: pairs (j, j + pairs), or (2 j,
    2 j + 1); the features behind 2 pairs stay."""
    y = np.asarray(x, np.float64).copy()
    n = len(angle)
    i, j = (np.arange(0, 2 * n, 2), np.arange(1, 2 * n, 2)) if interleaved else (np.arange(n), np.arange(n, 2 * n))
    c, s = amplitude * np.cos(angle), amplitude * np.sin(angle)
    a, b = y[..., i].copy(), y[..., j].copy()
    y[..., i], y[..., j] = a * c - b * s, b * c + a * s
    return y


def lineage(parents: List[int], i: int) -> List[int]:
    """Row i and its ancestors, the oldest first."""
    out = []
    while i >= 0:
        out.append(i)
        i = parents[i]
    return out[::-1]


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray, scale: float) -> np.ndarray:
    """softmax(scale q k^T) v of one head's query q [hd] over rows k, v [n, hd]."""
    z = scale * (np.asarray(k, np.float64) @ np.asarray(q, np.float64))
    p = np.exp(z - z.max())
    return (p / p.sum()) @ np.asarray(v, np.float64)


def walk(tokens, parents, nxt, rows: int) -> Tuple[int, List[int], int]:
    """(accepted, path, correction) of one request's tree."""
    if rows == 0:
        return -1, [], -1
    path = [0]
    while True:
        at = path[-1]
        child = [i for i in range(at + 1, rows) if parents[i] == at and tokens[i] == nxt[at]]
        if not child:
            return len(path) - 1, path, int(nxt[at])
        path.append(child[0])


def sample(logits: np.ndarray, u: float, temperature: float = 1.0, top_k: int = 0, top_p: float = 1.0,
           min_p: float = 0.0) -> Tuple[int, np.ndarray]:
    """(token, distribution [V]) of one row; the parameters as float32 holds them."""
    l = np.asarray(logits, np.float64).copy()
    l[np.isnan(l)] = -np.inf
    l = np.minimum(l, float(np.finfo(np.float32).max))
    V = len(l)
    p = np.zeros(V)
    if l.max() == -np.inf:
        return 0, p
    order = np.argsort(-l, kind="stable")
    if not temperature > 0:
        p[order[0]] = 1.0
        return int(order[0]), p
    t, top_p, min_p = (float(np.float32(x)) for x in (temperature, top_p, min_p))
    with np.errstate(invalid="ignore", over="ignore"):
        d = (l[order[0]] - l[order]) / t
    d[l[order] == -np.inf] = np.inf
    n = int((d <= 32.0).sum())
    if top_k > 0:
        n = min(n, top_k)
    w = np.exp(-d[:n])
    keep = n
    if top_p < 1:
        before = np.cumsum(w) - w
        keep = max(1, int((before < (top_p - 2.0 ** -40) * w.sum()).sum()))
    if min_p > 0:
        keep = min(keep, int((d[:n] <= -np.log(min(min_p, 1.0))).sum()))
    w = w[:keep] / w[:keep].sum()
    p[order[:keep]] = w
    score = np.full(V, -np.inf)
    score[order[:keep]] = -d[:keep] + gumbel_noise(uniform_seed(u), V)[order[:keep]]
    return int(np.argmax(score)), p


def depths(parents: Optional[List[int]], n: int) -> List[int]:
    return [i if parents is None else len(lineage(parents, i)) - 1 for i in range(n)]
