"""The operators of tree verification, as measurable cases.

A verifier that scores a tree of drafts instead of a chain appends every node's
row to the cache at its depth's position, lets it attend to the context and to
its own ancestors, draws every node's next token and keeps the path whose tokens
were drawn (``paper_2608_13076_amd.tree`` and ``.sampling``):

``append``  new rows of a layer: queries and keys rotated by their position
            (halves of the head or neighbours paired, the whole head or a part
            of it, frequencies scaled for long contexts), keys and values into
            the bfloat16 cache.  A pass also reads the new rows back.
``attend``  attention of the rows of a tree over the cache: a row sees the
            context, its ancestors and itself.
``sample``  a token per row of logits: temperature, top-k, top-p and min-p, drawn
            from a given uniform, and its probability; where asked, the whole
            filtered distribution.
``commit``  the walk from the root over the drawn tokens, the rows of its path
            closed up behind the context; the pass reads the rows back.

Head layouts are the ones of ``synth.configs`` (32 or 40 heads of 128 features,
32 query heads over 8 K/V heads, 4 heads of 64; vocabularies of 4096, 32000 and
128256 tokens) and generic small ones.
"""

import math
import random
from types import SimpleNamespace

import torch

own = False

DEV = "cuda:0"
_T = {"f32": torch.float32, "bf16": torch.bfloat16}


def _append(b, r, h, kvh, hd, dtype, lo, hi, rot, interleaved, scaling, chain, ragged, lens_seed=0, name=None):
    """lo..hi: cached positions of a request before its r new rows (of which a
    ragged batch uses 0..r); rot: rotated features of a head; chain: a prompt's
    rows (depth i) instead of a tree's."""
    c = {"op": "append", "b": b, "r": r, "h": h, "kvh": kvh, "hd": hd, "dtype": dtype, "lo": lo, "hi": hi, "rot": rot,
         "interleaved": interleaved, "scaling": scaling, "chain": chain, "ragged": ragged, "lens_seed": lens_seed}
    return {"name": name, **c} if name else c


def _attend(b, r, h, kvh, hd, dtype, lo, hi, ragged, lens_seed=0, name=None):
    """lo..hi: cached positions of a request before the r rows of its tree."""
    c = {"op": "attend", "b": b, "r": r, "h": h, "kvh": kvh, "hd": hd, "dtype": dtype, "lo": lo, "hi": hi,
         "ragged": ragged, "lens_seed": lens_seed}
    return {"name": name, **c} if name else c


def _sample(n, t, vocab, dtype, mix, probs, seed=0, name=None):
    """n requests of t rows; mix: how the requests sample ("filters": all
    filtered, "plain": temperature alone, "mixed": greedy ones among them)."""
    c = {"op": "sample", "n": n, "t": t, "vocab": vocab, "dtype": dtype, "mix": mix, "probs": probs, "lens_seed": seed}
    return {"name": name, **c} if name else c


def _commit(layers, b, r, kvh, hd, lo, hi, ragged, lens_seed=0, name=None):
    c = {"op": "commit", "layers": layers, "b": b, "r": r, "kvh": kvh, "hd": hd, "lo": lo, "hi": hi, "ragged": ragged,
         "lens_seed": lens_seed}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one decoded token of one request, grouped heads: the smallest append
        _append(1, 1, 32, 8, 128, "bf16", 1024, 1024, 128, False, "none", True, False, name="append_token_gqa"),
        # trees of a full batch, float32 projections, neighbours paired, half of the head rotated
        _append(16, 25, 32, 8, 128, "f32", 256, 4096, 64, True, "linear", False, True, 1, name="append_trees_b16"),
        # a long piece of a prompt of a multi-head model, frequencies stretched by a ramp, odd lengths
        _append(1, 4003, 32, 32, 128, "bf16", 30001, 30001, 128, False, "ramp", True, False, name="append_prompt_4k"),
        # the smallest call: a few drafts behind a short prompt
        _attend(1, 5, 32, 8, 128, "bf16", 129, 129, False, name="attend_short"),
        # one request of a multi-head model, float32 rows
        _attend(1, 26, 32, 32, 128, "f32", 1024, 1024, False, 2, name="attend_tree_b1"),
        # a batched verify of a grouped-query model, ragged contexts and trees
        _attend(16, 32, 32, 8, 128, "bf16", 256, 4096, True, 3, name="attend_trees_b16_gqa"),
        # the widest tree over a very long context
        _attend(1, 64, 32, 8, 128, "bf16", 120001, 120001, False, 4, name="attend_tree_120k"),
        # the edge's next draft: one row of a large vocabulary, filtered
        _sample(1, 1, 128256, "f32", "filters", False, 5, name="sample_token_128k"),
        # drafts of a batch with the distributions that a later acceptance needs
        _sample(16, 1, 32000, "f32", "mixed", True, 6, name="sample_drafts_b16"),
        # every node of a batch's trees, logits as the head's matrix product leaves them
        _sample(16, 25, 128256, "bf16", "mixed", False, 7, name="sample_trees_b16"),
        # one layer of one request
        _commit(1, 1, 8, 8, 128, 1000, 1000, False, 8, name="commit_b1"),
        # eight layers of a full batch
        _commit(8, 16, 32, 8, 128, 256, 4000, True, 9, name="commit_b16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = [(8, 4, 128), (32, 1, 128), (40, 1, 128), (4, 1, 64), (4, 3, 64), (8, 2, 128), (2, 8, 128), (1, 6, 64), (5, 1, 128)]


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "sample", "sample", "commit"])
    kvh, g, hd = rng.choice(_HEADS)
    dtype = rng.choice(["f32", "bf16"])
    seed = rng.randrange(1 << 20)
    if op == "append":
        chain = rng.random() < 0.5
        b = _log(rng, 1, 16)
        r = _log(rng, 1, max(1, 2000 // b)) if chain else _log(rng, 1, 64)
        r = max(1, min(r, 4000 * 96 // (b * kvh * (g + 2) * 2)))
        lo = rng.randrange(0, 200)
        rot = rng.choice([hd, hd, hd // 2, hd // 4, hd - 8])
        return _append(b, r, kvh * g, kvh, hd, dtype, lo, lo + _log(rng, 1, 30000), rot, rng.random() < 0.5,
                       rng.choice(["none", "linear", "base", "ramp"]), chain, rng.random() < 0.5, seed)
    if op == "attend":
        b = _log(rng, 1, 16)
        r = rng.choice([1, _log(rng, 2, 64), _log(rng, 2, 64)])
        # the largest listed case: 64 rows of 32 heads over 120 thousand positions
        hi = _log(rng, 1, min(120000, 64 * 32 * 120000 // (b * r * kvh * g * 2), 16 * 8 * 16000 // (b * kvh)))
        lo = rng.choice([hi, max(0, hi // 8), 0])
        return _attend(b, r, kvh * g, kvh, hd, dtype, lo, hi, rng.random() < 0.5, seed)
    if op == "sample":
        vocab = rng.choice([4096, 32000, 128256, _log(rng, 2, 200000)])
        n = _log(rng, 1, 16)
        t = _log(rng, 1, max(1, min(32, 16 * 25 * 128256 // (2 * n * vocab))))
        probs = rng.random() < 0.5 and n * t * vocab < 8000000
        return _sample(n, t, vocab, dtype, rng.choice(["filters", "plain", "mixed"]), probs, seed)
    layers, b = rng.randrange(1, 9), _log(rng, 1, 16)
    r = _log(rng, 1, 64)
    r = max(1, min(r, 8 * 16 * 32 * 8 // (layers * b * kvh)))
    return _commit(layers, b, r, kvh, hd, 0, _log(rng, 1, 4000), rng.random() < 0.5, seed)


def _counts(case):
    """Cached positions of every request and how many of its rows are in use."""
    rng = random.Random(1000 + case["lens_seed"])
    lens = [rng.randint(case["lo"], case["hi"]) for _ in range(case["b"])]
    r = case["r"]
    rows = [rng.randint(0, r) if case["ragged"] else r for _ in lens]
    if not any(rows):
        rows[0] = r
    return lens, rows


def _trees(case, rows):
    """Parents [b][r] (-1: none), every node's parent before it: a root with a
    few branches, most nodes hanging from recent ones."""
    rng = random.Random(2000 + case["lens_seed"])
    out = []
    for _ in rows:
        p = [-1]
        for i in range(1, case["r"]):
            p.append(max(0, i - 1 - int(rng.expovariate(0.25))))
        out.append(p)
    return out


def _depths(parents):
    out = []
    for p in parents:
        d = []
        for i, a in enumerate(p):
            d.append(0 if a < 0 else d[a] + 1)
        out.append(d)
    return out


def _history(gen, n, kvh, hd):
    """Keys or values of n positions: a few strong features per head, as the
    keys of trained models have, and a drift along the positions."""
    x = torch.randn(n, kvh, hd, generator=gen, device=DEV)
    x[:, :, ::17] *= 4.0
    return (x + 0.3 * torch.randn(1, kvh, hd, generator=gen, device=DEV)).to(torch.bfloat16)


def _frequencies(rot, scaling):
    """Angle per position of every pair, in double, and the factor of the
    rotated features."""
    n = rot // 2
    base, factor = 500000.0, 8.0
    i = torch.arange(n, dtype=torch.float64, device=DEV)
    if scaling == "base":
        base *= factor ** (rot / max(rot - 2, 1))
    f = base ** (-2.0 * i / rot)
    if scaling == "linear":
        f = f / factor
    if scaling == "ramp":
        # frequencies of more than 32 turns in 8192 positions stay, those of less than one are divided
        turns = 8192.0 * f / (2.0 * math.pi)
        keep = ((turns - 1.0) / 31.0).clamp(0.0, 1.0)
        return f * keep + f / factor * (1.0 - keep), 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _requests(case):
    """Temperature, top-k, top-p and min-p of every request, as lists."""
    rng = random.Random(3000 + case["lens_seed"])
    cols = [[], [], [], []]
    for _ in range(case["n"]):
        t, k, p, m = rng.uniform(0.5, 1.3), 0, 1.0, 0.0
        if case["mix"] != "plain":
            kind = rng.choice(["k", "p", "m", "kp", "kpm"])
            k = _log(rng, 1, 200) if "k" in kind else 0
            p = rng.uniform(0.6, 0.98) if "p" in kind else 1.0
            m = rng.uniform(0.01, 0.15) if "m" in kind else 0.0
        if case["mix"] == "mixed":
            kind = rng.random()
            if kind < 0.25:
                t = 0.0
            elif kind < 0.4:
                k, p, m = 0, 1.0, 0.0
        for c, x in zip(cols, (t, k, p, m)):
            c.append(x)
    return cols


def _inputs(case, seed):
    """The case's inputs, the same for either form."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = SimpleNamespace(case=case)
    if case["op"] == "sample":
        n, t, vocab = case["n"], case["t"], case["vocab"]
        rows = n * t
        # logits of a trained head: a broad floor and a few likely tokens, fewer in confident rows
        z = torch.randn(rows, vocab, generator=gen, device=DEV) * 2.0
        top = torch.randint(0, vocab, (rows, 24), generator=gen, device=DEV)
        z.scatter_add_(1, top, torch.rand(rows, 24, generator=gen, device=DEV) * 10.0 + 2.0)
        s.logits = z.to(_T[case["dtype"]])
        s.u = torch.rand(rows, generator=gen, device=DEV)
        t_, k_, p_, m_ = _requests(case)
        s.temperature = torch.tensor(t_, dtype=torch.float32, device=DEV)
        s.top_k = torch.tensor(k_, dtype=torch.int32, device=DEV)
        s.top_p = torch.tensor(p_, dtype=torch.float32, device=DEV)
        s.min_p = torch.tensor(m_, dtype=torch.float32, device=DEV)
        return s
    lens, rows = _counts(case)
    s.lens, s.rows = lens, rows
    b, r, kvh, hd = case["b"], case["r"], case["kvh"], case["hd"]
    s.d_lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s.d_rows = torch.tensor(rows, dtype=torch.int32, device=DEV)
    if case["op"] == "append":
        h = case["h"]
        # the output of a fused projection: queries, keys and values of a row
        x = torch.randn(b, r, h + 2 * kvh, hd, generator=gen, device=DEV)
        x[:, :, :, 3::29] *= 5.0
        s.qkv = x.to(_T[case["dtype"]])
        s.q, s.k, s.v = s.qkv[:, :, :h], s.qkv[:, :, h:h + kvh], s.qkv[:, :, h + kvh:]
        s.freq, s.amplitude = _frequencies(case["rot"], case["scaling"])
        s.depth = None
        if not case["chain"]:
            s.depth = torch.tensor(_depths(_trees(case, rows)), dtype=torch.int32, device=DEV)
        return s
    s.parents = _trees(case, rows)
    s.d_parents = torch.tensor(s.parents, dtype=torch.int32, device=DEV)
    if case["op"] == "attend":
        s.q = (1.5 * torch.randn(b, r, case["h"], hd, generator=gen, device=DEV)).to(_T[case["dtype"]])
        s.hist = [(_history(gen, n + m, kvh, hd), _history(gen, n + m, kvh, hd)) for n, m in zip(lens, rows)]
        return s
    rng = random.Random(seed)
    s.tokens = torch.randint(0, 32000, (b, r), generator=gen, device=DEV).to(torch.int32)
    tok = s.tokens.tolist()
    nxt = torch.randint(32000, 64000, (b, r), generator=gen, device=DEV).to(torch.int32).tolist()
    for p, m, x, y in zip(s.parents, rows, tok, nxt):
        # a path that the drawn tokens follow.  Its rows stay where they are or come from behind its
        # end, so a pass can be repeated on what the last one left
        for end in rng.sample(range(m), m) if m else []:
            path = [end]
            while path[-1]:
                path.append(p[path[-1]])
            path.reverse()
            if all(a == j or a >= len(path) for j, a in enumerate(path)):
                for a, c in zip(path, path[1:]):
                    y[a] = x[c]
                break
    s.next = torch.tensor(nxt, dtype=torch.int32, device=DEV)
    s.hist = [[(_history(gen, m, kvh, hd), _history(gen, m, kvh, hd)) for m in rows] for _ in range(case["layers"])]
    return s


# --- the plain form -------------------------------------------------------


def _rotate(x, angle, amplitude, interleaved):
    """x [rows, heads, hd] in 32 bits; angle [rows, pairs] in 64: the first
    2 pairs features turned, the others as they are."""
    x = x.float()
    n = angle.shape[-1]
    c, sn = (torch.cos(angle) * amplitude).float()[:, None], (torch.sin(angle) * amplitude).float()[:, None]
    if interleaved:
        a, b = x[..., 0:2 * n:2], x[..., 1:2 * n:2]
        y = torch.stack([a * c - b * sn, b * c + a * sn], -1).flatten(-2)
    else:
        a, b = x[..., :n], x[..., n:2 * n]
        y = torch.cat([a * c - b * sn, b * c + a * sn], -1)
    return torch.cat([y, x[..., 2 * n:]], -1)


def _plain_append(s):
    case, b, r = s.case, s.case["b"], s.case["r"]
    depth = s.depth if s.depth is not None else torch.arange(r, device=DEV).expand(b, r)
    at = (s.d_lens[:, None] + depth).reshape(-1).double()
    unused = (torch.arange(r, device=DEV)[None] >= s.d_rows[:, None]).reshape(-1)[:, None, None]
    angle = at[:, None] * s.freq[None]
    flat = [x.reshape(b * r, x.shape[2], x.shape[3]) for x in (s.q, s.k, s.v)]
    q = _rotate(flat[0], angle, s.amplitude, case["interleaved"])
    k = _rotate(flat[1], angle, s.amplitude, case["interleaved"])
    out = {}
    for name, x, t, like in (("q", q, s.q.dtype, s.q), ("k", k, torch.bfloat16, s.k), ("v", flat[2], torch.bfloat16, s.v)):
        out[name] = x.masked_fill(unused, 0.0).to(t).reshape(like.shape)
    return out


def _plain_attend(s):
    case = s.case
    b, r, h, kvh, hd = (case[x] for x in ("b", "r", "h", "kvh", "hd"))
    g = h // kvh
    out = torch.zeros(b, r, h, hd, dtype=s.q.dtype, device=DEV)
    for i, (n, m) in enumerate(zip(s.lens, s.rows)):
        if m == 0:
            continue
        # a row sees what its parent sees, and itself
        sees = torch.zeros(m, m, dtype=torch.bool, device=DEV)
        parent = s.d_parents[i, :m].long()
        at = torch.arange(m, device=DEV)
        while bool((at >= 0).any()):
            live = (at >= 0).nonzero()[:, 0]
            sees[live, at[live]] = True
            at = torch.where(at >= 0, parent[at.clamp_min(0)], at)
        hidden = torch.cat([torch.zeros(m, n, dtype=torch.bool, device=DEV), ~sees], 1)
        k = s.hist[i][0].float().transpose(0, 1)  # [kvh, n + m, hd]
        v = s.hist[i][1].float().transpose(0, 1)
        q = s.q[i, :m].float().reshape(m, kvh, g, hd).permute(1, 2, 0, 3).reshape(kvh, g * m, hd)
        z = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(hd)
        z = z.masked_fill(hidden.repeat(g, 1)[None], -math.inf)
        z = torch.exp(z - z.amax(-1, keepdim=True))
        o = torch.matmul(z, v.contiguous()) / z.sum(-1, keepdim=True)
        out[i, :m] = o.reshape(kvh, g, m, hd).permute(2, 0, 1, 3).reshape(m, h, hd).to(out.dtype)
    return {"out": out}


def _s64(x):
    return x - (1 << 64) if x >= 1 << 63 else x


def _noise(u, vocab):
    """Gumbel noise [rows, vocab] of the streams that the uniforms' bits seed:
    -log(-log U), U from output v of SplitMix64."""
    def shift(z, n):
        return (z >> n) & ((1 << (64 - n)) - 1)
    v = torch.arange(1, vocab + 1, dtype=torch.int64, device=DEV)
    z = u.view(torch.int32).long()[:, None] + (v * _s64(0x9E3779B97F4A7C15))[None]
    z = (z ^ shift(z, 30)) * _s64(0xBF58476D1CE4E5B9)
    z = (z ^ shift(z, 27)) * _s64(0x94D049BB133111EB)
    z = z ^ shift(z, 31)
    return -torch.log(-torch.log((shift(z, 41).double() + 0.5) * 2.0 ** -23))


def _lowest_max(x):
    """The lowest index of every row's largest value."""
    v = x.shape[-1]
    at = torch.arange(v, device=DEV)[None].expand_as(x)
    return at.masked_fill(x < x.amax(-1, keepdim=True), v).amin(-1).to(torch.int32)


def _plain_sample(s):
    case = s.case
    vocab, per = case["vocab"], case["t"]
    out = torch.empty(case["n"] * per, dtype=torch.int32, device=DEV)
    chosen = torch.empty(case["n"] * per, device=DEV)
    probs = torch.empty(case["n"] * per, vocab, device=DEV) if case["probs"] else None
    for i in range(case["n"]):
        rows = slice(i * per, (i + 1) * per)
        z = s.logits[rows].float()
        t = s.temperature[i].double()
        best = _lowest_max(z)
        d = z.double() - z.double().amax(-1, keepdim=True)
        d = d / torch.where(t > 0, t, torch.ones_like(t))
        w = torch.exp(d)
        ordered, order = torch.sort(z, dim=-1, descending=True, stable=True)
        w_sorted = torch.gather(w, 1, order)
        rank = torch.arange(vocab, device=DEV)[None]
        k = torch.where(s.top_k[i] > 0, s.top_k[i], vocab)
        w_sorted = w_sorted.masked_fill((rank >= k) | (w_sorted < math.exp(-32.0)), 0.0)
        before = torch.cumsum(w_sorted, -1) - w_sorted
        p = s.top_p[i].double()
        full = before < (p - 2.0 ** -40) * w_sorted.sum(-1, keepdim=True)
        keep = (w_sorted > 0) & ((p >= 1) | full | (rank == 0)) & (w_sorted >= s.min_p[i].double().clamp_max(1.0))
        keep = torch.zeros_like(keep).scatter_(1, order, keep)
        score = (d + _noise(s.u[rows], vocab)).masked_fill(~keep, -math.inf)
        out[rows] = torch.where(t > 0, _lowest_max(score), best)
        w = w.masked_fill(~keep, 0.0)
        w = w / w.sum(-1, keepdim=True)
        one = torch.ones_like(w[:, 0])
        chosen[rows] = torch.where(t > 0, torch.gather(w, 1, out[rows].long()[:, None])[:, 0], one).float()
        if probs is not None:
            greedy = torch.zeros_like(w).scatter_(1, best.long()[:, None], 1.0)
            probs[rows] = torch.where(t > 0, w, greedy).float()
    return {"tokens": out, "chosen": chosen, **({"probs": probs} if probs is not None else {})}


def _plain_commit(s):
    case = s.case
    b, r, layers = case["b"], case["r"], case["layers"]
    cur = torch.zeros(b, dtype=torch.long, device=DEV)
    live = s.d_rows > 0
    count = live.long()
    path = torch.full((b, r), -1, dtype=torch.int32, device=DEV)
    path[:, 0] = torch.where(live, 0, -1)
    at = torch.arange(r, device=DEV)[None]
    corr = torch.where(live, s.next[:, 0], -1)
    for j in range(1, r):
        nxt = torch.gather(s.next, 1, cur[:, None])
        ok = (s.d_parents == cur[:, None]) & (s.tokens == nxt) & (at > cur[:, None]) & (at < s.d_rows[:, None])
        child = torch.where(ok, at, r).amin(-1)
        live = live & (child < r)
        cur = torch.where(live, child, cur)
        path[:, j] = torch.where(live, cur.to(torch.int32), -1)
        count = count + live.long()
        corr = torch.where(live, torch.gather(s.next, 1, cur[:, None])[:, 0], corr)
    out = {"n": (count - 1).to(torch.int32), "path": path, "correction": corr, "lens": s.d_lens + count.to(torch.int32)}
    # position j of the kept rows is the path's row j, those behind stay
    src = torch.where(path >= 0, path.long(), at)
    for l in range(layers):
        for x, name in ((0, "k"), (1, "v")):
            out[f"{name}{l}"] = torch.gather(s.pad[l][x], 1, src[:, :, None, None].expand_as(s.pad[l][x]))
    return out


# --- the framework's operators --------------------------------------------


def _padded(hist, n):
    """Rows of every request side by side, zeros behind the last."""
    pad = [torch.zeros((len(hist), n) + tuple(hist[0][j].shape[1:]), dtype=torch.bfloat16, device=DEV) for j in (0, 1)]
    for i, kv in enumerate(hist):
        for j in (0, 1):
            pad[j][i, :len(kv[j])] = kv[j]
    return pad


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        if case["op"] == "commit":
            s.pad = [_padded(x, case["r"]) for x in s.hist]
            s.hist = None
        return s
    from paper_2608_13076_amd import sampling, tree
    if case["op"] == "sample":
        s.sampler = sampling.Sampler(case["n"] * case["t"], case["vocab"], device=DEV)
        s.probs = torch.empty(case["n"] * case["t"], case["vocab"], device=DEV) if case["probs"] else None
        return s
    b, r, kvh, hd = case["b"], case["r"], case["kvh"], case["hd"]
    cap = max(s.lens) + r
    if case["op"] == "append":
        s.cache = tree.TreeCache(1, b, case["h"], kvh, hd, cap, max_rows=1, device=DEV)
        s.cache.lens.copy_(s.d_lens)
        s.rope = tree.Rotary(s.freq, interleaved=case["interleaved"], amplitude=s.amplitude)
    elif case["op"] == "attend":
        s.cache = tree.TreeCache(1, b, case["h"], kvh, hd, cap, max_rows=r, device=DEV)
        pad = _padded(s.hist, max(len(x[0]) for x in s.hist))
        s.cache.append(0, pad[0], pad[1], rows=s.d_lens + s.d_rows)
        s.cache.lens.copy_(s.d_lens)
        s.max_keys = max(n + m for n, m in zip(s.lens, s.rows))
    else:
        s.cache = tree.TreeCache(case["layers"], b, kvh, kvh, hd, cap, max_rows=1, device=DEV)
        s.cache.lens.copy_(s.d_lens)
        for l in range(case["layers"]):
            pad = _padded(s.hist[l], r)
            # (every row of the batch, so that those behind a request's last hold zeros too)
            s.cache.append(l, pad[0], pad[1])
        s.lens_out = torch.empty_like(s.d_lens)
    s.hist = None
    return s


def run(s):
    case = s.case
    if not own:
        return {"append": _plain_append, "attend": _plain_attend, "sample": _plain_sample,
                "commit": _plain_commit}[case["op"]](s)
    if case["op"] == "append":
        q = s.cache.append(0, s.k, s.v, q=s.q, rope=s.rope, depth=s.depth, rows=s.d_rows)
        k, v = s.cache.read(0, case["r"], start=s.d_lens, rows=s.d_rows)
        return {"q": q, "k": k, "v": v}
    if case["op"] == "attend":
        return {"out": s.cache.attend(0, s.q, parents=s.d_parents, rows=s.d_rows, max_keys=s.max_keys)}
    if case["op"] == "sample":
        tokens, chosen = s.sampler.draw(s.logits, s.u, temperature=s.temperature, top_k=s.top_k, top_p=s.top_p,
                                        min_p=s.min_p, probs=s.probs)
        return {"tokens": tokens, "chosen": chosen, **({"probs": s.probs} if s.probs is not None else {})}
    n, path, corr = s.cache.commit(s.tokens, s.d_parents, s.next, rows=s.d_rows, lens_out=s.lens_out)
    out = {"n": n, "path": path, "correction": corr, "lens": s.lens_out}
    for l in range(case["layers"]):
        out[f"k{l}"], out[f"v{l}"] = s.cache.read(l, case["r"], start=s.d_lens)
    return out


# --- what a pass cannot do without ----------------------------------------


def work(case):
    if case["op"] == "sample":
        rows, vocab = case["n"] * case["t"], case["vocab"]
        by = rows * vocab * ((4 if case["dtype"] == "f32" else 2) + (4 if case["probs"] else 0)) + rows * 12
        return {"bytes": by, "flops": rows * vocab * 4}
    lens, rows = _counts(case)
    kvh, hd, n = case["kvh"], case["hd"], sum(rows)
    row = 4 * kvh * hd  # a position's keys and values in bfloat16
    e = 4 if case.get("dtype") == "f32" else 2
    if case["op"] == "append":
        h, all_rows = case["h"], case["b"] * case["r"]
        by = n * ((h + 2 * kvh) * hd * e + 2 * row) + all_rows * (h * hd * e + row)
        return {"bytes": by, "flops": n * (h + kvh) * case["rot"] * 3}
    if case["op"] == "attend":
        h = case["h"]
        by = sum((a + m) * row for a, m in zip(lens, rows) if m) + (n + case["b"] * case["r"]) * h * hd * e
        seen = 0
        for a, m, d in zip(lens, rows, _depths(_trees(case, rows))):
            seen += sum(a + x + 1 for x in d[:m])
        return {"bytes": by, "flops": 4 * h * hd * seen}
    # the kept rows' number follows the inputs; the read-back is what every pass has to do
    all_rows = case["layers"] * case["b"] * case["r"]
    return {"bytes": 2 * all_rows * row + case["b"] * case["r"] * 16, "flops": case["b"] * case["r"] * 4}


# --- the definition in 64 bits --------------------------------------------


def _exact_append(s):
    case, b = s.case, s.case["b"]
    n = case["rot"] // 2
    outs = {}
    for name, src in (("q", s.q), ("k", s.k), ("v", s.v)):
        y = torch.zeros(src.shape, dtype=torch.float64, device=DEV)
        for i in range(b):
            m = s.rows[i]
            if m == 0:
                continue
            x = src[i, :m].double()
            if name != "v":
                d = s.depth[i, :m] if s.depth is not None else torch.arange(m, device=DEV)
                angle = torch.outer((s.lens[i] + d).double(), s.freq)
                turn = s.amplitude * torch.polar(torch.ones_like(angle), angle)[:, None]
                if case["interleaved"]:
                    z = torch.view_as_complex(x[..., :2 * n].reshape(x.shape[:2] + (n, 2)).contiguous()) * turn
                    z = torch.view_as_real(z).reshape(x.shape[:2] + (2 * n,))
                else:
                    z = torch.complex(x[..., :n].contiguous(), x[..., n:2 * n].contiguous()) * turn
                    z = torch.cat([z.real, z.imag], -1)
                x = torch.cat([z, x[..., 2 * n:]], -1)
            y[i, :m] = x
        outs[name] = y
    return outs


def _exact_attend(s):
    case = s.case
    b, r, h, kvh, hd = (case[x] for x in ("b", "r", "h", "kvh", "hd"))
    g = h // kvh
    out = torch.zeros(b, r, h, hd, dtype=torch.float64, device=DEV)
    for i in range(b):
        n, m = s.lens[i], s.rows[i]
        for a in range(kvh if m else 0):
            k, v = (x[:, a].double() for x in s.hist[i])
            for j in range(m):
                anc, at = [], j
                while at >= 0:
                    anc.append(n + at)
                    at = s.parents[i][at]
                own_ = torch.tensor(anc[::-1], device=DEV)
                qj = s.q[i, j, a * g:(a + 1) * g].double()
                z = torch.cat([qj @ k[:n].t(), qj @ k[own_].t()], -1) * hd ** -0.5
                p = torch.softmax(z, -1)
                out[i, j, a * g:(a + 1) * g] = p[:, :n] @ v[:n] + p[:, n:] @ v[own_]
    return {"out": out}


def _mixed_up(z, right, odd):
    """z xor (z >> right), times odd, of 64-bit words held as signed ones."""
    z = z ^ torch.where(z < 0, (z >> right) & ~(torch.full_like(z, -1) << (64 - right)), z >> right)
    return z * (odd - (1 << 64) if odd >> 63 else odd)


def _exact_sample(s):
    """The filtered distributions, and the probabilities of the drawn tokens."""
    case = s.case
    per, vocab = case["t"], case["vocab"]
    t_, k_, p_, m_ = (x.tolist() for x in (s.temperature, s.top_k, s.top_p, s.min_p))
    chosen = torch.ones(case["n"] * per, dtype=torch.float64, device=DEV)
    probs = torch.zeros(case["n"] * per, vocab, dtype=torch.float64, device=DEV) if case["probs"] else None
    bits = s.u.view(torch.int32).tolist()
    golden = 0x9E3779B97F4A7C15 - (1 << 64)
    for row in range(case["n"] * per):
        i = row // per
        z = s.logits[row].double()
        order = torch.argsort(z, descending=True, stable=True)
        if t_[i] <= 0:
            if probs is not None:
                probs[row, order[0]] = 1.0
            continue
        e = torch.exp((z[order] - z[order[0]]) / t_[i])
        n = int((e >= math.exp(-32.0)).sum())
        if k_[i] > 0:
            n = min(n, k_[i])
        if p_[i] < 1:
            short = torch.cumsum(e[:n], 0) < (p_[i] - 2.0 ** -40) * e[:n].sum()
            n = min(n, int(short.sum()) + 1)
        n = max(1, min(n, int((e >= min(m_[i], 1.0)).sum())))
        kept = e[:n] / e[:n].sum()
        # the stream's outputs of the kept tokens alone
        x = bits[row] + (order[:n] + 1) * golden
        x = _mixed_up(_mixed_up(x, 30, 0xBF58476D1CE4E5B9), 27, 0x94D049BB133111EB)
        x = ((_mixed_up(x, 31, 1) >> 41) & 0x7FFFFF).double()
        gumbel = -torch.log(-torch.log((2.0 * x + 1.0) / 2.0 ** 24))
        chosen[row] = kept[torch.argmax(torch.log(e[:n]) + gumbel)]
        if probs is not None:
            probs[row, order[:n]] = kept
    return {"tokens": None, "chosen": chosen, **({"probs": probs} if probs is not None else {})}


def _exact_commit(s):
    case = s.case
    out = {"n": None, "path": None, "correction": None, "lens": None}
    tok, nxt = s.tokens.tolist(), s.next.tolist()
    for l in range(case["layers"]):
        for x, name in ((0, "k"), (1, "v")):
            y = torch.zeros(case["b"], case["r"], case["kvh"], case["hd"], dtype=torch.float64, device=DEV)
            for i in range(case["b"]):
                m = s.rows[i]
                src = s.hist[l][i][x].double()
                y[i, :m] = src
                cur, j = 0, 0
                while m:
                    y[i, j] = src[cur]
                    c = [a for a in range(cur + 1, m) if s.parents[i][a] == cur and tok[i][a] == nxt[i][cur]]
                    if not c:
                        break
                    cur, j = c[0], j + 1
            out[f"{name}{l}"] = y
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "sample": _exact_sample,
            "commit": _exact_commit}[case["op"]](s)
