"""The operators of the 4-bit K/V cache, as measurable cases.

A K/V cache in 4 bits holds, for every position and K/V head, a key and a value
of ``head_dim`` features as 4-bit codes n with one scale s and one minimum m
(both bfloat16): x = m + n s.  Three operators keep and read it
(``paper_2608_13076_amd.kvq``):

``append``  new rows of a layer: the RMSNorm of every query and key head (where
            the model has it), the rotation by position, the keys and values
            into the cache.  A pass also reads the new rows back, as the values
            the cache now holds.
``attend``  causal attention of R new rows per request over the cache, with
            grouped heads; where asked, the weight that every cached position
            received is added to the running weights of the cache.
``evict``   every (layer, request, K/V head) keeps its last positions and the
            heaviest of the others, closed up into a smaller cache; the pass
            reads that cache back.

Head layouts are the ones of ``synth.configs`` (32 or 40 heads of 128 features,
32 query heads over 8 K/V heads, 4 heads of 64) and generic small ones.
"""

import math
import random
from types import SimpleNamespace

import torch

own = False

DEV = "cuda:0"
_T = {"f32": torch.float32, "bf16": torch.bfloat16}


def _append(b, r, h, kvh, hd, dtype, lo, hi, norm, rope, ragged, lens_seed=0, name=None):
    """lo..hi: cached positions of a request before its r new rows (of which a
    ragged batch uses 0..r)."""
    c = {"op": "append", "b": b, "r": r, "h": h, "kvh": kvh, "hd": hd, "dtype": dtype, "lo": lo, "hi": hi,
         "norm": norm, "rope": rope, "ragged": ragged, "lens_seed": lens_seed}
    return {"name": name, **c} if name else c


def _attend(b, r, h, kvh, hd, dtype, lo, hi, weights, ragged, lens_seed=0, name=None):
    """lo..hi: cached positions of a request before its r new rows; weights:
    how many of the new rows are counted into the cache's running weights."""
    c = {"op": "attend", "b": b, "r": r, "h": h, "kvh": kvh, "hd": hd, "dtype": dtype, "lo": lo, "hi": hi,
         "weights": weights, "ragged": ragged, "lens_seed": lens_seed}
    return {"name": name, **c} if name else c


def _evict(layers, b, kvh, hd, dtype, lo, hi, budget, recent, lens_seed=0, name=None):
    """lo..hi: cached positions of a request; dtype: that of the read-back."""
    c = {"op": "evict", "layers": layers, "b": b, "kvh": kvh, "hd": hd, "dtype": dtype, "lo": lo, "hi": hi,
         "budget": budget, "recent": recent, "lens_seed": lens_seed}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one decoded token of one request, grouped heads: the smallest append
        _append(1, 1, 32, 8, 128, "bf16", 1024, 1024, True, True, False, name="append_token_gqa"),
        # the rows of a batched verify call, float32 projections, ragged drafts
        _append(16, 9, 32, 8, 128, "f32", 256, 4096, True, True, True, 1, name="append_verify_b16"),
        # a long piece of a prompt of a multi-head model without head norms
        _append(1, 2048, 32, 32, 128, "bf16", 4099, 4099, False, True, False, name="append_prompt_2k"),
        # small heads, odd counts
        _append(5, 13, 4, 4, 64, "f32", 0, 130, True, True, True, 2, name="append_hd64_odd"),
        # the first decode steps after a short prompt
        _attend(1, 1, 32, 8, 128, "bf16", 129, 129, 0, False, name="attend_token_short"),
        # the benchmark's verify call: 6 rows of one request over 1024 positions
        _attend(1, 6, 32, 32, 128, "f32", 1024, 1024, 0, False, name="attend_verify_b1"),
        # a batched verify of a grouped-query model, ragged contexts and drafts
        _attend(16, 9, 32, 8, 128, "f32", 256, 4096, 0, True, 3, name="attend_verify_b16_gqa"),
        # decoding a full batch with long contexts, weights kept for eviction
        _attend(16, 1, 32, 8, 128, "bf16", 5000, 16000, 1, False, 4, name="attend_token_b16_weights"),
        # one request with a very long context
        _attend(1, 1, 32, 8, 128, "bf16", 120001, 120001, 0, False, name="attend_token_120k"),
        # small heads, odd counts, every row counted into the weights
        _attend(3, 5, 12, 4, 64, "f32", 1, 700, 5, True, 5, name="attend_hd64_weights"),
        # a layer of one request just past its budget
        _evict(1, 1, 8, 128, "f32", 1100, 1100, 1024, 64, name="evict_b1"),
        # four layers of a full batch cut to a quarter or less, some requests below their budget
        _evict(4, 16, 8, 128, "bf16", 900, 12000, 2048, 256, 6, name="evict_b16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "evict"])
    kvh, g, hd = rng.choice([(8, 4, 128), (32, 1, 128), (40, 1, 128), (4, 1, 64), (4, 3, 64), (8, 2, 128), (2, 8, 128),
                             (1, 6, 64), (5, 1, 128)])
    dtype = rng.choice(["f32", "bf16"])
    seed = rng.randrange(1 << 20)
    if op == "append":
        b = _log(rng, 1, 16)
        r = _log(rng, 1, max(1, 2048 // b) if rng.random() < 0.3 else 16)
        lo = rng.randrange(0, 200)
        return _append(b, r, kvh * g, kvh, hd, dtype, lo, lo + _log(rng, 1, 4000), rng.random() < 0.6, rng.random() < 0.9,
                       rng.random() < 0.5, seed)
    if op == "attend":
        b = _log(rng, 1, 16)
        r = rng.choice([1, 1, rng.randrange(2, 17)])
        # the largest listed case holds 16 x 16000 positions of 8 K/V heads
        hi = _log(rng, 1, min(120000, 16000 * 16 * 8 // (2 * b * kvh * (2 if r > 1 else 1))))
        lo = rng.choice([hi, max(0, hi // 8), 0])
        return _attend(b, r, kvh * g, kvh, hd, dtype, lo, hi, rng.choice([0, 1, r]), rng.random() < 0.5, seed)
    b, layers = _log(rng, 1, 16), rng.randrange(1, 5)
    hi = _log(rng, 64, min(30000, 4 * 16 * 8 * 12000 // (layers * b * kvh)))
    budget = max(1, min(hi, 2048, int(hi * rng.uniform(0.1, 1.0))))
    return _evict(layers, b, kvh, hd, dtype, rng.choice([hi, hi // 3]), hi, budget,
                  rng.choice([0, budget, rng.randrange(0, budget + 1)]), seed)


def _counts(case):
    """Cached positions of every request and, of append and attend, its rows."""
    rng = random.Random(1000 + case["lens_seed"])
    lens = [rng.randint(case["lo"], case["hi"]) for _ in range(case["b"])]
    r = case.get("r", 0)
    rows = [rng.randint(0, r) if case.get("ragged") else r for _ in lens]
    if r and not any(rows):
        rows[0] = r
    return lens, rows


def _history(gen, n, kvh, hd):
    """Keys or values of n positions: a few strong features per head, as the
    keys of trained models have, and a drift along the positions."""
    x = torch.randn(n, kvh, hd, generator=gen, device=DEV)
    x[:, :, ::17] *= 4.0
    return (x + 0.3 * torch.randn(1, kvh, hd, generator=gen, device=DEV)).to(torch.bfloat16)


def _rope_table(n, hd, theta):
    pos = torch.arange(n, dtype=torch.float64, device=DEV)[:, None]
    inv = theta ** (-2.0 * torch.arange(hd // 2, dtype=torch.float64, device=DEV) / hd)
    return torch.stack([torch.cos(pos * inv), torch.sin(pos * inv)], -1).float().contiguous()


def _inputs(case, seed):
    """The case's inputs, the same for either form."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    lens, rows = _counts(case)
    s = SimpleNamespace(case=case, lens=lens, rows=rows)
    b, kvh, hd = case["b"], case["kvh"], case["hd"]
    t = _T[case["dtype"]]
    s.d_lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s.d_rows = torch.tensor(rows, dtype=torch.int32, device=DEV)
    if case["op"] == "append":
        h, r = case["h"], case["r"]
        # the output of a fused projection: queries, keys and values of a row
        x = torch.randn(b, r, h + 2 * kvh, hd, generator=gen, device=DEV)
        x[:, :, :, 3::29] *= 5.0
        s.qkv = x.to(t)
        s.q, s.k, s.v = s.qkv[:, :, :h], s.qkv[:, :, h:h + kvh], s.qkv[:, :, h + kvh:]
        s.gain_q = s.gain_k = s.rope = None
        if case["norm"]:
            s.gain_q = 1.0 + 0.2 * torch.randn(hd, generator=gen, device=DEV)
            s.gain_k = 1.0 + 0.2 * torch.randn(hd, generator=gen, device=DEV)
        if case["rope"]:
            s.rope = _rope_table(max(lens) + r, hd, 500000.0)
    elif case["op"] == "attend":
        h, r = case["h"], case["r"]
        s.q = (1.5 * torch.randn(b, r, h, hd, generator=gen, device=DEV)).to(t)
        s.hist = [(_history(gen, n + m, kvh, hd), _history(gen, n + m, kvh, hd)) for n, m in zip(lens, rows)]
        s.cap = max(lens) + r
        s.weights = None
        if case["weights"]:
            s.weights = torch.rand(b, kvh, s.cap, generator=gen, device=DEV) * 3.0
    else:
        s.cap = max(lens)
        s.hist = [[(_history(gen, n, kvh, hd), _history(gen, n, kvh, hd)) for n in lens]
                  for _ in range(case["layers"])]
        # heavy-tailed running weights; a quarter of the positions never got any, so there are ties
        w = torch.randn(case["layers"], b, kvh, s.cap, generator=gen, device=DEV).mul(2.0).exp()
        w[torch.rand(w.shape, generator=gen, device=DEV) < 0.25] = 0.0
        s.weights = w
    return s


# --- the plain form -------------------------------------------------------


def _quantise(x):
    """(codes, scale, minimum) of float rows [..., hd].  A row's values enter as
    float32; the quotient next to a border is taken in 64 bits."""
    x = x.float()
    m = x.amin(-1, keepdim=True).to(torch.bfloat16).float()
    d = (x.amax(-1, keepdim=True) - m).clamp_min(0.0)
    s = (d / 15.0).to(torch.bfloat16).float()
    t = (x.double() - m.double()) / torch.where(s > 0, s, torch.ones_like(s)).double()
    n = torch.where(s > 0, t, torch.zeros_like(t)).round().clamp(0, 15)
    return n.to(torch.uint8), s, m


def _values(c):
    n, s, m = c
    return m + n.float() * s


def _norm_rotate(x, gain, eps, table):
    """x [rows, heads, hd] in 64 bits: RMSNorm over a head, then the rotation
    of feature i with i + hd/2 by the row's angles (table [rows, hd/2, 2])."""
    x = x.double()
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double()
    if table is not None:
        half = x.shape[-1] // 2
        c, sn = table[:, None, :, 0].double(), table[:, None, :, 1].double()
        a, b = x[..., :half], x[..., half:]
        x = torch.cat([a * c - b * sn, b * c + a * sn], -1)
    return x


_EPS = 1e-5


def _plain_append(s):
    case, b, r = s.case, s.case["b"], s.case["r"]
    t = s.q.dtype
    # every row of the padded batch at once; the rows a request does not use give zeros
    at = (s.d_lens[:, None] + torch.arange(r, device=DEV)[None]).reshape(-1).long()
    live = (torch.arange(r, device=DEV)[None] < s.d_rows[:, None]).reshape(-1)
    tab = s.rope[at] if s.rope is not None else None
    flat = [x.reshape(b * r, x.shape[2], x.shape[3]) for x in (s.q, s.k, s.v)]
    q = _norm_rotate(flat[0], s.gain_q, _EPS, tab)
    k = _norm_rotate(flat[1], s.gain_k, _EPS, tab)
    zero = (~live)[:, None, None]
    q = q.masked_fill(zero, 0.0).to(t).reshape(s.q.shape)
    out = [_values(_quantise(x)).masked_fill(zero, 0.0).to(t).reshape(s.k.shape) for x in (k, flat[2])]
    return {"q": q, "k": out[0], "v": out[1]}


def _plain_attend(s):
    case = s.case
    b, r, h, kvh, hd = (case[x] for x in ("b", "r", "h", "kvh", "hd"))
    g = h // kvh
    out = torch.zeros(b, r, h, hd, dtype=s.q.dtype, device=DEV)
    w = torch.zeros_like(s.weights) if s.weights is not None else None
    for i, (n, m) in enumerate(zip(s.lens, s.rows)):
        if m == 0:
            if w is not None:
                w[i, :, :n] = s.weights[i, :, :n]
            continue
        k = _values(s.codes[i][0]).transpose(0, 1)  # [kvh, n + m, hd]
        v = _values(s.codes[i][1]).transpose(0, 1)
        q = s.q[i, :m].float().reshape(m, kvh, g, hd).permute(1, 2, 0, 3).reshape(kvh, g * m, hd)
        z = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(hd)
        row = torch.arange(g * m, device=DEV) % m
        hidden = torch.arange(n + m, device=DEV)[None] > (n + row)[:, None]
        z = z.masked_fill(hidden[None], -math.inf)
        z = torch.exp(z - z.amax(-1, keepdim=True))
        p = z / z.sum(-1, keepdim=True)
        o = torch.matmul(p, v.contiguous())
        out[i, :m] = o.reshape(kvh, g, m, hd).permute(2, 0, 1, 3).reshape(m, h, hd).to(out.dtype)
        if w is not None:
            c = min(case["weights"], m)
            add = p.reshape(kvh, g, m, n + m)[:, :, :c].sum((1, 2))
            w[i, :, :n + m] = s.weights[i, :, :n + m] + add
    return {"out": out, "weights": w} if w is not None else {"out": out}


def _plain_evict(s):
    case = s.case
    layers, b, kvh, hd = (case[x] for x in ("layers", "b", "kvh", "hd"))
    budget, recent = case["budget"], case["recent"]
    t = _T[case["dtype"]]
    kept = torch.full((layers, b, kvh, budget), -1, dtype=torch.int32, device=DEV)
    w = torch.zeros(layers, b, kvh, budget, device=DEV)
    k = torch.zeros(layers, b, budget, kvh, hd, dtype=t, device=DEV)
    v = torch.zeros_like(k)
    lens = []
    for i, n in enumerate(s.lens):
        m = min(n, budget)
        lens.append(m)
        for l in range(layers):
            if n <= budget:
                idx = torch.arange(n, device=DEV).expand(kvh, n)
            else:
                # ties go to the lowest position: a stable sort keeps it first
                old = torch.sort(s.weights[l, i, :, :n - recent], dim=-1, descending=True, stable=True)[1]
                old = torch.sort(old[:, :budget - recent], dim=-1)[0]
                idx = torch.cat([old, torch.arange(n - recent, n, device=DEV).expand(kvh, recent)], -1)
            kept[l, i, :, :m] = idx.to(torch.int32)
            w[l, i, :, :m] = torch.gather(s.weights[l, i], -1, idx)
            rows = idx.t()  # [m, kvh]
            for codes, dst in zip(s.codes[l][i], (k, v)):
                n4, sc, mn = codes
                pick = rows[:, :, None]
                dst[l, i, :m] = (torch.gather(mn, 0, pick) + torch.gather(n4, 0, pick.expand(m, kvh, hd)).float() *
                                 torch.gather(sc, 0, pick)).to(t)
    return {"kept": kept, "lens": torch.tensor(lens, dtype=torch.int32, device=DEV), "weights": w, "k": k, "v": v}


# --- the framework's operators --------------------------------------------


def _fill(cache, layer, hist, rows):
    """Keys and values of every request into an empty cache, as they stand."""
    n = max(len(x[0]) for x in hist)
    pad = [torch.zeros((len(hist), n) + tuple(hist[0][j].shape[1:]), dtype=torch.bfloat16, device=DEV) for j in (0, 1)]
    for i, kv in enumerate(hist):
        for j in (0, 1):
            pad[j][i, :len(kv[j])] = kv[j]
    cache.append(layer, pad[0], pad[1], rows=rows)


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        if case["op"] == "attend":
            s.codes = [(_quantise(k), _quantise(v)) for k, v in s.hist]
        elif case["op"] == "evict":
            s.codes = [[(_quantise(k), _quantise(v)) for k, v in layer] for layer in s.hist]
        s.hist = None
        return s
    from paper_2608_13076_amd import kvq
    b, kvh, hd = case["b"], case["kvh"], case["hd"]
    if case["op"] == "append":
        s.cache = kvq.QuantCache(1, b, case["h"], kvh, hd, max(s.lens) + case["r"], device=DEV)
        s.cache.lens.copy_(s.d_lens)
    elif case["op"] == "attend":
        s.cache = kvq.QuantCache(1, b, case["h"], kvh, hd, s.cap, max_rows=case["r"], device=DEV)
        _fill(s.cache, 0, s.hist, s.d_lens + s.d_rows)
        s.cache.lens.copy_(s.d_lens)
        s.max_keys = max(n + m for n, m in zip(s.lens, s.rows))
        s.weights_out = torch.zeros_like(s.weights) if s.weights is not None else None
    else:
        s.cache = kvq.QuantCache(case["layers"], b, kvh, kvh, hd, s.cap, device=DEV)
        for l in range(case["layers"]):
            _fill(s.cache, l, s.hist[l], s.d_lens)
        s.cache.lens.copy_(s.d_lens)
        s.out = kvq.QuantCache(case["layers"], b, kvh, kvh, hd, case["budget"], device=DEV)
        s.kept = torch.empty(case["layers"], b, kvh, case["budget"], dtype=torch.int32, device=DEV)
        s.weights_out = torch.zeros(case["layers"], b, kvh, case["budget"], device=DEV)
    s.hist = None
    return s


def run(s):
    case = s.case
    if not own:
        return {"append": _plain_append, "attend": _plain_attend, "evict": _plain_evict}[case["op"]](s)
    if case["op"] == "append":
        q = s.cache.append(0, s.k, s.v, q=s.q, gain_q=s.gain_q, gain_k=s.gain_k, eps=_EPS, rope=s.rope, rows=s.d_rows)
        k, v = s.cache.read(0, case["r"], start=s.d_lens, rows=s.d_rows, dtype=s.q.dtype)
        return {"q": q, "k": k, "v": v}
    if case["op"] == "attend":
        out = s.cache.attend(0, s.q, rows=s.d_rows, max_keys=s.max_keys, weights=s.weights, weights_out=s.weights_out,
                             weight_rows=case["weights"])
        return {"out": out, "weights": s.weights_out} if s.weights is not None else {"out": out}
    s.cache.evict(s.weights, case["budget"], case["recent"], s.kept, into=s.out, weights_out=s.weights_out)
    kv = [s.out.read(l, case["budget"], rows=s.out.lens, dtype=_T[case["dtype"]]) for l in range(case["layers"])]
    return {"kept": s.kept, "lens": s.out.lens, "weights": s.weights_out, "k": torch.stack([x[0] for x in kv]),
            "v": torch.stack([x[1] for x in kv])}


# --- what a pass cannot do without ----------------------------------------


def work(case):
    lens, rows = _counts(case)
    kvh, hd = case["kvh"], case["hd"]
    e = 4 if case["dtype"] == "f32" else 2
    row = kvh * (hd + 8)  # codes, scales and minima of a position's keys and values
    back = 2 * kvh * hd * e  # ... and the values they stand for
    if case["op"] == "append":
        h, n, all_rows = case["h"], sum(rows), case["b"] * case["r"]
        rope = max(lens) + case["r"] if case["rope"] else 0
        by = n * ((h + 2 * kvh) * hd * e + 2 * row) + all_rows * (h * hd * e + back) + min(n, rope) * hd * 4
        return {"bytes": by, "flops": n * ((h + kvh) * hd * 6 + 2 * kvh * hd * 4)}
    if case["op"] == "attend":
        h, r = case["h"], case["r"]
        keys = [n + m for n, m in zip(lens, rows)]
        by = sum(k * row for k, m in zip(keys, rows) if m) + sum(rows) * h * hd * e + case["b"] * r * h * hd * e
        if case["weights"]:
            by += sum(keys) * kvh * 8
        return {"bytes": by, "flops": sum(4 * m * h * hd * k for k, m in zip(keys, rows))}
    layers, budget = case["layers"], case["budget"]
    kept = sum(min(n, budget) for n in lens)
    by = layers * (sum(lens) * kvh * 4 + 3 * kept * row + kept * kvh * 4 + case["b"] * budget * (kvh * 4 + back))
    return {"bytes": by, "flops": layers * kvh * sum(lens)}


# --- the definition in 64 bits --------------------------------------------


def _bf16(x):
    """The bfloat16 nearest to the float32 nearest to x, ties to even, in 64 bits."""
    return x.to(torch.float32).to(torch.bfloat16).to(torch.float64)


def _held(x):
    """What the cache holds for rows x (64 bits): minimum, scale and codes by
    their definition, put together in 64 bits."""
    x = x.to(torch.float32).to(torch.float64)
    lo = _bf16(torch.min(x, dim=-1, keepdim=True)[0])
    span = (torch.max(x, dim=-1, keepdim=True)[0] - lo).to(torch.float32).clamp(min=0.0)
    step = _bf16(span / 15.0)
    ok = step > 0
    n = torch.round((x - lo) / step.masked_fill(~ok, 1.0)) * ok
    return lo + step * torch.clamp(n, 0.0, 15.0)


def _exact_append(s):
    b, r = s.case["b"], s.case["r"]
    half = s.case["hd"] // 2
    outs = {}
    for name, src, gain in (("q", s.q, s.gain_q), ("k", s.k, s.gain_k), ("v", s.v, None)):
        y = torch.zeros(src.shape, dtype=torch.float64, device=DEV)
        for i in range(b):
            m, n = s.rows[i], s.lens[i]
            x = src[i, :m].double()
            if m == 0:
                continue
            if name != "v":
                if gain is not None:
                    ms = torch.einsum("rhf,rhf->rh", x, x) / x.shape[-1]
                    x = gain.double() * x * torch.rsqrt(ms + _EPS)[:, :, None]
                if s.rope is not None:
                    z = torch.complex(x[..., :half].contiguous(), x[..., half:].contiguous())
                    e = s.rope[n:n + m].double()
                    z = z * torch.complex(e[..., 0].contiguous(), e[..., 1].contiguous())[:, None, :]
                    x = torch.cat([z.real, z.imag], -1)
            y[i, :m] = x if name == "q" else _held(x)
        outs[name] = y
    return outs


def _exact_attend(s):
    case = s.case
    b, r, h, kvh, hd = (case[x] for x in ("b", "r", "h", "kvh", "hd"))
    g = h // kvh
    out = torch.zeros(b, r, h, hd, dtype=torch.float64, device=DEV)
    w = s.weights.double() if s.weights is not None else None
    for i in range(b):
        n, m = s.lens[i], s.rows[i]
        for a in range(kvh):
            if m == 0:
                continue
            k, v = (_held(x[:, a].double()) for x in s.hist[i])
            for j in range(m):
                seen = n + j + 1
                z = s.q[i, j, a * g:(a + 1) * g].double() @ k[:seen].t() * hd ** -0.5
                p = torch.softmax(z, -1)
                out[i, j, a * g:(a + 1) * g] = p @ v[:seen]
                if w is not None and j < case["weights"]:
                    w[i, a, :seen] += p.sum(0)
        if w is not None:
            w[i, :, n + m:] = 0.0
    return {"out": out, "weights": w} if w is not None else {"out": out}


def _exact_evict(s):
    case = s.case
    layers, b, kvh, hd, budget, recent = (case[x] for x in ("layers", "b", "kvh", "hd", "budget", "recent"))
    w = torch.zeros(layers, b, kvh, budget, dtype=torch.float64, device=DEV)
    kv = [torch.zeros(layers, b, budget, kvh, hd, dtype=torch.float64, device=DEV) for _ in range(2)]
    for l in range(layers):
        for i in range(b):
            n, held = s.lens[i], [_held(x.double()) for x in s.hist[l][i]]
            for a in range(kvh):
                score = s.weights[l, i, a, :n].double()
                if n > budget:
                    order = torch.argsort(score[:n - recent], descending=True, stable=True)[:budget - recent]
                    keep = torch.zeros(n, dtype=torch.bool, device=DEV)
                    keep[order] = True
                    keep[n - recent:] = True
                else:
                    keep = torch.ones(n, dtype=torch.bool, device=DEV)
                m = min(n, budget)
                w[l, i, a, :m] = score[keep]
                for x, y in zip(held, kv):
                    y[l, i, :m, a] = x[keep, a]
    return {"kept": None, "lens": None, "weights": w, "k": kv[0], "v": kv[1]}


def exact(case, seed):
    s = _inputs(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "evict": _exact_evict}[case["op"]](s)
