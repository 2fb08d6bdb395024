"""Filtered sampling on the GPU against the float64 oracle (oracle/tree.py).

Tokens are compared for equality: the oracle's borders and draws are decided in 64
bits, the kernels' to 2^-34 or better, and the inputs are seeded, so a row whose
border or draw is closer than that would show in the first run.  A probability is a
quotient in double rounded once to float32: 2^-24 of it, with weights and sums good
to 2^-33: 2^-23 in all.
"""

import numpy as np
import pytest
import torch

from oracle import tree as otree
from paper_2608_13076_amd import sampling, spade

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TD = {"f32": torch.float32, "bf16": torch.bfloat16}


def check(logits, u, probs, tokens, chosen, per, **kw):
    """Rows against the oracle; kw: lists of one value per request."""
    l = logits.float().cpu().numpy().astype(np.float64)
    got_p = None if probs is None else probs.cpu().numpy().astype(np.float64)
    for row in range(len(l)):
        one = {k: v[row // per] for k, v in kw.items()}
        t, p = otree.sample(l[row], float(u[row]), **one)
        assert int(tokens[row]) == t, (row, one, int(tokens[row]), t, p[int(tokens[row])], p[t])
        assert abs(float(chosen[row]) - p[t]) <= 2.0 ** -23 * p[t], (row, one)
        if got_p is not None:
            assert ((got_p[row] > 0) == (p > 0)).all() or (np.abs(got_p[row] - p) <= 1e-38).all(), (row, one)
            assert (np.abs(got_p[row] - p) <= 2.0 ** -23 * p + 1e-38).all(), (row, one)


def settings(rng, n):
    t = np.where(rng.random(n) < 0.15, 0.0, rng.uniform(0.3, 1.5, n)).astype(np.float32)
    k = np.where(rng.random(n) < 0.5, 0, np.exp(rng.uniform(0, 8, n))).astype(np.int32)
    p = np.where(rng.random(n) < 0.4, 1.0, rng.uniform(0.05, 0.999, n)).astype(np.float32)
    m = np.where(rng.random(n) < 0.6, 0.0, rng.uniform(0.0, 0.3, n)).astype(np.float32)
    return {"temperature": t, "top_k": k, "top_p": p, "min_p": m}


def run(logits, u, kw, per=1, probs=True, sampler=None):
    rows, V = logits.shape
    s = sampler or sampling.Sampler(rows, V, device=DEV)
    pr = torch.full((rows, V), 7.0, device=DEV) if probs else None
    args = {k: (torch.from_numpy(np.ascontiguousarray(v)).to(DEV) if isinstance(v, np.ndarray) else v) for k, v in kw.items()}
    tok, ch = s.draw(logits, u, probs=pr, **args)
    return tok, ch, pr, s


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,per,V,scale", [(40, 1, 2, 1.0), (40, 1, 7, 3.0), (30, 2, 100, 2.0), (24, 1, 4095, 2.0),
                                           (24, 1, 4097, 5.0), (16, 3, 32000, 2.5), (8, 1, 128256, 2.0), (6, 1, 128256, 6.0),
                                           (3, 1, 300001, 0.5)])
def test_sample(n, per, V, scale, dtype):
    rng = np.random.default_rng(V + n)
    x = rng.normal(size=(n * per, V)).astype(np.float32) * scale
    x[:, rng.integers(0, V, 8)] += rng.uniform(0, 8, 8).astype(np.float32)
    logits = torch.from_numpy(x).to(DEV).to(TD[dtype])
    u = torch.from_numpy(rng.random(n * per, np.float32)).to(DEV)
    kw = settings(rng, n)
    tok, ch, pr, s = run(logits, u, kw, per)
    check(logits, u, pr, tok, ch, per, **kw)
    assert s.device_error() == 0
    # the same call gives the same bits, also without the distribution
    tok2, ch2, _, _ = run(logits, u, kw, per, probs=False, sampler=s)
    assert torch.equal(tok, tok2) and torch.equal(ch, ch2)


@pytest.mark.parametrize("kw", [dict(), dict(temperature=0.0), dict(temperature=0.7), dict(top_k=1), dict(top_k=50),
                                dict(top_p=0.9), dict(top_p=1e-9), dict(top_p=0.0), dict(top_p=-1.0), dict(min_p=0.1),
                                dict(min_p=1.0), dict(min_p=7.0), dict(top_k=50, top_p=0.5, min_p=0.05),
                                dict(top_k=100000), dict(temperature=-3.0), dict(top_k=-5),
                                dict(top_p=float(np.nextafter(np.float32(1), np.float32(0))))])
@pytest.mark.parametrize("V", [1000, 20000])
def test_one_setting_for_all(kw, V):
    rng = np.random.default_rng(V)
    logits = torch.from_numpy(rng.normal(size=(12, V)).astype(np.float32) * 3).to(DEV)
    u = torch.from_numpy(rng.random(12, np.float32)).to(DEV)
    tok, ch, pr, _ = run(logits, u, kw)
    check(logits, u, pr, tok, ch, 12, **{k: [v] for k, v in kw.items()})


def ties(V, kind, rng):
    if kind == "equal":
        return np.zeros(V, np.float32)
    if kind == "levels":
        return rng.integers(0, 4, V).astype(np.float32)
    if kind == "signed zeros":
        return np.where(rng.random(V) < 0.5, 0.0, -0.0).astype(np.float32)
    return np.repeat(rng.normal(size=(V + 6) // 7), 7)[:V].astype(np.float32)


@pytest.mark.parametrize("kind", ["equal", "levels", "signed zeros", "runs"])
@pytest.mark.parametrize("V", [16, 5000, 70000])
def test_ties_go_to_the_lowest_ids(kind, V):
    rng = np.random.default_rng(V)
    sets = [dict(top_k=k) for k in (1, 3, V // 2, V - 1)] + [dict(top_p=p) for p in (0.25, 0.5, 0.75, 0.9)]
    sets += [dict(top_k=V // 2, top_p=0.5), dict(min_p=1.0), dict(temperature=0.0)]
    row = ties(V, kind, rng)
    logits = torch.from_numpy(np.stack([row] * len(sets))).to(DEV)
    u = torch.from_numpy(rng.random(len(sets), np.float32)).to(DEV)
    base = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)
    cols = {k: np.array([{**base, **s}[k] for s in sets], np.int32 if k == "top_k" else np.float32) for k in base}
    tok, ch, pr, _ = run(logits, u, cols)
    check(logits, u, pr, tok, ch, 1, **cols)


@pytest.mark.parametrize("V", [50, 9000])
def test_masked_and_extreme_logits(V):
    """-infinity, the lowest number, +infinity and NaN among the logits, tiny and
    huge temperatures, rows with nothing left."""
    rng = np.random.default_rng(V)
    base = rng.normal(size=V).astype(np.float32) * 4
    rows, sets = [], []
    for fill in (-np.inf, np.finfo(np.float32).min, -1e30):
        for s in (dict(), dict(top_k=20), dict(top_p=0.8), dict(temperature=0.0), dict(top_k=V - 2, top_p=0.99)):
            r = base.copy()
            r[rng.random(V) < 0.9] = fill
            r[rng.integers(0, V)] = 1.0
            rows.append(r)
            sets.append(s)
    for s in (dict(), dict(top_k=5), dict(top_p=0.5), dict(temperature=0.0)):
        r = base.copy()
        r[[3, V - 1]] = np.inf
        rows.append(r)
        sets.append(s)
        r = np.full(V, -np.inf, np.float32)
        r[V // 2] = -1e38
        rows.append(r)
        sets.append(s)
    for t in (1e-45, 1e-30, 1e-6, 1e-3, 50.0, 1e30, np.inf):
        for s in (dict(), dict(top_k=9), dict(top_p=0.7), dict(min_p=0.2)):
            rows.append(base if t > 1e-20 else base * np.float32(1e20))
            sets.append(dict(s, temperature=t))
    for s in (dict(temperature=1e-20), dict(temperature=1e-3, top_k=7), dict(temperature=1e30, top_p=0.5)):
        r = base * np.float32(1e30)
        r[rng.integers(0, V, 9)] = r.max()
        rows.append(r)
        sets.append(s)
    logits = torch.from_numpy(np.stack(rows)).to(DEV)
    u = torch.from_numpy(rng.random(len(rows), np.float32)).to(DEV)
    d = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)
    cols = {k: np.array([{**d, **s}[k] for s in sets], np.int32 if k == "top_k" else np.float32) for k in d}
    tok, ch, pr, sm = run(logits, u, cols)
    check(logits, u, pr, tok, ch, 1, **cols)
    assert sm.device_error() == 0
    # NaN counts as -infinity and is flagged; rows of nothing give token 0 and no probability
    bad = logits[:4].clone()
    bad[0, ::2] = float("nan")
    bad[1] = float("nan")
    bad[2] = float("-inf")
    bad[3, :] = float("-inf")
    bad[3, V - 1] = float("nan")
    kw = dict(temperature=np.array([1, 1, 0.5, 0], np.float32), top_k=np.array([0, 5, 0, 0], np.int32))
    tok, ch, pr, sm = run(bad, u[:4].contiguous(), kw)
    assert sm.device_error() == spade.DERR_NAN and sm.device_error() == 0
    assert tok.tolist()[1:] == [0, 0, 0] and ch.tolist()[1:] == [0.0] * 3 and not pr[1:].any()
    check(bad[:1], u[:1], pr[:1], tok[:1], ch[:1], 1, temperature=[1.0])


def test_parameters_that_are_not_numbers():
    """NaN turns a filter off, of a temperature makes the row greedy."""
    rng = np.random.default_rng(1)
    logits = torch.from_numpy(rng.normal(size=(4, 600)).astype(np.float32)).to(DEV)
    u = torch.rand(4, device=DEV)
    nan = float("nan")
    kw = dict(temperature=np.array([1, nan, 1, 1], np.float32), top_p=np.array([nan, 0.5, 0.5, 1], np.float32),
              min_p=np.array([0, 0, nan, nan], np.float32))
    tok, ch, pr, _ = run(logits, u, kw)
    check(logits, u, pr, tok, ch, 1, temperature=[1, 0, 1, 1], top_p=[1, 1, 0.5, 1], min_p=[0] * 4)


def test_strides_in_place_and_reuse():
    """Rows of a wider buffer at odd addresses; the distribution over the logits;
    one sampler for smaller calls."""
    rng = np.random.default_rng(2)
    s = sampling.Sampler(9, 5003, device=DEV)
    for dtype in ("f32", "bf16"):
        wide = torch.from_numpy(rng.normal(size=(6, 5011)).astype(np.float32) * 3).to(DEV).to(TD[dtype])
        u = torch.from_numpy(rng.random(6, np.float32)).to(DEV)
        for off, V in ((0, 5003), (3, 5001), (1, 77)):
            logits = wide[:, off:off + V]
            tok, ch, pr, _ = run(logits, u, dict(top_p=0.7), sampler=s)
            check(logits, u, pr, tok, ch, 6, top_p=[0.7])
    logits = wide[:, :1999].float().contiguous()
    want = run(logits, u, dict(top_k=30, temperature=0.6), sampler=s)
    tok, ch = s.draw(logits, u, top_k=30, temperature=0.6, probs=logits)
    assert torch.equal(tok, want[0]) and torch.equal(ch, want[1]) and torch.equal(logits, want[2])


def test_the_same_draws_as_the_verifier():
    """Without filters and at one temperature the draw is spade_softmax's
    distribution and the verifier's bonus token of the same uniform."""
    rng = np.random.default_rng(3)
    V, B = 8011, 12
    logits = torch.from_numpy(rng.normal(size=(B, V)).astype(np.float32) * 2).to(DEV)
    u = torch.from_numpy(rng.random(B, np.float32)).to(DEV)
    n, corr, err = (torch.zeros(x, dtype=torch.int32, device=DEV) for x in (B, B, 1))
    modes = torch.ones(B, dtype=torch.uint8, device=DEV)
    spade.accept_from_logits_noalloc(logits[:, None].contiguous(), None, None, u, modes, 0.75, n, corr, err)
    tok, ch, pr, _ = run(logits, u, dict(temperature=0.75))
    assert torch.equal(tok, corr)
    sm = torch.empty_like(logits)
    spade.softmax_into(logits, sm, 0.75)
    assert ((pr - sm).abs() <= 1e-5 * sm + 1e-12).all()  # (spade_softmax is float32: exponents up to 22 rounded at 2^-20)


def test_distribution_of_the_draw():
    """Many uniforms over one row: chi-squared against the filtered distribution."""
    rng = np.random.default_rng(4)
    row = torch.from_numpy(rng.normal(size=50).astype(np.float32) * 1.5).to(DEV)
    N = 20000
    logits = row[None].expand(N, 50).contiguous()
    u = torch.from_numpy(rng.random(N, np.float32)).to(DEV)
    tok, _, _, _ = run(logits, u, dict(top_p=0.9), probs=False)
    _, p = otree.sample(row.cpu().numpy(), 0.5, top_p=0.9)
    got = np.bincount(tok.cpu().numpy(), minlength=50)
    ok = p > 0
    assert got[~ok].sum() == 0
    chi = ((got - N * p)[ok] ** 2 / (N * p[ok])).sum()
    k = ok.sum() - 1
    assert chi < k + 3.3 * np.sqrt(2 * k) + 6  # (0.1%)


@pytest.mark.parametrize("n", [1, 2, 63, 64, 255, 256, 257, 1024, 1025, 8191, 8192, 8193, 12000])
def test_borders_among_n_close_tokens(n):
    """n logits within a quarter of each other hold nearly all the weight, some of
    them equal: the borders lie among them, however they are looked for.  Calls
    in a row give the same bits."""
    rng = np.random.default_rng(n)
    V, sets = 20011, []
    for k in sorted({1, 2, n // 3 + 1, n - 1 or 1, n, n + 1}):
        sets += [dict(top_k=k), dict(top_k=k, top_p=0.6, min_p=0.9)]
    sets += [dict(top_p=p) for p in (1e-6, 0.1, 0.5, 0.97)]
    x = rng.uniform(-14, -12, size=(len(sets), V)).astype(np.float32)
    for r in range(len(sets)):
        x[r, rng.choice(V, n, replace=False)] = np.round(rng.uniform(0, 0.25, n) * 4096) / 4096
    logits, u = torch.from_numpy(x).to(DEV), torch.from_numpy(rng.random(len(sets), np.float32)).to(DEV)
    base = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)
    cols = {k: np.array([{**base, **s}[k] for s in sets], np.int32 if k == "top_k" else np.float32) for k in base}
    tok, ch, pr, s = run(logits, u, cols)
    check(logits, u, pr, tok, ch, 1, **cols)
    for _ in range(4):
        t2, c2, p2, _ = run(logits, u, cols, sampler=s)
        assert torch.equal(tok, t2) and torch.equal(ch, c2) and torch.equal(pr, p2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,scale", [(40000, 0.05), (128256, 1.0), (128256, 0.3), (262147, 0.5)])
def test_borders_among_more_tokens_than_a_list_holds(V, scale, dtype):
    """Flat rows, whose bins at the border hold tens of thousands of tokens."""
    rng = np.random.default_rng(V)
    sets = [dict(top_p=p) for p in (0.01, 0.5, 0.9, 0.9999)] + [dict(top_k=V // 2), dict(top_k=V // 2, top_p=0.7),
            dict(top_k=V - 9, top_p=0.95, min_p=0.3), dict(top_p=0.8, temperature=3.0, min_p=0.8)]
    logits = torch.from_numpy(rng.normal(size=(len(sets), V)).astype(np.float32) * scale).to(DEV).to(TD[dtype])
    u = torch.from_numpy(rng.random(len(sets), np.float32)).to(DEV)
    base = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)
    cols = {k: np.array([{**base, **s}[k] for s in sets], np.int32 if k == "top_k" else np.float32) for k in base}
    tok, ch, pr, s = run(logits, u, cols)
    check(logits, u, pr, tok, ch, 1, **cols)
    for _ in range(3):
        t2, c2, p2, _ = run(logits, u, cols, sampler=s)
        assert torch.equal(tok, t2) and torch.equal(ch, c2) and torch.equal(pr, p2)


@pytest.mark.parametrize("V", [5000, 128256, 1000003])
def test_tokens_at_the_end_of_the_window(V):
    """Logits 31.5 to 32.6 below the largest: those beyond 32 have no part in the
    weight that top_p refers to, not even where it is reached exactly."""
    rng = np.random.default_rng(V)
    sets = [dict(top_p=p, temperature=t) for p in (0.5, 0.25, 0.75) for t in (1.0, 0.25)]
    sets += [dict(top_p=0.5, top_k=k) for k in (3, V // 2)] + [dict(top_p=0.999999), dict(top_k=V // 2), dict(min_p=1e-14)]
    x = np.empty((len(sets), V), np.float32)
    for r, st in enumerate(sets):
        t = st.get("temperature", 1.0)
        lo, hi = ((32.02, 32.2), (31.9, 32.3), (31.5, 32.6))[r % 3]
        x[r] = -rng.uniform(lo, hi, V) * t + (0.0, 7.3, -3.21)[r % 3]
        x[r, rng.choice(V, 4, replace=False)] = (0.0, 7.3, -3.21)[r % 3]
    logits, u = torch.from_numpy(x).to(DEV), torch.from_numpy(rng.random(len(sets), np.float32)).to(DEV)
    base = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)
    cols = {k: np.array([{**base, **s}[k] for s in sets], np.int32 if k == "top_k" else np.float32) for k in base}
    tok, ch, pr, _ = run(logits, u, cols)
    check(logits, u, pr, tok, ch, 1, **cols)


def test_the_largest_vocabulary():
    rng = np.random.default_rng(20)
    V = 1 << 20
    logits = torch.from_numpy(rng.normal(size=(5, V)).astype(np.float32) * 3).to(DEV)
    u = torch.from_numpy(rng.random(5, np.float32)).to(DEV)
    kw = dict(temperature=np.array([1, 1, 0.7, 0, 1.5], np.float32), top_k=np.array([0, 0, 900000, 0, 300], np.int32),
              top_p=np.array([1, 0.9, 0.99, 1, 0.8], np.float32), min_p=np.array([0, 0, 1e-6, 0, 0.01], np.float32))
    tok, ch, pr, s = run(logits, u, kw)
    check(logits, u, pr, tok, ch, 1, **kw)
    assert s.device_error() == 0


def test_a_last_request_of_fewer_rows():
    """Five rows, two a request: the third has one."""
    rng = np.random.default_rng(21)
    rows, V = 5, 3001
    logits = torch.from_numpy(rng.normal(size=(rows, V)).astype(np.float32) * 2).to(DEV)
    u = torch.from_numpy(rng.random(rows, np.float32)).to(DEV)
    s = sampling.Sampler(rows, V, device=DEV)
    k = torch.tensor([1, 40, 7], dtype=torch.int32, device=DEV)
    tok, ch = torch.zeros(rows, dtype=torch.int32, device=DEV), torch.zeros(rows, device=DEV)
    spade._check(s.lib.spade_sample(rows, V, spade.F32, logits.data_ptr(), V, 2, None, None, k.data_ptr(), None, None,
                                    u.data_ptr(), tok.data_ptr(), ch.data_ptr(), None, s._at_ws, s._bytes, s._at_err,
                                    torch.cuda.current_stream().cuda_stream))
    check(logits, u, None, tok, ch, 2, top_k=[1, 40, 7])


def test_captured_draws():
    """A graph whose distribution takes the logits' place, replayed with eager draws of
    other settings in between."""
    rng = np.random.default_rng(22)
    rows, V = 6, 40009
    s, e = (sampling.Sampler(rows, V, device=DEV) for _ in range(2))
    x, u = torch.zeros(rows, V, device=DEV), torch.zeros(rows, device=DEV)
    k = torch.zeros(rows, dtype=torch.int32, device=DEV)
    p = torch.ones(rows, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.draw(x, u, top_k=k, top_p=p, probs=x)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        tok, ch = s.draw(x, u, top_k=k, top_p=p, probs=x)
    for i in range(4):
        logits = torch.from_numpy(rng.normal(size=(rows, V)).astype(np.float32) * (i + 1)).to(DEV)
        x.copy_(logits)
        u.copy_(torch.from_numpy(rng.random(rows, np.float32)))
        k.copy_(torch.from_numpy(rng.integers(0, 3, rows).astype(np.int32) * 60))
        p.copy_(torch.from_numpy(rng.choice([1.0, 0.9, 0.3], rows).astype(np.float32)))
        g.replay()
        e.draw(logits, u, temperature=0.5, min_p=0.1)
        torch.cuda.synchronize()
        check(logits, u, x, tok, ch, 1, top_k=k.tolist(), top_p=p.tolist())


def test_two_graphs_of_one_sampler():
    """Graphs that share a workspace, replayed in turn on one stream, with an eager draw
    of the same sampler in between."""
    rng = np.random.default_rng(23)
    rows, V = 7, 30011
    s = sampling.Sampler(rows, V, device=DEV)
    x, u = torch.zeros(rows, V, device=DEV), torch.zeros(rows, device=DEV)
    sets = [dict(top_k=300, top_p=0.8), dict(top_p=0.97, temperature=2.5), dict(min_p=0.02)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.draw(x, u)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for kw in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = s.draw(x, u, **kw)
        graphs.append((g, out))
    for i in range(3):
        x.copy_(torch.from_numpy(rng.normal(size=(rows, V)).astype(np.float32) * (1 + i)))
        u.copy_(torch.from_numpy(rng.random(rows, np.float32)))
        for (g, (tok, ch)), kw in list(zip(graphs, sets))[::-1 if i % 2 else 1]:
            g.replay()
            s.draw(x, u, temperature=0.0)
            torch.cuda.synchronize()
            check(x, u, None, tok, ch, rows, **{k: [v] for k, v in kw.items()})
    assert s.device_error() == 0


def test_draw_refuses():
    s = sampling.Sampler(4, 100, device=DEV)
    x, u = torch.zeros(4, 100, device=DEV), torch.zeros(4, device=DEV)
    for bad in (lambda: s.draw(x.half(), u), lambda: s.draw(x.cpu(), u), lambda: s.draw(x[0], u),
                lambda: s.draw(torch.zeros(5, 100, device=DEV), torch.zeros(5, device=DEV)),
                lambda: s.draw(torch.zeros(4, 101, device=DEV), u), lambda: s.draw(x, u[:3]),
                lambda: s.draw(x, u.double()), lambda: s.draw(x, u, top_k=torch.zeros(2, device=DEV)),
                lambda: s.draw(x, u, temperature=torch.zeros(3, device=DEV)),
                lambda: s.draw(x, u, temperature=torch.ones(2, device=DEV), top_p=torch.ones(4, device=DEV)),
                lambda: s.draw(x.t(), u), lambda: s.draw(x, u, probs=torch.zeros(4, 99, device=DEV))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(spade.SpadeError):
        s.draw(x[:0], u[:0])
    with pytest.raises(spade.SpadeError):
        sampling.Sampler(1, 1, device=DEV)


def test_two_threads_of_one_sampler():
    """Each on the default stream with its own rows and numbers: the draws that it has alone."""
    import threading
    rng = np.random.default_rng(12)
    s = sampling.Sampler(6, 20000, device=DEV)
    jobs = []
    for kw in (dict(top_k=40, temperature=0.7), dict(top_p=0.8, min_p=0.01)):
        x = torch.from_numpy(rng.normal(size=(6, 20000)).astype(np.float32) * 3).to(DEV)
        u = torch.from_numpy(rng.random(6, np.float32)).to(DEV)
        jobs.append((x, u, kw, [t.clone() for t in s.draw(x, u, **kw)]))
    torch.cuda.synchronize()
    got = [[], []]

    def run(i):
        for _ in range(20):
            got[i].append(s.draw(jobs[i][0], jobs[i][1], **jobs[i][2]))

    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for (_, _, _, (tok, ch)), draws in zip(jobs, got):
        assert len(draws) == 20
        for a, b in draws:
            assert torch.equal(a, tok) and torch.equal(b, ch)
