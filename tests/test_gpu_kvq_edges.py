"""4-bit K/V caches at the ends of what their calls allow: bounds below the
padded rows, captured calls over growing lengths, host bounds after evictions,
rows and queries near the ends of float32, and the precision of outputs and
running weights.

Precision.  Errors are taken as 2-norms over a request's rows in use.  With
scores of at most 16 (in units of log2) a float32 evaluation of the formulas is
off by: the exponent's argument and the log-sum-exp, half a step of numbers up
to 16 each, 2^-21 ln 2 = 3.3e-7; a score of 128 products in three terms, some
roundings of 2^-24 of sums below 16, 3e-7 in all as they have either sign; the
exponential and the quotient, 2^-23 each.  Together below 1e-6 of an output's
size, and of the size of a head's weights.  bfloat16 outputs add their own half
step, 2^-8 of the element; the probabilities times scales enter in 16 bits, half
a step 2^-17 of a term |n - 7.5| s <= 7.5 s_max.
"""

from dataclasses import replace

import numpy as np
import pytest
import torch

from oracle import kvq as okvq
from paper_2608_13076_amd import kvq, spade
from synth import ModelWeights, make_inputs, workload
from tests.helpers import LOGIT_TOL, gpu_setup
from tests.test_gpu_kvq import DEV, check_attend, f64, fill, i32, poison, rand
from tests.test_gpu_kvq_model import Given, caches_of, device_rows, gains, i4

pytestmark = pytest.mark.gpu


def check(q, k, v, lens, rows, out, dtype, weights=None, w_out=None, wr=0):
    """Outputs and weights of the requests against the oracle over the held
    rows, to the bounds above; rows that are not in use are zeros."""
    b, R, H, hd = q.shape
    KVH = k.shape[2]
    for i in range(b):
        n, end = rows[i], lens[i] + rows[i]
        assert not out[i, n:].any()
        want_w = f64(weights[i, :, :end]) if weights is not None else np.zeros((KVH, end))
        if n:
            kk, vv = okvq.held(f64(k[i, :end])), okvq.held(f64(v[i, :end]))
            o, p = okvq.attend(f64(q[i, :n]), kk, vv, lens[i], hd ** -0.5)
            err = f64(out[i, :n]) - o
            if dtype == "f32":
                assert np.linalg.norm(err) <= 1e-6 * np.linalg.norm(o), (i, np.linalg.norm(err) / np.linalg.norm(o))
            else:
                _, s, _ = okvq.codes(f64(v[i, :end]))
                inner = 7.5 * s.max() * 2.0 ** -17 + 4e-6 * np.abs(vv).max()
                assert (np.abs(err) <= 2.0 ** -8 * (np.abs(o) + inner) + inner).all(), (i, np.abs(err).max())
            want_w = want_w + p[:min(wr, n)].sum(0).reshape(KVH, H // KVH, end).sum(1)
        if w_out is not None:
            d = f64(w_out[i, :, :end]) - want_w
            # (and half a step of the running weights themselves)
            assert np.linalg.norm(d) <= (1e-6 + 2.0 ** -24) * np.linalg.norm(want_w), (i, np.linalg.norm(d) / np.linalg.norm(want_w))


# --- the bound of an attention call ---------------------------------------

SHORT = [
    # lens, rows, R, max_len, max_keys
    ([4], [3], 8, 40, 7),
    ([0, 1], [6, 1], 8, 40, 6),
    ([3, 0], [2, 0], 5, 40, 5),
    ([0, 0, 0], [1, 0, 2], 16, 40, 2),
    ([0], [1], 16, 1, 0),          # a cache shorter than the padded rows
    ([2, 5], [3, 0], 16, 5, 0),
    ([0] * 20, [1 + i % 3 for i in range(20)], 9, 33, 3),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("hd,h,kvh", [(128, 8, 2), (64, 3, 3)])
@pytest.mark.parametrize("lens,rows,R,max_len,max_keys", SHORT)
def test_attend_bound_below_the_padded_rows(lens, rows, R, max_len, max_keys, hd, h, kvh, weights, dtype):
    """max_keys bounds the rows in use: a ragged batch of short contexts has a
    bound below R, and a cache may be shorter than R."""
    rng = np.random.default_rng(R + max_len)
    b = len(lens)
    cache = kvq.QuantCache(1, b, h, kvh, hd, max_len, max_rows=R, device=DEV)
    poison(cache)
    n = max(a + c for a, c in zip(lens, rows))
    k, v = rand(rng, b, n, kvh, hd, dtype=dtype), rand(rng, b, n, kvh, hd, dtype=dtype)
    fill(cache, 0, k, v, rows=i32([a + c for a, c in zip(lens, rows)]))
    cache.lens.copy_(i32(lens))
    q = rand(rng, b, R, h, hd, dtype=dtype, strong=False)
    kw, w, wo = {}, None, None
    if weights:
        w = rand(rng, b, kvh, max_len, strong=False).abs()
        wo = torch.full_like(w, -3.0)
        kw = dict(weights=w, weights_out=wo, weight_rows=R)
    out = cache.attend(0, q, rows=i32(rows), max_keys=max_keys, **kw)
    assert cache.device_error() == 0
    check_attend(q, k, v, lens, rows, out, hd ** -0.5, dtype, w, wo, R, torch.full_like(wo, -3.0) if weights else None)


def test_attend_rows_beyond_the_bound_are_cut_and_flagged():
    """More rows in use than the bound: the first max_keys of them over the
    empty cache, zeros behind; with a length, the length is cut first."""
    rng = np.random.default_rng(4)
    cache = kvq.QuantCache(1, 3, 4, 2, 128, 30, max_rows=8, device=DEV)
    k, v = rand(rng, 3, 30, 2, 128), rand(rng, 3, 30, 2, 128)
    fill(cache, 0, k, v)
    q = rand(rng, 3, 8, 4, 128, strong=False)
    for lens in ([0, 9, -2], [2, 0, 2**31 - 1]):
        cache.lens.copy_(i32(lens))
        w = torch.zeros((3, 2, 30), device=DEV)
        out = cache.attend(0, q, rows=i32([8, 7, 8]), max_keys=5, weights_out=w, weight_rows=8)
        assert cache.device_error() == spade.DERR_CAPACITY
        check_attend(q, k, v, [0, 0, 0], [5, 5, 5], out, 128 ** -0.5, "f32", None, w, 8)
        assert not w[:, :, 5:].any()
    with pytest.raises(spade.SpadeError):  # without rows all R are in use
        cache.attend(0, q, max_keys=5)
    with pytest.raises(spade.SpadeError):
        cache.attend(0, q, rows=i32([1, 1, 1]), max_keys=31)
    with pytest.raises(spade.SpadeError):
        cache.attend(0, q, rows=i32([1, 1, 1]), max_keys=-1)


# --- captured verify calls ------------------------------------------------


@pytest.mark.parametrize("name", ["mini_bf16_mixed", "mini_gqa_mixed_b5", "mini_f32_greedy"])
def test_captured_verify_covers_growing_lengths(name):
    """One graph of a verify call, replayed after commits that move the lengths
    on: every replay equals the eager call at the same lengths (contexts of one
    attention part per head, whose bits do not depend on the bound)."""
    w = i4(name)
    model, kv = gpu_setup(w, max_len=200)
    W = kv.track_weights()
    rng = np.random.default_rng(2)
    kv.prefill_batch([rng.integers(0, w.model.vocab, 40 + 3 * b).astype(np.int32) for b in range(w.batch)])
    inp = make_inputs(w)
    buf = spade.VerifyBuffers(model, inp.drafts, inp.draft_probs, inp.uniforms, inp.modes, True)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            spade.verify(model, kv, buf, inp.temperature)
    torch.cuda.synchronize()
    R = w.gamma + 1
    n = torch.full((w.batch,), w.gamma, dtype=torch.int32, device=DEV)
    top = 39 + 3 * (w.batch - 1)
    while top + R <= 128:
        before = W.clone()
        graph.replay()
        torch.cuda.synchronize()
        got, got_w = buf.logits.clone(), W.clone()
        W.copy_(before)
        buf.logits.zero_()
        spade.verify(model, kv, buf, inp.temperature)
        torch.cuda.synchronize()
        assert torch.equal(got, buf.logits), top
        assert torch.equal(got_w, W), top
        kv.commit(n, buf.corr)
        top += R
    assert model.device_error() == 0


# --- host bounds after evictions ------------------------------------------


def drifted():
    """A model of 200 positions over a cache of 60: 30 rounds of verify, commit
    of no draft and eviction, whose host bound counts five positions each where
    one was evicted."""
    model, _ = gpu_setup(i4("mini_bf16_greedy"), max_len=200)
    kv = spade.KVCache(model, 1, 60)
    kv.track_weights()
    rng = np.random.default_rng(0)
    kv.prefill(0, rng.integers(0, 4001, 41).astype(np.int32))
    none = torch.zeros(1, dtype=torch.int32, device=DEV)
    for _ in range(30):
        buf = spade.VerifyBuffers(model, np.zeros((1, 4), np.int32), None, None, np.zeros(1, np.uint8), False)
        spade.verify(model, kv, buf)
        kv.commit(none, none)
        kv.evict(1, 40, 5)
    return model, kv, rng.integers(0, 4001, 131).astype(np.int32)


@pytest.mark.parametrize("how", ["prefill", "get_state and prefill", "batch"])
def test_prompts_after_evictions_fit_where_there_is_room(how):
    model, kv, ids = drifted()
    if how == "get_state and prefill":
        assert kv.get_state(1)[0].tolist() == [40]
    if how == "batch":
        kv.prefill_batch([ids[:15]])
    else:
        kv.prefill(0, ids[:15])
    assert kv.get_state(1)[0].tolist() == [54]
    assert model.device_error() == 0


def test_a_refusal_leaves_a_capture_as_it_is():
    """A capture cannot wait for the device's counts: the call is refused by the
    host's bound, the capture goes on, and outside of it the call fits."""
    model, kv, ids = drifted()
    none = torch.zeros(1, dtype=torch.int32, device=DEV)
    buf = spade.VerifyBuffers(model, np.zeros((1, 4), np.int32), None, None, np.zeros(1, np.uint8), False)
    spade.verify(model, kv, buf)
    kv.commit(none, none)
    kv.evict(1, 40, 5)  # the bound: 40 cached, 155 evicted
    wide = spade.VerifyBuffers(model, np.zeros((1, 5), np.int32), None, None, np.zeros(1, np.uint8), False)
    x = torch.zeros(8, device=DEV)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            x.add_(1)
            with pytest.raises(spade.SpadeError) as e:
                spade.verify(model, kv, wide)
            x.add_(1)
    torch.cuda.synchronize()
    assert e.value.status == -2
    for i in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert (x == 2 * (i + 1)).all()
    spade.verify(model, kv, wide)
    torch.cuda.synchronize()
    assert model.device_error() == 0


def test_get_state_brings_both_bounds_in_line():
    """After it a call needs no refresh: it fits in a capture too."""
    model, kv, ids = drifted()
    none = torch.zeros(1, dtype=torch.int32, device=DEV)
    buf = spade.VerifyBuffers(model, np.zeros((1, 4), np.int32), None, None, np.zeros(1, np.uint8), False)
    spade.verify(model, kv, buf)
    kv.commit(none, none)
    kv.evict(1, 40, 5)
    wide = spade.VerifyBuffers(model, np.zeros((1, 5), np.int32), None, None, np.zeros(1, np.uint8), True)
    assert kv.get_state(1)[0].tolist() == [40]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            spade.verify(model, kv, wide)
    torch.cuda.synchronize()
    spade.verify(model, kv, wide)
    want = wide.logits.clone()
    for _ in range(3):
        wide.logits.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(wide.logits, want)
    assert model.device_error() == 0


def test_refusals_name_what_ran_out():
    model, kv, ids = drifted()
    for call in (lambda: kv.prefill(0, ids[:30]), lambda: kv.prefill_batch([ids[:30]])):
        with pytest.raises(spade.SpadeError) as e:
            call()
        assert e.value.status == -2 and "60" in str(e.value)  # the cache
    big = spade.KVCache(model, 1, 190)
    big.track_weights()
    big.prefill(0, ids)
    big.evict(1, 10, 2)  # 120 of 130 positions
    for call in (lambda: big.prefill(0, ids[:71]), lambda: big.prefill_batch([ids[:71]])):
        with pytest.raises(spade.SpadeError) as e:
            call()
        assert e.value.status == -2 and "200 positions" in str(e.value)
    big.prefill(0, ids[:70])
    buf = spade.VerifyBuffers(model, np.zeros((1, 4), np.int32), None, None, np.zeros(1, np.uint8), False)
    with pytest.raises(spade.SpadeError) as e:
        spade.verify(model, big, buf)
    assert e.value.status == -2 and "200 positions" in str(e.value)


# --- ends of float32 ------------------------------------------------------


@pytest.mark.parametrize("hd", [64, 128])
def test_rows_whose_minimum_is_beyond_bfloat16_are_nan(hd):
    """max - m of a row above the largest bfloat16 is not finite: NaN, as the
    header says; next to it, rows that bfloat16 holds."""
    x = np.full((4, 1, hd), 3.4e38, np.float32)
    x[1, 0, ::2] = 3.398e38
    x[2] = 3.389e38
    x[3] = -3.4e38
    t = torch.from_numpy(x)[None].to(DEV)
    cache = kvq.QuantCache(1, 1, 1, 1, hd, 4, device=DEV)
    cache.append(0, t, t)
    for got in cache.read(0, 4):
        got = got[0].cpu().numpy()
        assert np.isnan(got[[0, 1, 3]]).all()
        np.testing.assert_array_equal(got[2], okvq.held(x[2]).astype(np.float32))
    want = okvq.held(x)
    assert np.isnan(want[[0, 1, 3]]).all() and np.isfinite(want[2]).all()


# --- norms of queries -----------------------------------------------------


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
@pytest.mark.parametrize("e", [-110, -70, 0, 64, 100, 120])
def test_queries_are_normed_over_the_range_of_float32(e, eps, dtype):
    """Squares of 2^70 leave float32, the norm does not.  The result is rounded
    once: half a step of its type."""
    rng = np.random.default_rng(e + 200)
    hd = 128
    cache = kvq.QuantCache(1, 2, 4, 2, hd, 20, device=DEV)
    q, k = rand(rng, 2, 5, 4, hd, dtype=dtype) * 2.0 ** e, rand(rng, 2, 5, 2, hd, dtype=dtype)
    g, tab = rand(rng, hd), kvq.rope_table(20, hd, 10000.0, DEV)
    out = f64(cache.append(0, k, k, q=q, gain_q=g, gain_k=g, eps=eps, rope=tab))
    eps = float(np.float32(eps))
    for b in (0, 1):
        for i in range(5):
            want = okvq.norm_rotate(f64(q[b, i]), f64(g), eps, f64(tab)[i])
            # (a result rounded to float32 first: 2^-24 more)
            half = 2.0 ** -24 if dtype == "f32" else 2.0 ** -8 + 2.0 ** -23
            tol = half * np.abs(want) + 2.0 ** -40 * np.abs(want).max() + (2.0 ** -149 if dtype == "f32" else 2.0 ** -133)
            assert (np.abs(out[b, i] - want) <= tol).all(), (e, eps)


# --- precision ------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,r,h,kvh,hd,most", [
    (16, 2, 16, 8, 128, 2500),  # ranges over the batch, several heads each
    (70, 1, 4, 2, 64, 2300),    # more requests than a wave has lanes
    (3, 16, 16, 2, 128, 2000),  # equal parts, tiles of 16 rows
    (16, 3, 16, 8, 128, 1300),  # whole heads of a workgroup
    (12, 16, 6, 1, 64, 700),
    (1, 16, 1, 1, 128, 600),
    (1, 2, 8, 2, 128, 30000),   # a long request
    (2, 9, 8, 2, 128, 200),     # one part per head
])
def test_outputs_and_weights_are_as_precise_as_float32(b, r, h, kvh, hd, most, dtype):
    """Whichever way the heads are divided; every row counted into the weights."""
    rng = np.random.default_rng(b + r + most)
    lens = [int(x) for x in rng.integers(most // 8, most, b)]
    lens[-1] = most
    rows = [int(x) for x in rng.integers(0, r + 1, b)]
    rows[-1] = r
    cache = kvq.QuantCache(1, b, h, kvh, hd, most + r, max_rows=r, device=DEV)
    k, v = rand(rng, b, most + r, kvh, hd, dtype=dtype), rand(rng, b, most + r, kvh, hd, dtype=dtype)
    fill(cache, 0, k, v, rows=i32([a + c for a, c in zip(lens, rows)]))
    cache.lens.copy_(i32(lens))
    q = rand(rng, b, r, h, hd, dtype=dtype, strong=False)
    w = rand(rng, b, kvh, cache.max_len, strong=False).abs() * 1e-3
    wo = torch.empty_like(w)
    out = cache.attend(0, q, rows=i32(rows), weights=w, weights_out=wo, weight_rows=r)
    assert cache.device_error() == 0
    check(q, k, v, lens, rows, out, dtype, w, wo, r)


@pytest.mark.parametrize("mul", [4, 32, 256])
def test_precision_of_large_scores(mul):
    """Float32 scores beyond 11: the products' sum, the minimum's term, the sum of
    both and the scale are half a step of the largest score each, 2^-22 of it
    together, which is what a probability moves by."""
    rng = np.random.default_rng(mul)
    n, hd = 1500, 128
    cache = kvq.QuantCache(1, 2, 8, 2, hd, n + 3, max_rows=3, device=DEV)
    k, v = rand(rng, 2, n + 3, 2, hd), rand(rng, 2, n + 3, 2, hd)
    fill(cache, 0, k, v)
    cache.lens.fill_(n)
    q = rand(rng, 2, 3, 8, hd, strong=False) * mul
    w = torch.zeros((2, 2, n + 3), device=DEV)
    out = cache.attend(0, q, weights_out=w, weight_rows=3)
    for b in (0, 1):
        kk, vv = okvq.held(f64(k[b])), okvq.held(f64(v[b]))
        o, p = okvq.attend(f64(q[b]), kk, vv, n, hd ** -0.5)
        top = max(np.abs(kk[:, h // 4] @ f64(q[b, i, h])).max() for i in range(3) for h in range(8)) * hd ** -0.5
        assert top > 11
        tol = 1e-6 + 2.0 ** -22 * top
        pw = p.sum(0).reshape(2, 4, n + 3).sum(1)
        assert np.linalg.norm(f64(out[b]) - o) <= tol * np.linalg.norm(o)
        assert np.linalg.norm(f64(w[b]) - pw) <= tol * np.linalg.norm(pw)


# --- long contexts in a model ---------------------------------------------


@pytest.mark.parametrize("name,ctx", [("mini_gqa_greedy", (2300, 2300)), ("mini_bf16_mixed", (40, 1500)),
                                      ("mini_f32_greedy", (1000, 1200))])
def test_verify_over_long_contexts(name, ctx):
    """A model's prompts of a thousand positions and more, where the attention's
    heads are divided: logits and the prompts' running weights against the oracle
    over the rows that the device stored.  Weights: scores of size 10 at most
    whose queries are 2^-14 off, 2e-3 of a probability."""
    w = i4(name).with_(ctx=ctx)
    weights = ModelWeights(w.model, w.seed)
    model, kv = gpu_setup(w, weights)
    dec = Given(w.model, weights.get, keep_f64=True)
    W = kv.track_weights()
    inp = make_inputs(w)
    kv.prefill_batch([np.asarray(p) for p in inp.prompts])
    caches = caches_of(w, dec, inp, kv, weights=True)
    rng = np.random.default_rng(3)
    drafts = rng.integers(0, w.model.vocab, (w.batch, w.gamma)).astype(np.int32)
    buf = spade.VerifyBuffers(model, drafts, None, None, np.zeros(w.batch, np.uint8), True)
    spade.verify(model, kv, buf)
    lg = buf.logits.cpu().numpy()
    dec.rows = device_rows(kv, kv.max_len)
    dec.count = 1
    for b, c in enumerate(caches):
        L = c.length
        want = dec.forward(c, [int(inp.pending[b])] + drafts[b].tolist())
        assert np.abs(lg[b] - want).max() <= LOGIT_TOL[w.model.weight_dtype], b
        for l in range(w.model.n_layers):
            got, ww = W[l, b, :, :L + 1].cpu().numpy(), c.weights[l][:, :L + 1]
            assert (np.abs(got - ww) <= 2e-3 * ww + 1e-6).all(), (l, b)
    assert model.device_error() == 0


@pytest.mark.parametrize("name", ["c2_7b_greedy", "gqa_8b_greedy"])
def test_verify_of_full_size_layers(name):
    """Two layers of the 7B and the grouped-query 8B shape (a short vocabulary),
    300 cached positions, head norms on: logits against the oracle over the
    device's rows."""
    w = workload(name).with_(ctx=(300, 300))
    w = w.with_(model=replace(w.model, n_layers=2, vocab=8011, kv_dtype="i4"))
    weights = ModelWeights(w.model, w.seed)
    model, kv = gpu_setup(w, weights)
    gq, gk = gains(w, True)
    model.set_head_norms(torch.from_numpy(gq).cuda(), torch.from_numpy(gk).cuda(), 1e-6)
    dec = Given(w.model, weights.get, gq, gk, 1e-6)
    inp = make_inputs(w)
    kv.prefill_batch([np.asarray(p) for p in inp.prompts])
    c = caches_of(w, dec, inp, kv)[0]
    drafts = np.random.default_rng(3).integers(0, w.model.vocab, (1, w.gamma)).astype(np.int32)
    buf = spade.VerifyBuffers(model, drafts, None, None, np.zeros(1, np.uint8), True)
    spade.verify(model, kv, buf)
    lg = buf.logits.cpu().numpy()
    dec.rows = device_rows(kv, kv.max_len)
    want = dec.forward(c, [int(inp.pending[0])] + drafts[0].tolist())
    assert np.abs(lg[0] - want).max() <= LOGIT_TOL["bf16"]
    assert model.device_error() == 0


# --- the binding ----------------------------------------------------------


def test_append_refuses_an_output_without_queries():
    cache = kvq.QuantCache(1, 1, 4, 2, 64, 8, device=DEV)
    x = torch.zeros((1, 2, 2, 64), device=DEV)
    with pytest.raises(ValueError):
        cache.append(0, x, x, q_out=torch.zeros((1, 2, 4, 64), device=DEV))


def test_evict_of_some_requests_says_so():
    """kept holds -1 for the requests that an eviction of the first B leaves alone."""
    w = i4("mini_gqa_mixed_b5")
    model, kv = gpu_setup(w, max_len=200)
    assert kv.weights is None
    assert kv.track_weights() is kv.weights
    rng = np.random.default_rng(5)
    kv.prefill_batch([rng.integers(0, w.model.vocab, 60).astype(np.int32) for _ in range(5)])
    torch.full((1 << 16,), 77, dtype=torch.int32, device=DEV)  # (freed memory that an allocation may find)
    kept = kv.evict(2, 40, 5)
    assert (kept[:, :2] >= 0).all() and (kept[:, 2:] == -1).all()
    assert kv.get_state(5)[0].tolist() == [40, 40, 59, 59, 59]
