"""Models whose K/V cache is held in 4 bits: verify, prefill, head norms,
running weights and eviction against the float64 oracle (oracle/kvq.py,
QuantDecoder).

A key or value enters the quantiser up to 2^-14 of its row's largest entry off
(activations in two bf16 terms, 2^-17 each, through a projection), which now
and then changes a code, or the rounding of a whole row's minimum or scale; the
float64 decoder itself, its rows moved by 1e-5 before they are quantised, moves
its logits by up to 0.3 on these shapes.  So the two sides are not compared
through their own caches: the oracle takes the rows that the device stored,
after checking that each is what the definition allows for its own value,
and everything behind them (attention over the cache, projections, logits,
weights) has to meet the usual bars: logits 5e-2 (bf16 weights) or 1e-4 (float32),
and decisions wherever the measured logit error cannot turn them.
"""

from dataclasses import replace

import numpy as np
import pytest
import torch

from oracle import kvq as okvq
from oracle import verify as oracle_verify
from paper_2608_13076_amd import spade
from synth import ModelWeights, make_inputs, mini_workloads
from tests.helpers import LOGIT_TOL, OracleRun, compare, gpu_prefill, gpu_setup, gpu_verify, report_parity

pytestmark = pytest.mark.gpu
MINIS = {w.name: w for w in mini_workloads()}


def i4(name):
    w = MINIS[name]
    return w.with_(model=replace(w.model, kv_dtype="i4"))


def gains(w, on):
    if not on:
        return None, None
    rng = np.random.default_rng(w.seed + 5)
    s = w.model
    return [(1 + 0.2 * rng.normal(size=(s.n_layers, s.head_dim))).astype(np.float32) for _ in range(2)]


def device_rows(kv, n):
    """K and V [n_layers][batch, n, KV heads, hd] as the model's cache holds them."""
    m = kv.model.shape
    sh = spade.KVQShape(m.n_layers, kv.max_batch, m.n_heads, m.kv_heads, m.head_dim, kv.max_len)
    out = []
    for l in range(m.n_layers):
        k = torch.empty((kv.max_batch, n, m.kv_heads, m.head_dim), device="cuda:0")
        v = torch.empty_like(k)
        st = kv.lib.spade_kvq_read(sh, l, kv.buf.data_ptr(), kv.max_batch, n, None, None, spade.F32, k.data_ptr(),
                                   v.data_ptr(), torch.cuda.current_stream().cuda_stream)
        assert st == 0
        out.append((k.cpu().numpy().astype(np.float64), v.cpu().numpy().astype(np.float64)))
    return out


class Given(okvq.QuantDecoder):
    """The oracle over the rows that the device stored (``rows`` from
    device_rows, request ``b`` an attribute of the cache)."""

    rows = None
    near = 2.0 ** -14

    def stored(self, l, cache, k, v):
        L, R = cache.length, k.shape[0]
        out = []
        for x, dev in zip((k, v), self.rows[l]):
            d = dev[cache.b, L:L + R]
            _, s, m = okvq.codes(x)
            # half a step, the rounding of minimum and scale, and the value's own error
            tol = s / 2 + 2.0 ** -8 * (np.abs(m) + 15 * s) + self.near * np.abs(x).max(-1, keepdims=True)
            assert (np.abs(d - x) <= tol).all(), (l, cache.b, np.abs(d - x).max())
            out.append(d)
        return out


def setup(name, norms=False, max_len=None):
    w = i4(name)
    weights = ModelWeights(w.model, w.seed)
    model, kv = gpu_setup(w, weights, max_len=max_len)
    gq, gk = gains(w, norms)
    if norms:
        model.set_head_norms(torch.from_numpy(gq).cuda(), torch.from_numpy(gk).cuda(), 1e-6)
    dec = Given(w.model, weights.get, gq, gk, 1e-6, keep_f64=True)
    return w, model, kv, dec


def caches_of(w, dec, inp, kv, weights=False):
    """The oracle's prefilled caches, over the device's rows."""
    dec.rows = device_rows(kv, kv.max_len)
    out = []
    for b in range(w.batch):
        c = dec.new_cache(kv.max_len)
        c.b = b
        if weights:
            c.weights = [np.zeros((w.model.kv_heads, kv.max_len)) for _ in range(w.model.n_layers)]
        dec.prefill(c, inp.prompts[b][:-1])
        out.append(c)
    return out


@pytest.mark.parametrize("norms", [False, True])
@pytest.mark.parametrize("batch", [False, True])
@pytest.mark.parametrize("name", ["mini_f32_greedy", "mini_bf16_greedy", "mini_bf16_sample", "mini_bf16_mixed",
                                  "mini_bf16_wide_b5", "mini_gqa_greedy", "mini_gqa_mixed_b5"])
def test_verify_matches_the_oracle(name, batch, norms):
    w, model, kv, dec = setup(name, norms)
    tol = LOGIT_TOL[w.model.weight_dtype]
    inp = make_inputs(w)
    if batch:
        kv.prefill_batch([np.asarray(p) for p in inp.prompts])
    else:
        gpu_prefill(kv, inp)
    lens, pending = kv.get_state(w.batch)
    assert lens.tolist() == [len(p) - 1 for p in inp.prompts]
    # drafts that the device itself would go on with (half of them, greedy requests)
    caches = caches_of(w, dec, inp, kv)
    rng = np.random.default_rng(w.seed)
    for b in range(w.batch):
        if inp.recipe[b] == "chain_half":
            inp.drafts[b] = rng.integers(0, w.model.vocab, w.gamma)
    first = gpu_verify(model, kv, inp)
    for b in range(w.batch):
        if inp.recipe[b] == "chain_half":
            inp.drafts[b, 0] = first[0][b, 0].argmax()
    outs = [gpu_verify(model, kv, inp) for _ in range(2)]  # idempotent
    assert np.array_equal(outs[0][0].view(np.uint32), outs[1][0].view(np.uint32))
    lg, n, c, _ = outs[1]
    dec.rows = device_rows(kv, kv.max_len)
    res = [oracle_verify(dec, caches[b], inp.pending[b], inp.drafts[b],
                         inp.draft_probs[b] if inp.modes[b] == 1 else None, inp.uniforms[b], int(inp.modes[b]),
                         inp.temperature) for b in range(w.batch)]
    p = compare(OracleRun(inp, res, caches), lg, n, c)
    report_parity(f"i4 {name} norms {norms} batch {batch}",
                  dict(logit_err=round(p.logit_err, 6), stable=p.stable_n, total=p.total, n_match=p.n_match_all))
    assert p.logit_err <= tol
    assert not p.stable_n_fail and not p.stable_corr_fail and p.stable_n > 0
    assert model.device_error() == 0


def test_head_norms_matter_and_turn_off():
    w, model, kv, _ = setup("mini_bf16_greedy")
    inp = make_inputs(w)
    gpu_prefill(kv, inp)
    a = gpu_verify(model, kv, inp)[0]
    g = torch.full((w.model.n_layers, w.model.head_dim), 1.5, device="cuda:0")
    model.set_head_norms(g, g)
    b = gpu_verify(model, kv, inp)[0]
    model.set_head_norms(None, None)
    c = gpu_verify(model, kv, inp)[0]
    assert np.abs(a - b).max() > 1e-3 and np.array_equal(a, c)


def test_only_4_bit_models_take_these_calls():
    w = MINIS["mini_bf16_greedy"]
    model, kv = gpu_setup(w)
    g = torch.ones((w.model.n_layers, w.model.head_dim), device="cuda:0")
    wt = torch.zeros((w.model.n_layers, 1, w.model.kv_heads, kv.max_len), device="cuda:0")
    for call in (lambda: model.set_head_norms(g, g), kv.track_weights, lambda: kv.evict(1, 8, 2)):
        with pytest.raises(spade.SpadeError) as e:
            call()
        assert e.value.status == -4
    w, model, kv, _ = setup("mini_bf16_greedy")
    for call in (lambda: kv.evict(1, 8, 2), lambda: model.set_head_norms(g, None), lambda: model.set_head_norms(g, g, -1.0)):
        with pytest.raises(spade.SpadeError) as e:
            call()
        assert e.value.status == -1
    kv.track_weights()
    for a in ((1, 0, 0), (1, kv.max_len + 1, 0), (2, 8, 2), (1, 8, 9), (1, 8, -1)):
        with pytest.raises(spade.SpadeError):
            kv.evict(*a)
    with pytest.raises(ValueError):
        model.set_head_norms(g[:1], g)


def drop(cache, kept, n):
    """The oracle's cache after an eviction that kept these positions."""
    for l in range(cache.n_layers):
        for a in range(cache.k[l].shape[0]):
            idx = kept[l, a][kept[l, a] >= 0]
            for t in (cache.k[l], cache.v[l], cache.weights[l]):
                t[a, :len(idx)] = t[a, idx]
    m = int((kept[0, 0] >= 0).sum())
    cache.shift = getattr(cache, "shift", 0) + n - m
    cache.length = m


@pytest.mark.parametrize("name,norms", [("mini_bf16_greedy", False), ("mini_gqa_mixed_b5", True), ("mini_f32_greedy", True)])
def test_weights_and_eviction_rounds(name, norms):
    """Prompt, then rounds of verify, commit and (every second one) an eviction
    to half of what is cached: logits of every round against the oracle, whose
    caches lose the positions that the device's weights chose.  The weights
    follow from scores of size 10 at most whose queries are 2^-14 off: every
    probability within 10 2^-14 sqrt(2), taken as 2e-3 of it."""
    w, model, kv, dec = setup(name, norms)
    tol = LOGIT_TOL[w.model.weight_dtype]
    inp = make_inputs(w)
    W = kv.track_weights()
    kv.prefill_batch([np.asarray(p) for p in inp.prompts])
    caches = caches_of(w, dec, inp, kv, weights=True)
    rng = np.random.default_rng(1)
    pending = [int(x) for x in inp.pending]
    for rnd in range(5):
        drafts = rng.integers(0, w.model.vocab, (w.batch, w.gamma)).astype(np.int32)
        buf = spade.VerifyBuffers(model, drafts, None, None, np.zeros(w.batch, np.uint8), True)
        spade.verify(model, kv, buf)
        lg, n, corr = buf.logits.cpu().numpy(), buf.n.cpu().numpy(), buf.corr.cpu().numpy()
        dec.rows = device_rows(kv, kv.max_len)
        kv.commit(buf.n, buf.corr)
        dec.count = 1
        for b, c in enumerate(caches):
            L = c.length
            want = dec.forward(c, [pending[b]] + drafts[b].tolist())
            assert np.abs(lg[b] - want).max() <= tol, (rnd, b)
            c.length = L + int(n[b]) + 1
            pending[b] = int(corr[b])
        lens, _ = kv.get_state(w.batch)
        assert lens.tolist() == [c.length for c in caches]
        for l in range(w.model.n_layers):
            for b, c in enumerate(caches):
                got, want = W[l, b, :, :c.length].cpu().numpy(), c.weights[l][:, :c.length]
                assert (np.abs(got - want) <= 2e-3 * want + 1e-6).all(), (rnd, l, b)
        if rnd % 2 == 1:
            budget = max(2, int(max(lens)) // 2)
            recent = min(4, budget)
            before = W.cpu().numpy()
            kept = kv.evict(w.batch, budget, recent).cpu().numpy()
            for b, c in enumerate(caches):
                for l in range(w.model.n_layers):
                    for a in range(w.model.kv_heads):
                        want = okvq.keep(before[l, b, a], c.length, budget, recent)
                        assert kept[l, b, a][kept[l, b, a] >= 0].tolist() == want.tolist()
                drop(c, kept[:, b], c.length)
            lens, _ = kv.get_state(w.batch)
            assert lens.tolist() == [c.length for c in caches]
    assert model.device_error() == 0


def test_positions_and_snapshots_after_eviction():
    """The cache is short, the sequence goes on to the model's max_len and not
    beyond; a snapshot does not survive an eviction; length 0 starts over."""
    w = i4("mini_bf16_greedy")
    model, _ = gpu_setup(w, max_len=200)
    kv = spade.KVCache(model, 1, 60)
    kv.track_weights()
    rng = np.random.default_rng(0)
    kv.prefill(0, rng.integers(0, 4001, 51))
    snap = kv.snapshot(1)
    total = 50
    mode = np.zeros(1, np.uint8)

    def step():
        buf = spade.VerifyBuffers(model, np.zeros((1, 4), np.int32), None, None, mode, False)
        spade.verify(model, kv, buf)
        kv.commit(buf.n, buf.corr)
        return int(buf.n.item()) + 1

    total += step()
    kv.restore(*snap)
    total = 50
    kv.evict(1, 20, 5)
    with pytest.raises(spade.SpadeError):
        kv.restore(*snap)
    while total + 5 <= 200:
        try:
            total += step()
        except spade.SpadeError as e:
            assert e.status == -2
            lens = int(kv.get_state(1)[0][0])
            assert lens + 5 > 60  # the cache is full, not the positions
            kv.evict(1, 20, 5)
    with pytest.raises(spade.SpadeError) as e:
        kv.evict(1, 20, 5)
        step()
    assert e.value.status == -2
    assert model.device_error() == 0
    kv.set_state([0], [0])
    kv.prefill(0, rng.integers(0, 4001, 51))
    step()
    assert model.device_error() == 0


def test_a_snapshot_does_not_survive_a_restart():
    """A request with evicted positions that starts over forgets them, and its
    snapshot's rows counted them."""
    w = i4("mini_bf16_greedy")
    model, _ = gpu_setup(w, max_len=200, max_batch=2)
    kv = spade.KVCache(model, 2, 60)
    kv.track_weights()
    rng = np.random.default_rng(0)
    for b in (0, 1):
        kv.prefill(b, rng.integers(0, 4001, 41))
    kv.evict(1, 20, 5)
    snap = kv.snapshot(2)
    kv.set_state([18, 0], [1, 1])
    kv.restore(*snap)  # request 1 never lost a position
    kv.set_state([0, 0], [0, 0])
    with pytest.raises(spade.SpadeError) as e:
        kv.restore(*snap)
    assert e.value.status == -1


def test_head_norms_refuse_strided_gains():
    w, model, kv, _ = setup("mini_bf16_greedy")
    g = torch.ones((w.model.n_layers, 2 * w.model.head_dim), device="cuda:0")[:, ::2]
    with pytest.raises(ValueError):
        model.set_head_norms(g, g.contiguous())


def test_batched_prefill_stores_the_same_first_layer():
    """Ragged prompts at once or one by one: the first layer's rows do not see
    the attention, so they are the same bits; placeholder rows are not stored."""
    w = i4("mini_gqa_mixed_b5")
    weights = ModelWeights(w.model, w.seed)
    inp = make_inputs(w)
    model, a = gpu_setup(w, weights)
    b = spade.KVCache(model, w.batch, a.max_len)
    for kv in (a, b):
        kv.buf[:-256].fill_(255)
    gpu_prefill(a, inp)
    b.prefill_batch([np.asarray(p) for p in inp.prompts])
    n = w.batch * w.model.kv_heads * ((a.max_len + 31) // 32) * 32 * (w.model.head_dim + 8)
    assert torch.equal(a.buf[:n], b.buf[:n])


@pytest.mark.parametrize("name", ["mini_bf16_mixed", "mini_gqa_mixed_b5", "mini_f32_greedy"])
def test_captured_verify_replays_match_eager(name):
    w, model, kv, _ = setup(name, True)
    inp = make_inputs(w)
    kv.prefill_batch([np.asarray(p) for p in inp.prompts])
    ref = gpu_verify(model, kv, inp)
    buf = spade.VerifyBuffers(model, inp.drafts, inp.draft_probs, inp.uniforms, inp.modes, True)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            spade.verify(model, kv, buf, inp.temperature)
    torch.cuda.synchronize()
    for i in range(4):
        buf.logits.zero_()
        buf.n.fill_(-1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(buf.logits.cpu().numpy().view(np.uint32), ref[0].view(np.uint32)), i
        assert np.array_equal(buf.n.cpu().numpy(), ref[1])
        assert np.array_equal(gpu_verify(model, kv, inp)[0].view(np.uint32), ref[0].view(np.uint32)), i


def test_algorithm1_over_4_bit_caches():
    """The loop of the paper with target and early-exit draft on 4-bit caches:
    greedy, it emits the target's own tokens."""
    from paper_2608_13076_amd import algorithm1 as alg
    w = i4("mini_bf16_wide_b5")
    prompt = np.random.default_rng(3).integers(0, w.model.vocab, 90).astype(np.int32)
    u = np.random.default_rng(4).random(4000, dtype=np.float32)
    target = alg.load_model(w.model, w.seed, 160, 4)
    draft = alg.load_model(w.model, w.seed, 160, 4, n_layers=1)
    base = alg.run_target_only(target, prompt, 24, 0, u)
    got = alg.run_algorithm1(target, draft, prompt, 3, 24, 0, u)
    # (rows of one call and rows one by one differ in their last bits: a token may only
    # differ where the two best logits are as near, which 24 tokens of this model do not meet)
    assert got.tokens == base.tokens and got.calls <= 24
