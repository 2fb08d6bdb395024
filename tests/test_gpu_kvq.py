"""4-bit K/V caches on the GPU against the float64 oracle (oracle/kvq.py).

Tolerances.  What the cache holds is compared for equality: keys are normed and
rotated in double on both sides, and a row's minimum, scale and codes follow
exactly.  An attention output o = sum p x moves by

  scores   queries are exact (a float32 one in three bf16 terms, 2^-24); the
           float32 sums of s sum q (16 + n) make at most 40 roundings of terms
           below 31 s |q|:
             dz = scale max_t s_t sum_f |q_f| 31 (40 + 1) 2^-24
           a probability is then off by a factor of at most 1 +- 2.1 dz;
  values   float32 calls hold p s in 24 bits, bf16 calls in one bf16 (half a
           step, 2^-8), and it multiplies |n - 8| <= 8: at most 8 s_max r;
           sums of up to N terms of size 31 s in float32 add
           2^-24 sqrt(N) 31 s, taken as 2^-18 31 s;
  output   bf16: half a step, 2^-8 |o|.
"""

import math

import numpy as np
import pytest
import torch

from oracle import kvq as okvq
from paper_2608_13076_amd import kvq, spade

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TD = {"f32": torch.float32, "bf16": torch.bfloat16}


def rand(rng, *shape, dtype="f32", strong=True):
    x = rng.normal(size=shape).astype(np.float32)
    if strong:
        x[..., 3::17] *= 4
    return torch.from_numpy(x).to(DEV).to(TD[dtype])


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device=DEV)


def fill(cache, layer, k, v, rows=None):
    """Positions 0.. of an empty cache as they stand."""
    cache.lens.zero_()
    cache.append(layer, k, v, rows=rows)


def poison(cache):
    """Every byte 0xff: codes 15, scales and minima NaN."""
    cache.buf.fill_(255)


# --- append and read ------------------------------------------------------

APPEND = [
    # b, r, h, kvh, hd, lens
    (1, 1, 8, 2, 128, [0]),
    (1, 1, 8, 2, 64, [31]),
    (3, 5, 4, 4, 128, [30, 0, 97]),
    (2, 16, 12, 4, 64, [1, 60]),
    (2, 70, 6, 1, 128, [3, 33]),
    (4, 3, 5, 5, 64, [0, 1, 2, 3]),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("norm,rope", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("b,r,h,kvh,hd,lens", APPEND)
def test_append_holds_what_the_definition_gives(b, r, h, kvh, hd, lens, norm, rope, dtype):
    rng = np.random.default_rng(b * 100 + r + hd)
    cache = kvq.QuantCache(2, b, h, kvh, hd, max(lens) + r + 3, device=DEV)
    poison(cache)
    cache.lens.copy_(i32(lens))
    qkv = rand(rng, b, r, h + 2 * kvh, hd, dtype=dtype)  # fused rows: strided views
    q, k, v = qkv[:, :, :h], qkv[:, :, h:h + kvh], qkv[:, :, h + kvh:]
    gq = rand(rng, hd, strong=False) if norm else None
    gk = rand(rng, hd, strong=False) if norm else None
    tab = kvq.rope_table(max(lens) + r, hd, 500000.0, DEV) if rope else None
    rows = [r] + [int(x) for x in rng.integers(0, r + 1, b - 1)]
    out = cache.append(1, k, v, q=q, gain_q=gq, gain_k=gk, eps=1e-6, rope=tab, rows=i32(rows))
    kk, vv = cache.read(1, r, start=cache.lens, rows=i32(rows))
    n = lambda t: None if t is None else f64(t)
    for i in range(b):
        for j in range(r):
            if j >= rows[i]:
                assert not out[i, j].any() and not kk[i, j].any() and not vv[i, j].any()
                continue
            ang = None if tab is None else f64(tab)[lens[i] + j]
            wq = okvq.norm_rotate(f64(q[i, j]), n(gq), 1e-6, ang)
            wk = okvq.held(okvq.norm_rotate(f64(k[i, j]), n(gk), 1e-6, ang))
            wv = okvq.held(f64(v[i, j]))
            # m + n s rounded once to float32
            np.testing.assert_array_equal(kk[i, j].cpu().numpy(), wk.astype(np.float32))
            np.testing.assert_array_equal(vv[i, j].cpu().numpy(), wv.astype(np.float32))
            # float32 queries: a sum of hd squares, a root, a quotient, two products and a
            # rotation, at most hd / 8 + 16 roundings of 2^-24 of the head's largest entries
            top = np.abs(wq).max(-1, keepdims=True) * 2
            tol = (hd / 8 + 16) * 2.0 ** -24 * top + (2.0 ** -8 * np.abs(wq) if dtype == "bf16" else 0)
            assert (np.abs(f64(out[i, j]) - wq) <= tol).all()
    # everything else of the cache is as it was: other layers, other positions
    whole_k, _ = cache.read(1, cache.max_len)
    other, _ = cache.read(0, cache.max_len)
    assert torch.isnan(other).all()
    for i in range(b):
        assert torch.isnan(whole_k[i, :lens[i]]).all() and torch.isnan(whole_k[i, lens[i] + rows[i]:]).all()
    assert cache.device_error() == 0


@pytest.mark.parametrize("hd,r,h,kvh,dtype", [(128, 3001, 8, 4, "f32"), (64, 6011, 8, 4, "bf16"), (128, 9000, 2, 1, "bf16")])
def test_append_long_prompts(hd, r, h, kvh, dtype):
    """Prompts whose rows a workgroup takes in several rounds, the second
    request's shorter than the call."""
    rng = np.random.default_rng(r)
    rows, lens = [r, r - 1234], [3, 0]
    cache = kvq.QuantCache(1, 2, h, kvh, hd, r + 5, device=DEV)
    poison(cache)
    cache.lens.copy_(i32(lens))
    q, k, v = (rand(rng, 2, r, n, hd, dtype=dtype) for n in (h, kvh, kvh))
    gain = rand(rng, hd).abs()
    tab = kvq.rope_table(r + 5, hd, 10000.0, DEV)
    out = cache.append(0, k, v, q=q, gain_q=gain, gain_k=gain, rope=tab, rows=i32(rows))
    assert cache.device_error() == 0
    gk, gv = cache.read(0, r, start=cache.lens, rows=i32(rows))
    for b in (0, 1):
        n, ang = rows[b], f64(tab)[lens[b]:lens[b] + rows[b], None]
        y = f64(k[b, :n])
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + 1e-5) * f64(gain)
        a, c = y[..., :hd // 2], y[..., hd // 2:]
        y = np.concatenate([a * ang[..., 0] - c * ang[..., 1], c * ang[..., 0] + a * ang[..., 1]], -1)
        np.testing.assert_array_equal(gk[b, :n].cpu().numpy(), okvq.held(y).astype(np.float32))
        np.testing.assert_array_equal(gv[b, :n].cpu().numpy(), okvq.held(f64(v[b, :n])).astype(np.float32))
        for i in (0, n // 2, n - 1):
            want = okvq.norm_rotate(f64(q[b, i]), f64(gain), 1e-5, f64(tab)[lens[b] + i])
            # roundings: as in test_append_holds_what_the_definition_gives
            top = np.abs(want).max(-1, keepdims=True) * 2
            tol = (hd / 8 + 16) * 2.0 ** -24 * top + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0)
            assert (np.abs(f64(out[b, i]) - want) <= tol).all()
    assert not out[1, rows[1]:].any() and not gk[1, rows[1]:].any()


def test_append_rows_at_borders():
    """Constant rows, zeros, halves of steps (ties to even), tiny and huge
    rows, rows that are not finite."""
    hd = 128
    x = np.zeros((12, 1, hd), np.float32)
    x[1] = 2.5
    x[2] = 1e-3  # not a bfloat16: minimum rounded
    x[3, 0] = np.arange(hd) % 31 * 0.5  # steps of 1, every other value half-way
    x[4, 0] = -np.arange(hd) % 31 * 0.5
    x[5, 0] = np.arange(hd) * 1e-39  # subnormal
    x[6, 0] = np.linspace(-3e38, 1e38, hd)
    x[7, 0, 5] = np.nan
    x[8, 0, 7] = np.inf
    x[9, 0, 9] = -np.inf
    x[10, 0] = np.linspace(-1, 1, hd)
    x[11, 0] = 1e30
    x[11, 0, 0] = -1e-30
    t = torch.from_numpy(x)[None].to(DEV)
    cache = kvq.QuantCache(1, 1, 1, 1, hd, 12, device=DEV)
    cache.append(0, t, t)
    k, v = cache.read(0, 12)
    want = okvq.held(x).astype(np.float32)
    np.testing.assert_array_equal(k[0].cpu().numpy(), want)
    np.testing.assert_array_equal(v[0].cpu().numpy(), want)
    # (row 6 spans 4e38, more than float32 holds)
    assert np.isnan(want[6:10]).all() and np.isfinite(np.delete(want, [6, 7, 8, 9], 0)).all()


def test_append_past_the_end_drops_and_flags():
    cache = kvq.QuantCache(1, 2, 2, 2, 64, 20, device=DEV)
    poison(cache)
    before = cache.buf.clone()
    cache.lens.copy_(i32([18, 25]))
    rng = np.random.default_rng(0)
    x = rand(rng, 2, 4, 2, 64)
    cache.append(0, x, x)
    assert cache.device_error() == spade.DERR_CAPACITY
    k, _ = cache.read(0, 4, start=cache.lens)
    assert not k[0, 2:].any() and not k[1].any()
    np.testing.assert_array_equal(k[0, :2].cpu().numpy(), okvq.held(f64(x[0, :2])).astype(np.float32))
    cache.lens.copy_(i32([-3, -9]))
    cache.buf.copy_(before)
    cache.append(0, x, x)
    assert cache.device_error() == spade.DERR_CAPACITY
    k, _ = cache.read(0, 20)
    assert torch.isnan(k[1]).all() and torch.isnan(k[0, 1:]).all()  # row 3 of request 0 is position 0


def test_append_positions_of_a_table():
    """pos moves the angles alone; positions past the table are clamped and flagged."""
    rng = np.random.default_rng(3)
    tab = kvq.rope_table(10, 64, 10000.0, DEV)
    x = rand(rng, 1, 2, 1, 64)
    cache = kvq.QuantCache(1, 1, 1, 1, 64, 8, device=DEV)
    for pos, ang, flag in ((4, (4, 5), 0), (9, (9, 9), spade.DERR_CAPACITY), (-5, (0, 0), spade.DERR_CAPACITY)):
        q = cache.append(0, x, x, q=x, rope=tab, pos=i32([pos]))
        k, _ = cache.read(0, 2)
        for j in (0, 1):
            want = okvq.norm_rotate(f64(x[0, j]), None, 0, f64(tab)[ang[j]])
            np.testing.assert_array_equal(k[0, j].cpu().numpy(), okvq.held(want).astype(np.float32))
            assert np.abs(f64(q[0, j]) - want).max() <= 2.0 ** -20 * np.abs(want).max()
        assert cache.device_error() == flag


def test_append_clears_weights_of_new_positions():
    cache = kvq.QuantCache(1, 2, 2, 1, 64, 9, device=DEV)
    cache.lens.copy_(i32([2, 5]))
    w = torch.full((2, 1, 9), 3.0, device=DEV)
    x = torch.ones((2, 3, 1, 64), device=DEV)
    cache.append(0, x, x, rows=i32([3, 1]), weights=w)
    want = np.full((2, 1, 9), 3.0)
    want[0, 0, 2:5] = 0
    want[1, 0, 5] = 0
    assert w.cpu().numpy().tolist() == want.tolist()


# --- attention ------------------------------------------------------------


def check_attend(q, k, v, lens, rows, out, scale, dtype, weights=None, w_out=None, wr=0, w_before=None):
    b, R, H, hd = q.shape
    G = H // k.shape[2]
    for i in range(b):
        n = rows[i]
        assert not out[i, n:].any()
        if w_out is not None:
            end = lens[i] + n
            want_w = f64(weights[i, :, :end]) if weights is not None else np.zeros((k.shape[2], end))
            tol_w = np.zeros_like(want_w)
            if w_before is not None:  # behind the request: as they were
                assert torch.equal(w_out[i, :, end:], w_before[i, :, end:])
        if n:
            kk, vv = okvq.held(f64(k[i, :lens[i] + n])), okvq.held(f64(v[i, :lens[i] + n]))
            _, ks, _ = okvq.codes(f64(k[i, :lens[i] + n]))
            _, vs, _ = okvq.codes(f64(v[i, :lens[i] + n]))
            qq = f64(q[i, :n])
            o, p = okvq.attend(qq, kk, vv, lens[i], scale)
            for h in range(H):
                a = np.abs(qq[:, h])
                dz = scale * a.sum(-1) * ks[:, h // G].max() * 31 * 41 * 2.0 ** -24  # [n]
                s = vs[:, h // G].max()
                vmax = np.abs(vv[:, h // G]).max()
                r = 2.0 ** -24 if dtype == "f32" else 2.0 ** -8
                tol = 2.1 * dz[:, None] * vmax + 8 * s * r + 2.0 ** -18 * 31 * s
                if dtype == "bf16":
                    tol = tol + 2.0 ** -8 * np.abs(o[:, h])
                err = np.abs(f64(out[i, :n, h]) - o[:, h])
                assert (err <= tol).all(), (i, h, err.max(), tol.min())
                if w_out is not None:
                    m = min(wr, n)
                    want_w[h // G] += p[:m, h].sum(0)
                    # a probability: the scores' error, and the float32 exponent and log-sum-exp
                    # (below 64 in size: 4 roundings of 2^-24 64)
                    tol_w[h // G] += (p[:m, h] * (2.1 * dz[:m, None] + 2.0 ** -15)).sum(0)
        if w_out is not None:
            got = f64(w_out[i, :, :end])
            assert (np.abs(got - want_w) <= tol_w + 2.0 ** -21 * np.abs(want_w) + 1e-30).all()


ATTEND = [
    # b, r, h, kvh, hd, lens
    (1, 1, 1, 1, 128, [0]),
    (1, 1, 8, 2, 64, [31]),
    (1, 6, 4, 4, 128, [32]),
    (2, 1, 8, 2, 128, [511, 0]),
    (2, 2, 6, 2, 64, [510, 512]),
    (3, 9, 8, 2, 128, [513, 1, 1030]),  # 36 packed rows: three tiles
    (1, 16, 16, 1, 64, [700]),  # 256 packed rows
    (2, 16, 3, 3, 128, [15, 2048]),
    (5, 5, 10, 2, 64, [0, 3, 40, 255, 260]),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("wr", [None, 0, 1, 99])
@pytest.mark.parametrize("b,r,h,kvh,hd,lens", ATTEND)
def test_attend(b, r, h, kvh, hd, lens, wr, dtype):
    rng = np.random.default_rng(17 * r + h + hd)
    cache = kvq.QuantCache(2, b, h, kvh, hd, max(lens) + r + 5, max_rows=r, device=DEV)
    poison(cache)
    rows = [r] + [int(x) for x in rng.integers(0, r + 1, b - 1)]
    n = max(lens) + r
    k, v = rand(rng, b, n, kvh, hd, dtype=dtype), rand(rng, b, n, kvh, hd, dtype=dtype)
    fill(cache, 1, k, v, rows=i32([a + c for a, c in zip(lens, rows)]))
    cache.lens.copy_(i32(lens))
    q = rand(rng, b, r, h + 3, hd, dtype=dtype)[:, :, 1:1 + h]  # strided rows
    scale = 1 / math.sqrt(hd)
    kw, w, wo, before = {}, None, None, None
    if wr is not None:
        wr = min(wr, r)
        w = rand(rng, b, kvh, cache.max_len, strong=False).abs()
        wo = rand(rng, b, kvh, cache.max_len, strong=False)
        before = wo.clone()
        kw = dict(weights=w, weights_out=wo, weight_rows=wr)
    out = cache.attend(1, q, rows=i32(rows), max_keys=n, **kw)
    check_attend(q, k, v, lens, rows, out, scale, dtype, w, wo, wr or 0, before)
    assert cache.device_error() == 0
    # the bound only sizes the launch (other chunks: the last bits may move), weights in place
    if wr is not None:
        w2 = w.clone()
        cache.attend(1, q, out=out, rows=i32(rows), weights=w2, weights_out=w2, weight_rows=wr)
        check_attend(q, k, v, lens, rows, out, scale, dtype, w, w2, wr, w)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,r,h,kvh,hd,most", [
    (16, 2, 16, 8, 128, 2500),  # ranges over the batch, several heads each
    (70, 1, 4, 2, 64, 2300),    # more requests than a wave has lanes
    (3, 16, 16, 2, 128, 2000),  # equal parts, tiles of 16 rows
    (16, 3, 16, 8, 128, 1300),  # whole heads of a workgroup
    (12, 16, 6, 1, 64, 700),
    (1, 16, 1, 1, 128, 600),
])
def test_attend_cuts(b, r, h, kvh, hd, most, dtype):
    """Batches of requests of all lengths, some without rows in use, whichever
    way their heads are divided among workgroups; weights too."""
    rng = np.random.default_rng(b + r)
    lens = [int(x) for x in rng.integers(0, most, b)]
    lens[-1] = most
    rows = [int(x) for x in rng.integers(0, r + 1, b)]
    rows[-1] = r
    cache = kvq.QuantCache(1, b, h, kvh, hd, most + r, max_rows=r, device=DEV)
    poison(cache)
    k, v = rand(rng, b, most + r, kvh, hd, dtype=dtype), rand(rng, b, most + r, kvh, hd, dtype=dtype)
    fill(cache, 0, k, v, rows=i32([a + c for a, c in zip(lens, rows)]))
    cache.lens.copy_(i32(lens))
    q = rand(rng, b, r, h, hd, dtype=dtype)
    w = torch.zeros((b, kvh, cache.max_len), device=DEV)
    out = cache.attend(0, q, rows=i32(rows), weights_out=w, weight_rows=1)
    check_attend(q, k, v, lens, rows, out, hd ** -0.5, dtype, None, w, 1)
    assert cache.device_error() == 0
    assert torch.equal(cache.attend(0, q, rows=i32(rows)), out)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attend_scale_and_large_scores(dtype):
    """Scores of some thousands (a softmax that is one position), and a scale
    of its own."""
    rng = np.random.default_rng(5)
    cache = kvq.QuantCache(1, 1, 2, 1, 128, 300, device=DEV)
    k, v = rand(rng, 1, 300, 1, 128, dtype=dtype), rand(rng, 1, 300, 1, 128, dtype=dtype)
    fill(cache, 0, k, v)
    cache.lens.fill_(297)
    for scale, mul in ((0.02, 1), (1.0, 16)):
        q = (rand(rng, 1, 3, 2, 128) * mul).to(TD[dtype])
        out = cache.attend(0, q, scale=scale)
        check_attend(q, k, v, [297], [3], out, scale, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("qx,kx,vx", [(50, -50, 0), (-40, 40, 0), (60, -70, 40), (-30, 30, -37), (0, 0, 48)])
def test_attend_keeps_its_precision_over_the_range(qx, kx, vx, dtype):
    """Queries, keys and values of other magnitudes (by powers of two): the same
    bounds, which are relative to the rows' scales."""
    rng = np.random.default_rng(12)
    cache = kvq.QuantCache(1, 2, 4, 1, 128, 400, device=DEV)
    k, v = rand(rng, 2, 400, 1, 128, dtype=dtype) * 2.0 ** kx, rand(rng, 2, 400, 1, 128, dtype=dtype) * 2.0 ** vx
    fill(cache, 0, k, v)
    cache.lens.copy_(i32([395, 17]))
    q = rand(rng, 2, 3, 4, 128, dtype=dtype) * 2.0 ** qx
    scale = 2.0 ** (-qx - kx) / math.sqrt(128)
    out = cache.attend(0, q, scale=scale)
    check_attend(q, k, v, [395, 17], [3, 3], out, scale, dtype)


@pytest.mark.parametrize("hd,h,kvh,lens", [(128, 8, 2, [300, 2000]), (64, 6, 6, [40, 900])])
def test_attend_precision_of_float32_calls(hd, h, kvh, lens):
    """The header's figure, about 1e-6 of an output's size (2-norms), with a factor
    of two for other inputs than it was measured on."""
    rng = np.random.default_rng(13)
    cache = kvq.QuantCache(1, 2, h, kvh, hd, max(lens) + 4, device=DEV)
    k, v = rand(rng, 2, max(lens) + 4, kvh, hd), rand(rng, 2, max(lens) + 4, kvh, hd)
    fill(cache, 0, k, v)
    cache.lens.copy_(i32(lens))
    q = rand(rng, 2, 4, h, hd, strong=False)
    out = cache.attend(0, q)
    for b, L in enumerate(lens):
        want, _ = okvq.attend(f64(q[b]), okvq.held(f64(k[b, :L + 4])), okvq.held(f64(v[b, :L + 4])), L, hd ** -0.5)
        assert np.linalg.norm(f64(out[b]) - want) <= 2e-6 * np.linalg.norm(want)


def test_attend_hidden_positions_may_hold_anything():
    """Draft rows that are not finite, stale rows and empty space do not reach
    the rows that cannot see them; the rows that see them are NaN."""
    rng = np.random.default_rng(6)
    for L in (0, 20, 31, 600):
        cache = kvq.QuantCache(1, 1, 4, 2, 128, L + 10, device=DEV)
        poison(cache)
        k, v = rand(rng, 1, L + 4, 2, 128), rand(rng, 1, L + 4, 2, 128)
        clean_k, clean_v = k.clone(), v.clone()
        k[0, L + 2, 0, 7] = float("nan")
        v[0, L + 3, 1, 9] = float("inf")
        fill(cache, 0, k, v)
        cache.lens.fill_(L)
        q = rand(rng, 1, 4, 4, 128)
        w = torch.zeros((1, 2, cache.max_len), device=DEV)
        out = cache.attend(0, q, weights_out=w, weight_rows=2)
        check_attend(q[:, :2], clean_k, clean_v, [L], [2], out[:, :2], 128 ** -0.5, "f32")
        assert torch.isnan(out[0, 2:, :2]).all()  # heads of K/V head 0 see position L + 2
        assert torch.isfinite(out[0, 2, 2:]).all() and torch.isnan(out[0, 3, 2:]).all()
        assert torch.isfinite(w).all() and not w[:, :, L + 2:].any()


def test_attend_nan_query_stays_in_its_row():
    rng = np.random.default_rng(7)
    cache = kvq.QuantCache(1, 1, 4, 2, 64, 100, device=DEV)
    k, v = rand(rng, 1, 100, 2, 64), rand(rng, 1, 100, 2, 64)
    fill(cache, 0, k, v)
    cache.lens.fill_(97)
    q = rand(rng, 1, 3, 4, 64)
    want = cache.attend(0, q)
    q2 = q.clone()
    q2[0, 1, 2, 5] = float("nan")
    got = cache.attend(0, q2)
    assert torch.isnan(got[0, 1, 2]).all()
    got[0, 1, 2] = want[0, 1, 2]
    assert torch.equal(got, want)


def test_attend_longer_than_the_bound_is_cut_and_flagged():
    rng = np.random.default_rng(8)
    cache = kvq.QuantCache(1, 2, 2, 2, 64, 80, device=DEV)
    k, v = rand(rng, 2, 80, 2, 64), rand(rng, 2, 80, 2, 64)
    fill(cache, 0, k, v)
    q = rand(rng, 2, 2, 2, 64)
    cache.lens.copy_(i32([60, 30]))
    out = cache.attend(0, q, max_keys=40)
    assert cache.device_error() == spade.DERR_CAPACITY
    check_attend(q, k, v, [38, 30], [2, 2], out, 64 ** -0.5, "f32")
    cache.lens.copy_(i32([-1, 300]))
    out = cache.attend(0, q)
    assert cache.device_error() == spade.DERR_CAPACITY
    check_attend(q, k, v, [0, 78], [2, 2], out, 64 ** -0.5, "f32")


def test_lengths_at_the_end_of_their_type():
    """lens, pos and start near 2^31: their sums with row numbers stop at the
    type's end, so rows are dropped, cut and flagged as at any other length."""
    rng = np.random.default_rng(11)
    big = 2**31 - 1
    cache = kvq.QuantCache(1, 2, 2, 2, 64, 80, device=DEV)
    k, v = rand(rng, 2, 80, 2, 64), rand(rng, 2, 80, 2, 64)
    fill(cache, 0, k, v)
    before = cache.buf.clone()
    cache.lens.copy_(i32([big, big - 2]))
    tab = kvq.rope_table(10, 64, 10000.0, DEV)
    x = rand(rng, 2, 4, 2, 64)
    q = cache.append(0, x, x, q=x, rope=tab)
    assert cache.device_error() == spade.DERR_CAPACITY
    assert torch.equal(cache.buf, before)
    want = okvq.norm_rotate(f64(x).reshape(-1, 64), None, 0, f64(tab)[9]).reshape(x.shape)  # the table's last position
    assert np.abs(f64(q) - want).max() <= 2.0 ** -20 * np.abs(want).max()
    w = torch.zeros((2, 2, 80), device=DEV)
    out = cache.attend(0, x, weights_out=w, weight_rows=1)
    assert cache.device_error() == spade.DERR_CAPACITY
    check_attend(x, k, v, [76, 76], [4, 4], out, 64 ** -0.5, "f32", None, w, 1)
    for t in cache.read(0, 4, start=cache.lens):
        assert not t.any()


@pytest.mark.parametrize("n", [20000, 131072])
def test_attend_long(n):
    rng = np.random.default_rng(9)
    cache = kvq.QuantCache(1, 1, 4, 1, 128, n + 1, max_rows=1, device=DEV)
    k, v = rand(rng, 1, n + 1, 1, 128, dtype="bf16"), rand(rng, 1, n + 1, 1, 128, dtype="bf16")
    fill(cache, 0, k, v)
    cache.lens.fill_(n)
    q = rand(rng, 1, 1, 4, 128)
    w = torch.zeros((1, 1, n + 1), device=DEV)
    out = cache.attend(0, q, weights_out=w, weight_rows=1)
    check_attend(q, k, v, [n], [1], out, 128 ** -0.5, "f32", None, w, 1)


def test_attend_does_not_depend_on_other_layers_offsets():
    """A region that starts beyond 2^32 bytes: the last layer of a large cache."""
    rng = np.random.default_rng(10)
    cache = kvq.QuantCache(2, 16, 2, 1, 128, 1 << 20, max_rows=1, device=DEV)
    assert cache.buf.numel() > 1 << 32
    n = 700
    k, v = rand(rng, 16, n, 1, 128), rand(rng, 16, n, 1, 128)
    fill(cache, 1, k, v)
    cache.lens.fill_(n - 1)
    q = rand(rng, 16, 1, 2, 128)
    out = cache.attend(1, q, max_keys=n)
    check_attend(q, k, v, [n - 1] * 16, [1] * 16, out, 128 ** -0.5, "f32")
    kk, _ = cache.read(1, n)
    np.testing.assert_array_equal(kk[15].cpu().numpy(), okvq.held(f64(k[15])).astype(np.float32))


# --- eviction -------------------------------------------------------------

EVICT = [
    # layers, b, kvh, hd, lens, budget, recent
    (1, 1, 1, 128, [5], 1, 0),
    (1, 1, 1, 64, [5], 1, 1),
    (2, 3, 2, 128, [0, 40, 100], 40, 8),
    (1, 2, 3, 64, [1500, 1024], 700, 700),
    (2, 2, 2, 64, [3000, 2999], 1030, 0),
    (1, 2, 2, 128, [1024, 1025], 1024, 100),
]


@pytest.mark.parametrize("kind", ["random", "ties", "zeros", "odd"])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("layers,b,kvh,hd,lens,budget,recent", EVICT)
def test_evict(layers, b, kvh, hd, lens, budget, recent, in_place, kind):
    rng = np.random.default_rng(budget + len(kind))
    cap = max(lens) + 2
    cache = kvq.QuantCache(layers, b, kvh, kvh, hd, cap, device=DEV)
    poison(cache)
    for l in range(layers):
        x = rand(rng, b, cap, kvh, hd), rand(rng, b, cap, kvh, hd)
        fill(cache, l, *x, rows=i32(lens))
    cache.lens.copy_(i32(lens))
    w = {"random": rng.exponential(size=(layers, b, kvh, cap)), "ties": rng.integers(0, 3, (layers, b, kvh, cap)),
         "zeros": np.zeros((layers, b, kvh, cap)), "odd": rng.normal(size=(layers, b, kvh, cap))}[kind].astype(np.float32)
    if kind == "odd":
        w[..., ::7] = np.nan
        w[..., 1::11] = np.inf
        w[..., 2::13] = -np.inf
        w[..., 3::5] = -0.0
        w[..., 4::5] = 0.0
        w[..., 5::17] = 1e-42
    before = [cache.read(l, cap) for l in range(layers)]
    dw = torch.from_numpy(w).to(DEV)
    if in_place:
        dst, wo = cache, dw
        kept = cache.evict(dw, budget, recent, weights_out=dw)
    else:
        dst = kvq.QuantCache(layers, b, kvh, kvh, hd, budget + 1, device=DEV)
        poison(dst)
        wo = torch.full((layers, b, kvh, budget + 1), -7.0, device=DEV)
        kept = cache.evict(dw, budget, recent, into=dst, weights_out=wo)
        assert torch.equal(cache.lens, i32(lens))
    assert dst.lens.tolist() == [min(n, budget) for n in lens]
    kept, wo = kept.cpu().numpy(), wo.cpu().numpy()
    for l in range(layers):
        kk, vv = dst.read(l, dst.max_len)
        for i in range(b):
            m = min(lens[i], budget)
            for h in range(kvh):
                want = okvq.keep(w[l, i, h], lens[i], budget, recent)
                assert kept[l, i, h].tolist() == want.tolist() + [-1] * (budget - m)
                idx = torch.from_numpy(want).to(DEV)
                assert torch.equal(kk[i, :m, h], before[l][0][i, idx, h])
                assert torch.equal(vv[i, :m, h], before[l][1][i, idx, h])
                np.testing.assert_array_equal(wo[l, i, h, :m], w[l, i, h, want])
                if in_place:  # behind the kept ones: as they were
                    np.testing.assert_array_equal(wo[l, i, h, max(m, lens[i]):], w[l, i, h, max(m, lens[i]):])
                else:
                    assert (wo[l, i, h, m:] == -7).all() and torch.isnan(kk[i, m:, h]).all()


# --- together -------------------------------------------------------------


@pytest.mark.parametrize("hd,h,kvh", [(128, 8, 2), (64, 3, 3)])
def test_a_stream_longer_than_its_cache(hd, h, kvh):
    """Prompt, verify-like calls of five rows of which some are kept, eviction
    in place whenever the cache is nearly full: two layers, two requests, the
    angles counting every row that ever was.  The oracle keeps its own caches."""
    rng = np.random.default_rng(hd)
    layers, b, cap, budget, recent, R = 2, 2, 90, 48, 16, 5
    cache = kvq.QuantCache(layers, b, h, kvh, hd, cap, max_rows=R, device=DEV)
    poison(cache)
    tab = kvq.rope_table(400, hd, 10000.0, DEV)
    gq, gk = rand(rng, hd, strong=False), rand(rng, hd, strong=False)
    W = torch.zeros((layers, b, kvh, cap), device=DEV)
    ok = [[np.zeros((0, kvh, hd)) for _ in range(b)] for _ in range(layers)]
    ov = [[np.zeros((0, kvh, hd)) for _ in range(b)] for _ in range(layers)]
    ow = [[np.zeros((kvh, 0)) for _ in range(b)] for _ in range(layers)]
    pos = [0, 0]
    evictions = 0
    for step in range(24):
        r = 40 if step == 0 else R
        rows = [r, r - 7] if step == 0 else [R, int(rng.integers(1, R + 1))]
        for l in range(layers):
            q, k, v = (rand(rng, b, r, n, hd) for n in (h, kvh, kvh))
            qo = cache.append(l, k, v, q=q, gain_q=gq, gain_k=gk, rope=tab, pos=i32(pos), rows=i32(rows), weights=W[l])
            out = None
            if step:
                out = cache.attend(l, qo, rows=i32(rows), weights=W[l], weights_out=W[l], weight_rows=1)
            for i in range(b):
                ang = f64(tab)
                kk = np.stack([okvq.norm_rotate(f64(k[i, j]), f64(gk), 1e-5, ang[pos[i] + j]) for j in range(rows[i])])
                L = len(ok[l][i])
                tk, tv = np.concatenate([ok[l][i], okvq.held(kk)]), np.concatenate([ov[l][i], okvq.held(f64(v[i, :rows[i]]))])
                tw = np.concatenate([ow[l][i], np.zeros((kvh, rows[i]))], -1)
                if step:
                    o, p = okvq.attend(f64(qo[i, :rows[i]]), tk, tv, L, hd ** -0.5)
                    # values of some units and scores below some hundreds: dz below 2^-11
                    assert np.abs(f64(out[i, :rows[i]]) - o).max() <= 2.0 ** -9 * np.abs(tv).max()
                    g = h // kvh
                    tw = tw + p[0].reshape(kvh, g, -1).sum(1)[:, :L + rows[i]]
                keep = rows[i] if step == 0 else max(1, rows[i] - 2)
                ok[l][i], ov[l][i], ow[l][i] = tk[:L + keep], tv[:L + keep], tw[:, :L + keep]
        keep = [n if step == 0 else max(1, n - 2) for n in rows]
        cache.lens += i32(keep)
        pos = [a + c for a, c in zip(pos, keep)]
        if int(cache.lens.max()) + R > cap:
            evictions += 1
            # the device's own weights decide (they are near the oracle's, not equal)
            w = W.cpu().numpy()
            for l in range(layers):
                for i in range(b):
                    n = len(ok[l][i])
                    np.testing.assert_allclose(w[l, i, :, :n], ow[l][i], rtol=2e-2, atol=2e-3)
            kept = cache.evict(W, budget, recent, weights_out=W).cpu().numpy()
            for l in range(layers):
                for i in range(b):
                    n = len(ok[l][i])
                    m = min(n, budget)
                    nk, nv, nw = np.zeros((m, kvh, hd)), np.zeros((m, kvh, hd)), np.zeros((kvh, m))
                    for a in range(kvh):
                        idx = okvq.keep(w[l, i, a], n, budget, recent)
                        assert kept[l, i, a, :m].tolist() == idx.tolist()
                        nk[:, a], nv[:, a], nw[a] = ok[l][i][idx, a], ov[l][i][idx, a], w[l, i, a, idx]
                    ok[l][i], ov[l][i], ow[l][i] = nk, nv, nw
        for l in range(layers):
            kk, vv = cache.read(l, cap)
            for i in range(b):
                n = len(ok[l][i])
                np.testing.assert_array_equal(kk[i, :n].cpu().numpy(), ok[l][i].astype(np.float32))
                np.testing.assert_array_equal(vv[i, :n].cpu().numpy(), ov[l][i].astype(np.float32))
    assert evictions >= 1 and cache.device_error() == 0


def test_captured_and_replayed():
    """One graph of append, attend with weights, and eviction into another
    cache; every replay, with eager work between, equals the eager calls."""
    rng = np.random.default_rng(11)
    b, h, kvh, hd, L, R = 2, 4, 2, 128, 700, 3
    cache = kvq.QuantCache(1, b, h, kvh, hd, L + R, max_rows=R, device=DEV)
    dst = kvq.QuantCache(1, b, h, kvh, hd, 300, device=DEV)
    k, v = rand(rng, b, L, kvh, hd), rand(rng, b, L, kvh, hd)
    fill(cache, 0, k, v)
    cache.lens.fill_(L)
    tab = kvq.rope_table(L + R, hd, 10000.0, DEV)
    q0, k0, v0 = (rand(rng, b, R, n, hd) for n in (h, kvh, kvh))
    W = rand(rng, 1, b, kvh, L + R, strong=False).abs()
    W2, qo, out = torch.zeros_like(W), torch.empty_like(q0), torch.empty_like(q0)
    kept = torch.empty((1, b, kvh, 300), dtype=torch.int32, device=DEV)

    def step():
        cache.append(0, k0, v0, q=q0, rope=tab, q_out=qo)
        cache.attend(0, qo, out=out, weights=W[0], weights_out=W2[0], weight_rows=R)
        cache.evict(W2, 300, 20, kept, into=dst)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        for t in (q0, k0, v0):
            t.copy_(rand(rng, *t.shape))
        for t in (out, W2, qo):
            t.fill_(float("nan"))
        kept.fill_(-5)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, W2, kept, dst.lens, *dst.read(0, 300))]
        for t in (out, W2, qo):
            t.fill_(float("nan"))
        step()
        torch.cuda.synchronize()
        for a, c in zip(got, (out, W2, kept, dst.lens, *dst.read(0, 300))):
            assert torch.equal(a, c), i


def test_same_call_twice_gives_the_same_bits():
    rng = np.random.default_rng(12)
    cache = kvq.QuantCache(1, 3, 8, 2, 128, 3000, max_rows=9, device=DEV)
    k, v = rand(rng, 3, 3000, 2, 128), rand(rng, 3, 3000, 2, 128)
    fill(cache, 0, k, v)
    cache.lens.copy_(i32([2991, 5, 1700]))
    q = rand(rng, 3, 9, 8, 128)
    w = torch.zeros((2, 3, 2, 3000), device=DEV)
    a = [cache.attend(0, q, weights_out=w[i], weight_rows=9) for i in (0, 1)]
    assert torch.equal(a[0], a[1]) and torch.equal(w[0], w[1])


def test_binding_refuses():
    cache = kvq.QuantCache(1, 2, 4, 2, 64, 50, max_rows=4, device=DEV)
    x = torch.zeros((2, 3, 2, 64), device=DEV)
    q = torch.zeros((2, 3, 4, 64), device=DEV)
    for call in (lambda: cache.append(0, x[:, :, :1], x), lambda: cache.append(0, x, x.bfloat16()),
                 lambda: cache.append(0, x.double(), x.double()), lambda: cache.append(0, x.cpu(), x),
                 lambda: cache.append(0, x.transpose(0, 1), x), lambda: cache.append(0, x, x, rows=i32([1])),
                 lambda: cache.append(0, x, x, rope=torch.zeros((9, 32), device=DEV)),
                 lambda: cache.attend(0, q.half()), lambda: cache.attend(0, q[..., :32]),
                 lambda: cache.attend(0, q, weights_out=torch.zeros((2, 2, 49), device=DEV)),
                 lambda: cache.attend(0, torch.zeros((2, 3, 64, 4), device=DEV).transpose(2, 3)),
                 lambda: cache.evict(torch.zeros((1, 2, 2, 50), device=DEV), 10, 1, kept=i32([0])),
                 lambda: cache.read(0, 4, dtype=torch.float16)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: cache.append(1, x, x), lambda: cache.attend(0, torch.zeros((2, 5, 4, 64), device=DEV)),
                 lambda: cache.evict(torch.zeros((1, 2, 2, 50), device=DEV), 51, 1),
                 lambda: kvq.QuantCache(1, 1, 3, 2, 64, 8, device=DEV), lambda: cache.attend(0, q, scale=0.0)):
        with pytest.raises(spade.SpadeError):
            call()
