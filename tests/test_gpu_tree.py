"""Trees of drafts on the GPU against the float64 oracle (oracle/tree.py).

Tolerances, u = 2^-24.

append    cosine and sine come from an angle in double and are rounded once, u
          each of at most 1; of x cos - y sin the products and the sum round three
          times: 5 u amplitude (|x| + |y|), the features as the inputs hold them.  A
          bfloat16 result adds half a step, 2^-8 of it (of a value that is itself
          off by less than 2^-16 of it).  Values are the input's rounding.
attend    a score's float32 sum takes 4 (head_dim 128) products of 32 for each of up
          to three terms, each rounding at most twice what it has so far:
            dz = scale 24 u sum_f |q_f k_f| + 2 u |scale q.k|   (the exponent)
          moves a probability by a factor of at most 1 +- 2.1 dz; probabilities are
          held in 24 bits (bfloat16 calls 16: 2^-17) and come from an exponential of
          2^-22; sums over n keys in blocks of 32, three products a block, each
          rounding once, take (3 n / 32 + 8) u of the largest value (the sum of
          probabilities likewise, hence twice).  An output rounds: u, or 2^-8.
"""

import math

import numpy as np
import pytest
import torch

from oracle import tree as otree
from paper_2608_13076_amd import sampling, spade, tree

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TD = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24
HALF = 2.0 ** -8 * (1 + 2.0 ** -8)  # half a step of bfloat16


def rand(rng, *shape, dtype="f32", strong=True):
    x = rng.normal(size=shape).astype(np.float32)
    if strong:
        x[..., 3::17] *= 4
    return torch.from_numpy(x).to(DEV).to(TD[dtype])


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def poison(cache):
    """Every element NaN."""
    cache.buf.fill_(255)


def a_tree(rng, n, wide=0.25):
    return [-1] + [max(0, i - 1 - int(rng.exponential(1 / wide))) for i in range(1, n)]


# --- append and read ----------------------------------------------------------

APPEND = [
    # b, r, h, kvh, hd, lens, rot, interleaved
    (1, 1, 8, 2, 128, [0], 128, False),
    (1, 1, 8, 2, 64, [31], 64, True),
    (3, 5, 4, 4, 128, [254, 0, 97], 64, False),
    (2, 16, 12, 4, 64, [1, 60], 40, True),
    (2, 70, 6, 1, 128, [3, 250], 120, False),
    (4, 3, 5, 5, 64, [0, 1, 2, 3], 8, False),
    (2, 300, 3, 3, 128, [7, 500], 128, True),
    (2, 9, 4, 2, 64, [5, 6], 0, False),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,r,h,kvh,hd,lens,rot,inter", APPEND)
def test_append_holds_what_the_definition_gives(b, r, h, kvh, hd, lens, rot, inter, dtype):
    rng = np.random.default_rng(b * 100 + r + hd)
    cache = tree.TreeCache(2, b, h, kvh, hd, max(lens) + r + 3, max_rows=1, device=DEV)
    poison(cache)
    cache.lens.copy_(i32(lens))
    qkv = rand(rng, b, r, h + 2 * kvh, hd, dtype=dtype)  # fused rows: strided views
    q, k, v = qkv[:, :, :h], qkv[:, :, h:h + kvh], qkv[:, :, h + kvh:]
    rope = amp = None
    if rot:
        freq, amp = tree.rotary_frequencies(rot, 500000.0, "ramp", 4.0, trained=1000, device=DEV)
        rope = tree.Rotary(freq, inter, amp)
    rows = [r] + [int(x) for x in rng.integers(0, r + 1, b - 1)]
    depth = None if r > 64 else [otree.depths(a_tree(rng, r), r) for _ in range(b)]
    out = cache.append(1, k, v, q=q, rope=rope, depth=None if depth is None else i32(depth), rows=i32(rows))
    kk, vv = cache.read(1, r, start=cache.lens, rows=i32(rows), dtype=torch.float32)
    assert cache.device_error() == 0
    half = rot // 2
    for i in range(b):
        n = rows[i]
        assert not out[i, n:].any() and not kk[i, n:].any() and not vv[i, n:].any()
        np.testing.assert_array_equal(f64(vv[i, :n]), f64(v[i, :n].to(torch.bfloat16)))
        for j in range(n):
            at = lens[i] + (j if depth is None else depth[i][j])
            ang = at * f64_freq(rope) if rot else np.zeros(0)
            for src, got, bf in ((q, out, dtype == "bf16"), (k, kk, True)):
                x = f64(src[i, j])
                want = otree.rotate(x, ang, inter, amp or 1.0)
                size = np.abs(x)
                if rot:  # |x| + |y| of a pair
                    a, c = (slice(0, rot, 2), slice(1, rot, 2)) if inter else (slice(0, half), slice(half, rot))
                    s = size[:, a] + size[:, c]
                    size[:, a], size[:, c] = s, s
                tol = 5 * U * (amp or 1.0) * size + (HALF * np.abs(want) if bf else 0)
                assert (np.abs(f64(got[i, j]) - want) <= tol).all()
                if rot < hd and bf == (dtype == "bf16"):  # features behind the rotated ones
                    np.testing.assert_array_equal(f64(got[i, j])[:, rot:], x[:, rot:])
    # everything else of the cache is as it was: other layers, other positions
    whole_k, whole_v = cache.read(1, cache.max_len)
    other, _ = cache.read(0, cache.max_len)
    assert torch.isnan(other).all()
    for i in range(b):
        for t in (whole_k, whole_v):
            assert torch.isnan(t[i, :lens[i]]).all() and torch.isnan(t[i, lens[i] + rows[i]:]).all()


def f64_freq(rope):
    return rope.freq.cpu().numpy()


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dtype,hd,r", [("bf16", 128, 2100), ("f32", 128, 1300), ("bf16", 64, 4203), ("f32", 64, 2111)])
def test_append_of_long_prompts_equals_its_pieces(dtype, hd, r, inter):
    """A call of more than 64 MB, ragged and from strided rows, against calls of a few rows."""
    b, h, kvh, step = 2, 32, 32, 307
    gen = torch.Generator(device=DEV).manual_seed(r)
    qkv = torch.randn(b, r, h + 2 * kvh, hd, generator=gen, device=DEV).to(TD[dtype])
    q, k, v = qkv[:, :, :h], qkv[:, :, h:h + kvh], qkv[:, :, h + kvh:]
    rope = tree.Rotary(tree.rotary_frequencies(hd, device=DEV)[0], inter)
    big, small = (tree.TreeCache(1, b, h, kvh, hd, r + 40, max_rows=1, device=DEV) for _ in range(2))
    rows = [r, r - 501]
    for c in (big, small):
        poison(c)
        c.lens.copy_(i32([5, 33]))
    out = torch.full((b, r, h, hd), 7.0, device=DEV).to(TD[dtype])
    big.append(0, k, v, q=q, rope=rope, rows=i32(rows), q_out=out)
    for s in range(0, r, step):
        m = min(step, r - s)
        part = small.append(0, *(t[:, s:s + m].contiguous() for t in (k, v)), q=q[:, s:s + m].contiguous(), rope=rope,
                            rows=i32([max(0, min(m, n - s)) for n in rows]))
        assert torch.equal(part, out[:, s:s + m])
        small.lens += m
    assert big.device_error() == 0 and small.device_error() == 0
    for x, y in zip(big.read(0, r + 40), small.read(0, r + 40)):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))


def test_append_at_far_positions():
    """Angles of positions up to 2^30 keep their fraction of a turn."""
    rng = np.random.default_rng(5)
    freq, _ = tree.rotary_frequencies(128, 10000.0, device=DEV)
    cache = tree.TreeCache(1, 3, 2, 1, 128, 8, max_rows=1, device=DEV)
    q = rand(rng, 3, 2, 2, 128)
    pos = [100003, (1 << 30) + 7, -12345]
    out = cache.append(0, q[:, :, :1].contiguous(), q[:, :, 1:].contiguous(), q=q, rope=tree.Rotary(freq), pos=i32(pos))
    for b in range(3):
        for j in range(2):
            ang = (pos[b] + j) * freq.cpu().numpy()  # in double, as the definition says
            x = f64(q[b, j])
            tol = 5 * U * (np.abs(x) + np.abs(np.roll(x, 64, -1))) + 2.0 ** -53 * abs(pos[b]) * 4 * np.abs(x).max()
            assert (np.abs(f64(out[b, j]) - otree.rotate(x, ang, False)) <= tol).all()


def test_append_in_place_and_past_the_end():
    rng = np.random.default_rng(6)
    cache = tree.TreeCache(1, 3, 2, 2, 64, 20, max_rows=1, device=DEV)
    poison(cache)
    cache.lens.copy_(i32([18, 25, -3]))
    freq, _ = tree.rotary_frequencies(64, device=DEV)
    x = rand(rng, 3, 4, 2, 64)
    q = x.clone()
    want = cache.append(0, x, x, q=x, rope=tree.Rotary(freq))
    assert cache.device_error() == spade.DERR_CAPACITY
    got = cache.append(0, x, x, q=q, rope=tree.Rotary(freq), q_out=q)
    assert got is q and torch.equal(q, want)
    _, v = cache.read(0, 20)
    assert torch.equal(v[0, 18:], x[0, :2].to(torch.bfloat16)) and torch.isnan(v[0, :18]).all()
    assert torch.isnan(v[1]).all() and torch.isnan(v[2, 1:]).all() and torch.equal(v[2, 0], x[2, 3].to(torch.bfloat16))
    # reads outside the cache give zeros
    k, v = cache.read(0, 4, start=i32([18, -2, 2147483646]))
    assert torch.equal(v[0, :2], x[0, :2].to(torch.bfloat16)) and not v[0, 2:].any() and not v[1, :2].any() and not v[2].any()
    assert not k[0, 2:].any() and not k[1, :2].any() and not k[2].any()
    cache.lens.copy_(i32([2147483647, -2147483648, 0]))
    cache.append(0, x, x)
    assert cache.device_error() == spade.DERR_CAPACITY


def test_append_lays_out_a_models_cache():
    """Fragments as include/spade.h describes them."""
    rng = np.random.default_rng(7)
    hd, n = 128, 300
    cache = tree.TreeCache(2, 2, 2, 2, hd, n, max_rows=1, device=DEV)
    k, v = (rand(rng, 2, n, 2, hd, dtype="bf16") for _ in range(2))
    cache.append(1, k, v)
    half = cache.buf.view(torch.bfloat16).reshape(2, 2, 2, 2, 2, hd * 256)  # K/V, layer, request, head, block
    for b, h, t, f in ((0, 0, 0, 0), (1, 1, 299, 127), (0, 1, 255, 64), (1, 0, 131, 37), (1, 1, 256, 8)):
        blk, p = divmod(t, 256)
        at_k = (((p // 16) * (hd // 32) + f // 32) * 64 + (f // 8) % 4 * 16 + p % 16) * 8 + f % 8
        at_v = (((f // 16) * 8 + p // 32) * 64 + (p // 8) % 4 * 16 + f % 16) * 8 + p % 8
        assert half[0, 1, b, h, blk, at_k] == k[b, t, h, f] and half[1, 1, b, h, blk, at_v] == v[b, t, h, f]


# --- attend ---------------------------------------------------------------------


def check_attend(cache, layer, q, k, v, lens, rows, parents, out, dtype, scale=None):
    """out against the oracle; k, v float64 [b][n, kvh, hd] per request."""
    b, r, h, hd = q.shape
    g = h // cache.n_kv_heads
    scale = scale or hd ** -0.5
    for i in range(b):
        assert not out[i, rows[i]:].any()
        for j in range(rows[i]):
            see = list(range(lens[i])) + [lens[i] + a for a in otree.lineage(parents[i], j)]
            for x in range(h):
                kk, vv, qq = k[i][see][:, x // g], v[i][see][:, x // g], f64(q[i, j, x])
                want = otree.attend(qq, kk, vv, scale)
                dz = 24 * U * scale * (np.abs(kk) @ np.abs(qq)).max() + 2 * U * scale * np.abs(kk @ qq).max()
                vm = np.abs(vv).max()
                tol = 2 * vm * (2.1 * dz + 2.0 ** -22 + (3 * len(see) / 32 + 8) * U + (2.0 ** -17 if dtype == "bf16" else U))
                tol = tol + np.abs(want) * (HALF if dtype == "bf16" else U)
                err = np.abs(f64(out[i, j, x]) - want)
                assert (err <= tol).all(), (i, j, x, err.max(), tol.min())


ATTEND = [
    # b, r, h, kvh, hd, lens, rows (None: all)
    (1, 1, 4, 4, 128, [0], None),
    (1, 1, 4, 1, 64, [1], None),
    (1, 5, 8, 2, 128, [129], None),
    (2, 7, 6, 2, 64, [31, 32], [7, 0]),
    (3, 13, 12, 4, 64, [0, 30, 700], [13, 1, 6]),
    (2, 16, 4, 4, 128, [255, 256], None),
    (2, 33, 3, 3, 128, [17, 1000], [33, 20]),
    (1, 64, 8, 1, 128, [40], None),
    (2, 64, 2, 1, 64, [95, 3], [64, 37]),
    (1, 26, 2, 2, 128, [3000], None),
    (5, 3, 2, 2, 128, [0, 1, 2, 3, 4], [1, 2, 3, 0, 1]),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,r,h,kvh,hd,lens,rows", ATTEND)
def test_attend(b, r, h, kvh, hd, lens, rows, dtype):
    rng = np.random.default_rng(sum(lens) + r + hd)
    used = rows or [r] * b
    cache = tree.TreeCache(2, b, h, kvh, hd, max(lens) + r + 5, max_rows=r, device=DEV)
    poison(cache)
    n = max(a + m for a, m in zip(lens, used))
    k, v = (rand(rng, b, n, kvh, hd, dtype="bf16") for _ in range(2))
    cache.append(1, k, v, rows=i32([a + m for a, m in zip(lens, used)]))
    cache.lens.copy_(i32(lens))
    q = rand(rng, b, r, h, hd, dtype=dtype)
    parents = [a_tree(rng, r) for _ in range(b)]
    kf, vf = f64(k), f64(v)
    drows = None if rows is None else i32(rows)
    outs = [cache.attend(1, q, parents=i32(parents), rows=drows, max_keys=mk) for mk in (0, max(n, 1 if rows else r))]
    for out in outs:
        check_attend(cache, 1, q, kf, vf, lens, used, parents, out, dtype)
    assert torch.equal(outs[0], cache.attend(1, q, parents=i32(parents), rows=drows))
    chain = [[i - 1 for i in range(r)]] * b
    check_attend(cache, 1, q, kf, vf, lens, used, chain, cache.attend(1, q, rows=drows, scale=0.05), dtype, 0.05)
    assert cache.device_error() == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,r,h,kvh", [(130, 3, 2, 1), (70, 40, 2, 2), (44, 3, 16, 16), (9, 5, 64, 64)])
def test_attend_large_batches(b, r, h, kvh, dtype):
    """More requests than a wave has lanes, their keys split or not; ragged lengths,
    requests without rows among them, whose output rows are zeros over what was there."""
    rng = np.random.default_rng(b + r)
    hd = 64
    cache = tree.TreeCache(1, b, h, kvh, hd, 900, max_rows=r, device=DEV)
    poison(cache)
    lens = [int(x) for x in np.exp(rng.uniform(0, math.log(800), b))]
    used = [int(x) for x in rng.integers(0, r + 1, b)]
    used[:3], used[-1] = [0, r, 0], 0
    n = max(a + m for a, m in zip(lens, used))
    k, v = (rand(rng, b, n, kvh, hd, dtype="bf16") for _ in range(2))
    cache.append(0, k, v, rows=i32([a + m for a, m in zip(lens, used)]))
    cache.lens.copy_(i32(lens))
    q = rand(rng, b, r, h, hd, dtype=dtype)
    parents = [a_tree(rng, r) for _ in range(b)]
    out = torch.full_like(q, 7)
    cache.attend(0, q, parents=i32(parents), rows=i32(used), out=out)
    assert cache.device_error() == 0
    some = list(range(0, b, max(1, b * r * h // 1500)))
    pick = torch.tensor(some, device=DEV)
    check_attend(cache, 0, q[pick], f64(k[pick]), f64(v[pick]), [lens[i] for i in some], [used[i] for i in some],
                 [parents[i] for i in some], out[pick], dtype)
    for i in range(b):
        assert not out[i, used[i]:].any() and torch.isfinite(out[i].float()).all()
    # a length outside the cache is flagged, also where a request uses no rows
    cache.lens[b - 1] = 901
    again = cache.attend(0, q, parents=i32(parents), rows=i32(used))
    assert cache.device_error() == spade.DERR_CAPACITY
    assert torch.equal(out, again)


def check_picks(picks, kvh, q, k, v, lens, rows, parents, out, dtype):
    """Like check_attend, for some (request, row, query head) of many."""
    h, hd = q.shape[2:]
    scale = hd ** -0.5
    for i, j, x in picks:
        if j >= rows[i]:
            assert not out[i, j, x].any()
            continue
        see = list(range(lens[i])) + [lens[i] + a for a in otree.lineage(parents[i], j)]
        kk, vv = (f64(t[i, :, x // (h // kvh)])[see] for t in (k, v))
        qq = f64(q[i, j, x])
        want = otree.attend(qq, kk, vv, scale)
        dz = 24 * U * scale * (np.abs(kk) @ np.abs(qq)).max() + 2 * U * scale * np.abs(kk @ qq).max()
        tol = 2 * np.abs(vv).max() * (2.1 * dz + 2.0 ** -22 + (3 * len(see) / 32 + 8) * U + (2.0 ** -17 if dtype == "bf16" else U))
        tol = tol + np.abs(want) * (HALF if dtype == "bf16" else U)
        err = np.abs(f64(out[i, j, x]) - want)
        assert (err <= tol).all(), (i, j, x, err.max(), tol.min())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("b,r,h,kvh,n", [(1, 33, 32, 32, 2900), (2, 64, 64, 64, 700), (1, 40, 200, 100, 3300), (2, 20, 80, 20, 4000),
                                         (1, 64, 32, 8, 13000), (4, 40, 128, 64, 150), (9, 61, 64, 64, 97), (3, 17, 200, 200, 40)])
def test_attend_many_rows(b, r, h, kvh, n, hd, dtype):
    """Trees of up to 64 nodes over heads and contexts enough that every kernel has its
    turn; ragged lengths, NaN in a row that only its descendants see."""
    rng = np.random.default_rng(n + hd)
    cache = tree.TreeCache(1, b, h, kvh, hd, n + r, max_rows=r, device=DEV)
    poison(cache)
    lens = [n] + [int(x) for x in rng.integers(0, n + 1, b - 1)]
    used = [r] + [int(x) for x in rng.integers(1, r + 1, b - 1)]
    gen = torch.Generator(device=DEV).manual_seed(n)
    k, v = (torch.randn(b, n + r, kvh, hd, generator=gen, device=DEV).bfloat16() for _ in range(2))
    cache.append(0, k, v, rows=i32([x + m for x, m in zip(lens, used)]))
    cache.lens.copy_(i32(lens))
    q = torch.randn(b, r, h, hd, generator=gen, device=DEV).to(TD[dtype])
    parents = [a_tree(rng, r) for _ in range(b)]
    out = cache.attend(0, q, parents=i32(parents), rows=i32(used))
    picks = [(int(rng.integers(b)), int(rng.integers(r)), int(rng.integers(h))) for _ in range(60)]
    picks += [(0, 0, 0), (0, r - 1, h - 1), (b - 1, r - 1, 0), (b - 1, used[-1] - 1, h - 1)]
    check_picks(picks, kvh, q, k, v, lens, used, parents, out, dtype)
    assert torch.isfinite(out.float()).all() and cache.device_error() == 0
    bad = r // 2
    broken = v.clone()
    broken[0, n + bad, kvh - 1, 7] = float("nan")
    cache.lens.zero_()
    cache.append(0, k, broken, rows=i32([x + m for x, m in zip(lens, used)]))
    cache.lens.copy_(i32(lens))
    again = cache.attend(0, q, parents=i32(parents), rows=i32(used))
    see = [i for i in range(r) if bad in otree.lineage(parents[0], i)]
    mask = torch.zeros_like(out, dtype=torch.bool)
    mask[0, see, h - h // kvh:, 7] = True
    assert torch.isnan(again)[mask].all() and torch.equal(again[~mask], out[~mask])


def test_attend_strided_rows():
    """Queries of a fused projection, outputs between other columns."""
    rng = np.random.default_rng(11)
    b, r, h, kvh, hd, lens = 2, 6, 4, 2, 64, [40, 9]
    cache = tree.TreeCache(1, b, h, kvh, hd, 60, max_rows=r, device=DEV)
    k, v = (rand(rng, b, 46, kvh, hd, dtype="bf16") for _ in range(2))
    cache.append(0, k, v)
    cache.lens.copy_(i32(lens))
    wide = rand(rng, b, r, h + 3, hd, dtype="bf16")
    q = wide[:, :, 1:1 + h]
    big = torch.full((b, r, h + 2, hd), 7.0, dtype=torch.bfloat16, device=DEV)
    parents = [a_tree(rng, r) for _ in range(b)]
    out = cache.attend(0, q, parents=i32(parents), out=big[:, :, 1:1 + h])
    check_attend(cache, 0, q, f64(k), f64(v), lens, [r] * b, parents, out, "bf16")
    assert (big[:, :, 0] == 7).all() and (big[:, :, -1] == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,r", [(0, 20), (31, 20), (100, 64), (2000, 9)])
def test_attend_is_not_touched_by_what_a_row_does_not_see(lens, r, dtype):
    """Infinities and NaN in keys and values of siblings, behind the last row and in
    rows not in use; the rows that see a value that is not finite get NaN."""
    rng = np.random.default_rng(lens + r)
    h, kvh, hd = 4, 2, 64
    n_used = r - 2
    cache = tree.TreeCache(1, 1, h, kvh, hd, lens + r + 40, max_rows=r, device=DEV)
    poison(cache)
    k, v = (rand(rng, 1, lens + r, kvh, hd, dtype="bf16") for _ in range(2))
    parents = a_tree(rng, r)
    parents[3] = 1
    parents[4] = 1
    for i in range(5, r):  # nobody sees row 4, some see row 3
        if parents[i] == 4:
            parents[i] = 3
    clean_k, clean_v = k.clone(), v.clone()
    k[0, lens + 4] = float("nan")
    v[0, lens + 4, :, ::3] = float("inf")
    v[0, lens + 4, :, 1::3] = float("nan")
    v[0, lens + 3, 1, 5] = float("-inf")
    v[0, lens + n_used:], k[0, lens + n_used:] = float("nan"), float("inf")
    cache.append(0, k, v)
    cache.lens.fill_(lens)
    q = rand(rng, 1, r, h, hd, dtype=dtype)
    out = cache.attend(0, q, parents=i32([parents]), rows=i32([n_used]))
    see3 = [i for i in range(n_used) if 3 in otree.lineage(parents, i)]
    assert len(see3) >= 1
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[0, see3, h // kvh:, 5] = True
    bad[0, 4] = True
    assert torch.isnan(out)[bad].all() and not torch.isnan(out)[~bad].any()
    cache.lens.zero_()
    cache.append(0, clean_k, clean_v)
    cache.lens.fill_(lens)
    want = cache.attend(0, q, parents=i32([parents]), rows=i32([n_used]))
    assert torch.equal(out[~bad], want[~bad])


def test_attend_nan_in_the_context_reaches_every_row():
    rng = np.random.default_rng(2)
    cache = tree.TreeCache(1, 1, 2, 1, 128, 600, max_rows=4, device=DEV)
    k, v = (rand(rng, 1, 500, 1, 128, dtype="bf16") for _ in range(2))
    v[0, 77, 0, 9] = float("nan")
    cache.append(0, k, v)
    cache.lens.fill_(496)
    q = rand(rng, 1, 4, 2, 128)
    out = cache.attend(0, q)
    assert torch.isnan(out[..., 9]).all() and torch.isnan(out).sum() == 8
    k[0, 30, 0, 3] = float("nan")
    cache.lens.zero_()
    cache.append(0, k, v)
    cache.lens.fill_(496)
    assert torch.isnan(cache.attend(0, q)).all()


def test_attend_flags_bad_parents_and_lengths():
    rng = np.random.default_rng(3)
    r = 5
    cache = tree.TreeCache(1, 2, 2, 1, 64, 50, max_rows=r, device=DEV)
    k, v = (rand(rng, 2, 50, 1, 64, dtype="bf16") for _ in range(2))
    cache.append(0, k, v)
    cache.lens.copy_(i32([10, 45]))
    q = rand(rng, 2, r, 2, 64)
    par = [[-1, 1, 7, -2, 2147483647], [0, 0, 1, 2, -2147483648]]
    out = cache.attend(0, q, parents=i32(par))
    assert cache.device_error() == spade.DERR_TREE
    fixed = [[-1, -1, -1, -1, -1], [-1, 0, 1, 2, -1]]
    assert torch.equal(out, cache.attend(0, q, parents=i32(fixed)))
    assert cache.device_error() == 0
    check_attend(cache, 0, q, f64(k), f64(v), [10, 45], [r, r], fixed, out, "f32")
    # lengths that leave the bound: cut to it and flagged, nothing is read out of the cache
    for lens, cut in (([46, 10], [45, 10]), ([-7, 0], [0, 0]), ([2147483647, -2147483648], [45, 0])):
        cache.lens.copy_(i32(lens))
        out = cache.attend(0, q)
        assert cache.device_error() == spade.DERR_CAPACITY
        check_attend(cache, 0, q, f64(k), f64(v), cut, [r, r], [[i - 1 for i in range(r)]] * 2, out, "f32")
    cache.lens.copy_(i32([10, 10]))
    out = cache.attend(0, q, rows=i32([9, -3]), max_keys=12)
    assert cache.device_error() == spade.DERR_CAPACITY
    check_attend(cache, 0, q, f64(k), f64(v), [7, 10], [5, 0], [[i - 1 for i in range(r)]] * 2, out, "f32")


@pytest.mark.parametrize("dtype,g,r,n", [("bf16", 4, 32, 40000), ("f32", 1, 3, 70001), ("bf16", 8, 64, 20011)])
def test_attend_long_contexts(dtype, g, r, n):
    """Many splits; rows against the formulas in double."""
    rng = np.random.default_rng(n)
    hd = 128
    cache = tree.TreeCache(1, 1, g, 1, hd, n + r, max_rows=r, device=DEV)
    k, v = (rand(rng, 1, n + r, 1, hd, dtype="bf16") for _ in range(2))
    cache.append(0, k, v)
    cache.lens.fill_(n)
    q = rand(rng, 1, r, g, hd, dtype=dtype)
    parents = a_tree(rng, r)
    out = cache.attend(0, q, parents=i32([parents]))
    for j in sorted({0, r // 2, r - 1}):
        see = np.array(list(range(n)) + [n + a for a in otree.lineage(parents, j)])
        for x in (0, g - 1):
            kk, vv, qq = f64(k[0, :, 0])[see], f64(v[0, :, 0])[see], f64(q[0, j, x])
            want = otree.attend(qq, kk, vv, hd ** -0.5)
            dz = 24 * U * hd ** -0.5 * (np.abs(kk) @ np.abs(qq)).max() + 2 * U * hd ** -0.5 * np.abs(kk @ qq).max()
            # (a wave's own keys of a split are few: the sums' roundings as those of 4096 keys)
            tol = 2 * np.abs(vv).max() * (2.1 * dz + 2.0 ** -22 + (3 * 4096 / 32 + 8) * U + (2.0 ** -17 if dtype == "bf16" else U))
            tol = tol + np.abs(want) * (HALF if dtype == "bf16" else U)
            assert (np.abs(f64(out[0, j, x]) - want) <= tol).all()


def test_attend_beyond_32_bit_offsets():
    """Heads behind the first 4 GiB of keys: the last of a large cache."""
    rng = np.random.default_rng(4)
    hd, n = 128, 1 << 20
    cache = tree.TreeCache(9, 1, 2, 2, hd, n, max_rows=2, device=DEV)  # 2 x 4.5 GiB
    k, v = (rand(rng, 1, 300, 2, hd, dtype="bf16") for _ in range(2))
    at = n - 300
    cache.lens.fill_(at)
    cache.append(8, k, v)
    kk, vv = cache.read(8, 300, start=cache.lens)
    assert torch.equal(kk, k) and torch.equal(vv, v)
    # a context of zeros: equal scores, so the last rows' values in their share
    for t in (cache.buf[:cache.buf.numel() // 2], cache.buf[cache.buf.numel() // 2:]):
        t.view(torch.bfloat16).reshape(9, 2, n * hd)[8].zero_()
    cache.append(8, torch.zeros_like(k), torch.full_like(v, 3.0))
    cache.lens.fill_(n - 2)
    q = rand(rng, 1, 2, 2, hd)
    out = cache.attend(8, q)
    # row 0 sees 299 of n - 1 positions with value 3, row 1 300 of n (sums of up to n terms 1 in
    # float32 over splits of 2048 positions are whole numbers; the quotient rounds)
    want = torch.tensor([3.0 * 299 / (n - 1), 3.0 * 300 / n], device=DEV)
    assert ((out[0, :, :, :] - want[:, None, None]).abs() <= 2.0 ** -20 * want[:, None, None]).all()
    assert cache.device_error() == 0


# --- commit ---------------------------------------------------------------------

COMMIT = [(1, 1, 1, 1, 64, [0]), (2, 3, 8, 2, 128, [5, 250, 31]), (3, 2, 64, 1, 64, [0, 700]), (1, 4, 33, 3, 128, [7, 8, 9, 255]),
          (2, 40, 5, 2, 64, list(range(40)))]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("layers,b,r,kvh,hd,lens", COMMIT)
def test_commit(layers, b, r, kvh, hd, lens, in_place):
    rng = np.random.default_rng(r * b + hd)
    cache = tree.TreeCache(layers, b, kvh, kvh, hd, max(lens) + r + 9, max_rows=1, device=DEV)
    n = cache.max_len
    hist = []
    for l in range(layers):
        cache.lens.zero_()
        k, v = (rand(rng, b, n, kvh, hd, dtype="bf16") for _ in range(2))
        cache.append(l, k, v)
        hist.append((k, v))
    cache.lens.copy_(i32(lens))
    rows = [int(x) for x in rng.integers(0, r + 1, b)]
    rows[0] = r
    parents = [a_tree(rng, r) for _ in range(b)]
    tokens = rng.integers(0, 3, (b, r))  # few tokens: several children match
    nxt = rng.integers(0, 3, (b, r))
    lens_out = None if in_place else torch.zeros(b, dtype=torch.int32, device=DEV)
    acc, path, corr = cache.commit(i32(tokens.tolist()), i32(parents), i32(nxt.tolist()), rows=i32(rows), lens_out=lens_out)
    got_lens = (cache.lens if in_place else lens_out).tolist()
    if not in_place:
        assert cache.lens.tolist() == lens
    read = [cache.read(l, n) for l in range(layers)]
    for i in range(b):
        a, p, c = otree.walk(tokens[i], parents[i], nxt[i], rows[i])
        assert (int(acc[i]), int(corr[i]), got_lens[i]) == (a, c, lens[i] + a + 1)
        assert path[i].tolist() == p + [-1] * (r - len(p))
        for l in range(layers):
            for x in (0, 1):
                want = hist[l][x][i].clone()
                for j, s in enumerate(p):
                    want[lens[i] + j] = hist[l][x][i, lens[i] + s]
                assert torch.equal(read[l][x][i], want)
    assert cache.device_error() == 0


def test_commit_of_a_chain_and_refused_lengths():
    cache = tree.TreeCache(1, 4, 1, 1, 64, 20, max_rows=1, device=DEV)
    x = torch.ones(4, 20, 1, 64, device=DEV)
    cache.append(0, x, x)
    tokens = i32([[9, 1, 2, 3]] * 4)
    cache.lens.copy_(i32([4, 18, -1, 25]))
    before = cache.buf.clone()
    acc, path, corr = cache.commit(tokens, None, i32([[1, 2, 7, 8]] * 4))
    assert cache.device_error() == spade.DERR_CAPACITY
    assert acc.tolist() == [2, 1, -1, -1] and corr.tolist() == [7, 2, -1, -1]
    assert path.tolist() == [[0, 1, 2, -1], [0, 1, -1, -1], [-1] * 4, [-1] * 4]
    assert cache.lens.tolist() == [7, 20, -1, 25] and torch.equal(cache.buf, before)
    cache.lens.zero_()
    cache.commit(tokens, i32([[-1, 0, 2, -5]] * 4), i32([[1, 2, 7, 8]] * 4))
    assert cache.device_error() == spade.DERR_TREE


# --- together -------------------------------------------------------------------


class Decoder:
    """Two layers of attention and a residual product around the calls."""

    def __init__(self, seed, vocab=300, h=4, kvh=2, hd=64, layers=2, max_len=200, batch=2):
        g = torch.Generator().manual_seed(seed)
        d = h * hd
        m = lambda *s: (torch.randn(*s, generator=g) / math.sqrt(s[0])).to(DEV)
        self.embed, self.head = m(vocab, d) * math.sqrt(vocab), m(d, vocab) * 3.0
        self.qkv = [m(d, d + 2 * kvh * hd) for _ in range(layers)]
        self.o = [m(d, d) for _ in range(layers)]
        self.h, self.kvh, self.hd, self.vocab = h, kvh, hd, vocab
        self.cache = tree.TreeCache(layers, batch, h, kvh, hd, max_len, max_rows=64, device=DEV)
        freq, amp = tree.rotary_frequencies(48, 10000.0, "linear", 2.0, device=DEV)
        self.rope = tree.Rotary(freq, True, amp)
        self.sampler = sampling.Sampler(batch * 64, vocab, device=DEV)

    def logits(self, tokens, parents=None, depth=None, rows=None):
        b, r = tokens.shape
        x = self.embed[tokens.long()]
        for l in range(len(self.qkv)):
            y = x / x.pow(2).mean(-1, keepdim=True).sqrt()
            y = (y @ self.qkv[l]).reshape(b, r, self.h + 2 * self.kvh, self.hd)
            q, k, v = y[:, :, :self.h], y[:, :, self.h:self.h + self.kvh], y[:, :, self.h + self.kvh:]
            q = self.cache.append(l, k, v, q=q, rope=self.rope, depth=depth, rows=rows)
            a = self.cache.attend(l, q, parents=parents, rows=rows)
            x = x + a.reshape(b, r, -1) @ self.o[l]
        return (x @ self.head).reshape(b * r, self.vocab)


SETTINGS = [dict(temperature=0.0), dict(temperature=0.8, top_k=20, top_p=0.9), dict(temperature=1.2, min_p=0.02)]


@pytest.mark.parametrize("setting", range(len(SETTINGS)))
def test_trees_emit_what_token_by_token_sampling_emits(setting):
    """Uniforms belong to positions, so a tree whose drafts hold some of the right
    tokens and many wrong ones emits the same text, in fewer calls."""
    rng = np.random.default_rng(setting)
    B, steps, kw = 2, 24, SETTINGS[setting]
    u = torch.from_numpy(rng.random((B, 400), np.float32)).to(DEV)
    prompt = i32(rng.integers(0, 300, (B, 9)).tolist())

    def prefill(dec):
        dec.logits(prompt[:, :-1].contiguous())
        dec.cache.lens += 8

    one = Decoder(1)
    prefill(one)
    text, pend = [], prompt[:, -1:].contiguous()
    for i in range(steps):
        tok, _ = one.sampler.draw(one.logits(pend), u[:, i].contiguous(), **kw)
        one.cache.lens += 1
        text.append(tok.tolist())
        pend = tok[:, None].contiguous()
    text = np.array(text).T  # [B, steps]

    dec = Decoder(1)
    prefill(dec)
    pend, done, calls, R = prompt[:, -1].tolist(), [0] * B, 0, 14
    emitted = [[] for _ in range(B)]
    while min(done) < steps - 8:
        calls += 1
        par, tok, dep = [], [], []
        for b in range(B):
            p = a_tree(rng, R)
            d = otree.depths(p, R)
            t = [pend[b]] + [int(x) for x in rng.integers(0, 300, R - 1)]
            # a right path of random length: the first child of each row on it
            at = 0
            for _ in range(int(rng.integers(0, 5))):
                kids = [i for i in range(1, R) if p[i] == at]
                if not kids or done[b] + d[kids[-1]] > steps:
                    break
                at = kids[-1]
                t[at] = int(text[b, done[b] + d[at] - 1])
            par.append(p)
            tok.append(t)
            dep.append(d)
        tok, par_t, dep_t = i32(tok), i32(par), i32(dep)
        lg = dec.logits(tok, par_t, dep_t)
        at = torch.tensor(done, device=DEV)[:, None] + dep_t.long()
        nxt, _ = dec.sampler.draw(lg, torch.gather(u, 1, at).reshape(-1).contiguous(), **kw)
        n, path, corr = dec.cache.commit(tok, par_t, nxt.reshape(B, R))
        for b in range(B):
            kept = path[b, 1:int(n[b]) + 1].tolist()
            emitted[b] += [int(tok[b, i]) for i in kept] + [int(corr[b])]
            done[b] = len(emitted[b])
            pend[b] = int(corr[b])
    for b in range(B):
        m = min(steps, len(emitted[b]))
        assert emitted[b][:m] == text[b, :m].tolist()
        assert dec.cache.lens[b] == 8 + done[b]
    assert calls < min(done)
    assert dec.cache.device_error() == 0 and dec.sampler.device_error() == 0


def test_a_captured_step_equals_the_eager_one():
    """append, attend, sample and commit in a graph, replayed over growing lengths
    with eager work in between."""
    rng = np.random.default_rng(8)
    B, R = 2, 6
    a, c = Decoder(2), Decoder(2)
    for d in (a, c):
        d.logits(i32([[1, 2, 3, 4, 5]] * B))
        d.cache.lens.fill_(5)
    tok = i32([[7, 7, 8, 7, 9, 8]] * B)
    par, u = i32([[-1, 0, 0, 1, 2, 4]] * B), torch.rand(B * R, device=DEV)
    dep = i32([otree.depths([-1, 0, 0, 1, 2, 4], R)] * B)

    def step(d):
        lg = d.logits(tok, par, dep)
        nxt, chosen = d.sampler.draw(lg, u, temperature=0.9, top_p=0.95)
        return (lg, nxt, chosen) + d.cache.commit(tok, par, nxt.reshape(B, R))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(c)
    torch.cuda.current_stream().wait_stream(side)
    c.cache.lens.fill_(5)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = step(c)
    for i in range(5):
        u.copy_(torch.from_numpy(rng.random(B * R, np.float32)))
        tok.copy_(i32(rng.integers(0, 300, (B, R)).tolist()))
        want = step(a)
        # a tree that follows its own draws, so that rows move
        tok[:, 4] = want[1].reshape(B, R)[:, 2]
        tok[:, 2] = want[1].reshape(B, R)[:, 0]
        a.cache.lens.copy_(c.cache.lens)
        want = step(a)
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip(want, outs):
            assert torch.equal(x, y)
        assert torch.equal(a.cache.lens, c.cache.lens)
        ka, va = a.cache.read(1, 40, rows=a.cache.lens)
        kc, vc = c.cache.read(1, 40, rows=c.cache.lens)
        assert torch.equal(ka, kc) and torch.equal(va, vc)


def test_two_graphs_of_one_workspace():
    """Attention of few and of many rows captured over one cache, replayed in turn while
    the lengths change."""
    rng = np.random.default_rng(10)
    cache = tree.TreeCache(1, 3, 16, 4, 64, 6000, max_rows=64, device=DEV)
    k, v = (torch.from_numpy(rng.normal(size=(3, 6000, 4, 64)).astype(np.float32)).to(DEV) for _ in range(2))
    cache.append(0, k, v)
    par = [i32([a_tree(rng, r) for _ in range(3)]) for r in (3, 64)]
    qs = [rand(rng, 3, r, 16, 64, dtype="bf16") for r in (3, 64)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for q, p in zip(qs, par):
            cache.attend(0, q, parents=p)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for q, p in zip(qs, par):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = cache.attend(0, q, parents=p)
        graphs.append((g, out))
    other = tree.TreeCache(1, 3, 16, 4, 64, 6000, max_rows=64, device=DEV, buf=cache.buf)
    for lens in ([5000, 1, 700], [0, 0, 0], [5936, 5936, 5936], [64, 4000, 31]):
        cache.lens.copy_(i32(lens))
        other.lens.copy_(i32(lens))
        for g, _ in graphs + graphs[::-1]:
            g.replay()
        want = [other.attend(0, q, parents=p) for q, p in zip(qs, par)]
        torch.cuda.synchronize()
        for (_, out), w in zip(graphs, want):
            assert torch.equal(out, w)
    assert cache.device_error() == 0 and other.device_error() == 0


def test_calls_on_another_stream():
    """Caches and samplers of their own on two streams at once."""
    rng = np.random.default_rng(9)
    B, R = 2, 11
    decs = [Decoder(3), Decoder(3)]
    prompt = i32(rng.integers(0, 300, (B, 150)).tolist())
    par = i32([a_tree(rng, R)] * B)
    dep = i32([otree.depths(par[0].tolist(), R)] * B)
    toks = [i32(rng.integers(0, 300, (B, R)).tolist()) for _ in range(2)]
    u = torch.rand(B * R, device=DEV)

    def go(d, tok):
        for s in range(0, 150, 50):
            d.logits(prompt[:, s:s + 50].contiguous())
            d.cache.lens += 50
        lg = d.logits(tok, par, dep)
        return lg, d.sampler.draw(lg, u, top_k=40)[0]

    want = [go(d, t) for d, t in zip(decs, toks)]
    for d in decs:
        d.cache.lens.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for d, t, s in zip(decs, toks, streams):
        with torch.cuda.stream(s):
            got.append(go(d, t))
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert torch.equal(w[0], g[0]) and torch.equal(w[1], g[1])


def test_a_models_cache():
    """spade_prefill's keys and values as the tree's calls read them, rows of a tree
    behind them, and a model's own call after that."""
    from synth import ModelWeights, make_inputs, mini_workloads
    from oracle import Decoder as ODecoder
    from tests.helpers import gpu_prefill, gpu_setup, gpu_verify
    w = next(x for x in mini_workloads() if x.name == "mini_gqa_greedy")
    s = w.model
    weights = ModelWeights(s, w.seed)
    model, kv = gpu_setup(w, weights)
    inp = make_inputs(w)
    gpu_prefill(kv, inp)
    n = int(kv.get_state(1)[0][0])
    cache = tree.TreeCache.over(kv, max_rows=3)
    od = ODecoder(s, weights.get)
    oc = od.new_cache(n)
    od.prefill(oc, np.asarray(inp.prompts[0][:-1], dtype=np.int64))
    k, v = cache.read(0, n, dtype=torch.float32)
    for got, want in ((k, oc.k[0]), (v, oc.v[0])):
        want = np.asarray(want, np.float64)[:, :n].swapaxes(0, 1)
        # the same value rounded to bfloat16 on either side: a step apart at most, 2^-7 (and a
        # little of the row's size, from float32 sums of different orders)
        assert (np.abs(f64(got[0]) - want) <= 2.0 ** -7 * np.abs(want) + 2.0 ** -14 * np.abs(want).max()).all()
    before = gpu_verify(model, kv, inp)
    rng = np.random.default_rng(0)
    x = rand(rng, 1, 3, s.kv_heads, s.head_dim, dtype="bf16")
    q = rand(rng, 1, 3, s.n_heads, s.head_dim)
    cache.append(0, x, x)
    out = cache.attend(0, q, parents=i32([[-1, 0, 0]]), max_keys=n + 3)
    k, v = cache.read(0, n + 3, dtype=torch.float32)
    check_attend(cache, 0, q, f64(k), f64(v), [n], [3], [[-1, 0, 0]], out, "f32")
    after = gpu_verify(model, kv, inp)
    for a, b in zip(before[:3], after[:3]):
        np.testing.assert_array_equal(a, b)
    # what commit adds is the model's to know
    acc, _, corr = cache.commit(i32([[1, 2, 3]]), i32([[-1, 0, 0]]), i32([[3, 0, 9]]))
    assert kv.lens[0] == n + 2
    kv.set_state([n + 2], [int(corr[0])])
    assert kv.get_state(1)[0][0] == n + 2
    assert cache.device_error() == 0 and model.device_error() == 0


def test_over_refuses_other_caches():
    from types import SimpleNamespace
    with pytest.raises(ValueError):
        tree.TreeCache.over(SimpleNamespace(model=SimpleNamespace(shape=SimpleNamespace(kv_dtype="f32"))))


def test_the_binding_refuses():
    c = tree.TreeCache(1, 2, 4, 2, 64, 50, max_rows=4, device=DEV)
    x, q = torch.zeros(2, 3, 2, 64, device=DEV), torch.zeros(2, 3, 4, 64, device=DEV)
    f, _ = tree.rotary_frequencies(64, device=DEV)
    par = torch.zeros(2, 3, dtype=torch.int32, device=DEV)
    for bad in (lambda: c.append(0, x.half(), x), lambda: c.append(0, x, x.cpu()), lambda: c.append(0, x, x, q_out=q),
                lambda: c.append(0, x, x[:, :2]), lambda: c.append(0, x, x, q=q[..., :32]),
                lambda: c.append(0, x, x, depth=par[:1]), lambda: c.append(0, x, x, pos=par[0]),
                lambda: c.append(0, x, x, rope=tree.Rotary(f.cpu())), lambda: c.attend(0, q.half()),
                lambda: c.attend(0, q, parents=par.long()), lambda: c.attend(0, q, parents=par[:, :2]),
                lambda: c.attend(0, q.transpose(1, 2)), lambda: c.commit(par, par, par[:1]), lambda: c.commit(par[0], None, par[0]),
                lambda: c.commit(par, par, par, lens_out=par[0]), lambda: tree.Rotary(f.float()),
                lambda: c.read(0, 4, dtype=torch.float16)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: c.append(1, x, x), lambda: c.attend(0, torch.zeros(2, 5, 4, 64, device=DEV)),
                lambda: tree.TreeCache(1, 2, 4, 3, 64, 50, device=DEV), lambda: c.attend(0, q, out=q),
                lambda: c.append(0, x, x, rope=tree.Rotary(f[:6].contiguous()))):
        with pytest.raises(spade.SpadeError):
            bad()
