"""Trees of drafts and filtered sampling without a GPU: buffer sizes, refusals on
the host, the rotation's frequencies, and the oracle's own pins."""

import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import tree as otree
from paper_2608_13076_amd import spade, tree

OK, EINVAL, ECAP, EUNSUP = 0, -1, -2, -4
PTR = 1 << 20  # an aligned address that no refused call touches


@pytest.fixture(scope="module")
def lib():
    return spade.load_library()


def shape(**kw):
    d = dict(n_layers=2, batch=3, n_heads=8, n_kv_heads=2, head_dim=128, max_len=1000)
    d.update(kw)
    return spade.TreeShape(*(d[k] for k in ("n_layers", "batch", "n_heads", "n_kv_heads", "head_dim", "max_len")))


def test_a_cache_is_a_models(lib):
    from synth import workload
    for name in ("c2_7b_greedy", "gqa_8b_greedy"):
        m = workload(name).model
        s = spade.TreeShape(m.n_layers, 3, m.n_heads, m.kv_heads, m.head_dim, 1000)
        cfg = spade.config_from(m)
        assert lib.spade_tree_bytes(ctypes.byref(s)) == lib.spade_kv_bytes(ctypes.byref(cfg), 3, 1000)


@pytest.mark.parametrize("kw", [dict(n_layers=0), dict(batch=0), dict(n_heads=0), dict(n_kv_heads=0),
                                dict(n_kv_heads=3), dict(head_dim=96), dict(head_dim=256), dict(max_len=0),
                                dict(max_len=(1 << 20) + 1), dict(batch=1 << 20, n_layers=1 << 10), dict(batch=-1)])
def test_bad_shapes(lib, kw):
    s = shape(**kw)
    assert lib.spade_tree_bytes(ctypes.byref(s)) == 0
    assert lib.spade_tree_workspace_bytes(ctypes.byref(s), 1) == 0
    assert lib.spade_last_error().decode()


def test_workspace_grows_with_the_rows(lib):
    s = shape()
    n = [lib.spade_tree_workspace_bytes(ctypes.byref(s), r) for r in (1, 2, 16, 64)]
    assert 0 < n[0] <= n[1] <= n[2] <= n[3]
    assert lib.spade_tree_workspace_bytes(ctypes.byref(s), 0) == 0
    assert lib.spade_tree_workspace_bytes(ctypes.byref(s), 65) == 0


def call_append(lib, s=None, rot=None, **kw):
    d = dict(layer=0, cache=PTR, B=3, R=2, dtype=1, q=1 << 24, q_ld=1024, k=1 << 25, k_ld=256, v=1 << 26, v_ld=256, pos=None,
             depth=None, lens=PTR, rows=None, qo=1 << 27, qo_ld=1024, err=None)
    d.update(kw)
    s = s or shape()
    return lib.spade_tree_append(ctypes.byref(s) if s != "null" else None, d["layer"], d["cache"], d["B"], d["R"],
                                 d["dtype"], d["q"], d["q_ld"], d["k"], d["k_ld"], d["v"], d["v_ld"],
                                 None if rot is None else ctypes.byref(spade.RotaryArgs(*rot)), d["pos"], d["depth"],
                                 d["lens"], d["rows"], d["qo"], d["qo_ld"], d["err"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(s="null"), EINVAL), (dict(layer=2), EINVAL), (dict(layer=-1), EINVAL), (dict(B=0), ECAP), (dict(B=4), ECAP),
    (dict(R=0), EINVAL), (dict(dtype=2), EINVAL), (dict(cache=None), EINVAL), (dict(k=None), EINVAL), (dict(v=None), EINVAL),
    (dict(lens=None), EINVAL), (dict(qo=None), EINVAL), (dict(q_ld=1020), EINVAL), (dict(k_ld=258), EINVAL),
    (dict(v_ld=252), EINVAL), (dict(k=PTR + 4), EINVAL), (dict(dtype=0, v=PTR + 8), EINVAL), (dict(qo_ld=1022), EINVAL),
    (dict(cache=PTR + 16), EINVAL), (dict(R=1 << 30), ECAP), (dict(rot=(PTR, 12, 0, 1.0)), EINVAL),
    (dict(rot=(PTR, 0, 0, 1.0)), EINVAL), (dict(rot=(PTR, 136, 0, 1.0)), EINVAL), (dict(rot=(None, 64, 0, 1.0)), EINVAL),
    (dict(rot=(PTR + 4, 64, 0, 1.0)), EINVAL), (dict(rot=(PTR, 64, 0, float("nan"))), EINVAL),
    (dict(rot=(PTR, 64, 0, float("inf"))), EINVAL), (dict(qo=1 << 24, qo_ld=1536), EINVAL), (dict(qo=(1 << 24) + 8), EINVAL),
    (dict(qo=1 << 25), EINVAL), (dict(qo=(1 << 26) + 5 * 512 + 504), EINVAL),
])
def test_append_refuses(lib, kw, want):
    assert call_append(lib, **kw) == want
    assert lib.spade_last_error().decode()


def call_attend(lib, s=None, **kw):
    d = dict(layer=0, cache=PTR, B=3, R=2, dtype=1, q=1 << 24, q_ld=1024, scale=0.1, parents=PTR, lens=PTR, rows=None,
             max_keys=0, out=1 << 25, out_ld=1024, ws=PTR, wsb=1 << 30, err=None)
    d.update(kw)
    s = s or shape()
    return lib.spade_tree_attend(ctypes.byref(s) if s != "null" else None, d["layer"], d["cache"], d["B"], d["R"],
                                 d["dtype"], d["q"], d["q_ld"], d["scale"], d["parents"], d["lens"], d["rows"],
                                 d["max_keys"], d["out"], d["out_ld"], d["ws"], d["wsb"], d["err"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(s="null"), EINVAL), (dict(layer=2), EINVAL), (dict(B=0), ECAP), (dict(B=4), ECAP), (dict(R=0), ECAP),
    (dict(R=65), ECAP), (dict(dtype=5), EINVAL), (dict(cache=None), EINVAL), (dict(q=None), EINVAL), (dict(out=None), EINVAL),
    (dict(lens=None), EINVAL), (dict(ws=None), EINVAL), (dict(q_ld=512), EINVAL), (dict(out=PTR + 4), EINVAL),
    (dict(cache=PTR + 128), EINVAL), (dict(ws=PTR + 64), EINVAL), (dict(scale=0.0), EINVAL), (dict(scale=-1.0), EINVAL),
    (dict(scale=float("inf")), EINVAL), (dict(scale=float("nan")), EINVAL), (dict(scale=2.0 ** 51), EINVAL),
    (dict(scale=2.0 ** -51), EINVAL), (dict(max_keys=1), ECAP), (dict(max_keys=1001), ECAP), (dict(wsb=0), ECAP),
    (dict(out=1 << 24), EINVAL), (dict(out=(1 << 24) + 2040), EINVAL),
])
def test_attend_refuses(lib, kw, want):
    assert call_attend(lib, **kw) == want
    assert lib.spade_last_error().decode()


def test_attend_refuses_a_small_workspace(lib):
    one = lib.spade_tree_workspace_bytes(ctypes.byref(shape()), 1)
    assert call_attend(lib, R=64, wsb=one) == ECAP


@pytest.mark.parametrize("kw,want", [(dict(layer=9), EINVAL), (dict(B=0), ECAP), (dict(R=0), EINVAL), (dict(k=None), EINVAL),
                                     (dict(v=PTR + 8), EINVAL), (dict(dtype=-1), EINVAL), (dict(cache=None), EINVAL),
                                     (dict(cache=PTR + 4), EINVAL), (dict(R=1 << 30), ECAP)])
def test_read_refuses(lib, kw, want):
    d = dict(layer=0, cache=PTR, B=3, R=2, dtype=0, k=PTR, v=PTR)
    d.update(kw)
    s = shape()
    assert lib.spade_tree_read(ctypes.byref(s), d["layer"], d["cache"], d["B"], d["R"], None, None, d["dtype"], d["k"],
                               d["v"], None) == want


@pytest.mark.parametrize("kw,want", [
    (dict(B=0), ECAP), (dict(B=4), ECAP), (dict(R=0), ECAP), (dict(R=65), ECAP), (dict(cache=None), EINVAL),
    (dict(cache=PTR + 8), EINVAL), (dict(tokens=None), EINVAL), (dict(nxt=None), EINVAL), (dict(lens=None), EINVAL),
    (dict(lo=None), EINVAL), (dict(n=None), EINVAL), (dict(path=None), EINVAL), (dict(corr=None), EINVAL),
    (dict(n=5 << 20), EINVAL), (dict(path=(3 << 20) - 8), EINVAL), (dict(corr=2 << 20), EINVAL),
    (dict(path=(6 << 20) - 8), EINVAL), (dict(lo=(4 << 20) + 8), EINVAL),
])
def test_commit_refuses(lib, kw, want):
    d = dict(cache=PTR, B=3, R=8, tokens=2 << 20, parents=None, nxt=3 << 20, rows=None, lens=4 << 20, lo=4 << 20, n=6 << 20,
             path=7 << 20, corr=8 << 20)
    if kw.get("n") == 5 << 20:
        d["rows"] = 5 << 20
    d.update(kw)
    s = shape()
    assert lib.spade_tree_commit(ctypes.byref(s), d["cache"], d["B"], d["R"], d["tokens"], d["parents"], d["nxt"], d["rows"],
                                 d["lens"], d["lo"], d["n"], d["path"], d["corr"], None, None) == want
    assert lib.spade_last_error().decode()


@pytest.mark.parametrize("kw,want", [
    (dict(rows=0), EINVAL), (dict(V=1), EINVAL), (dict(V=(1 << 20) + 1), EINVAL), (dict(dtype=2), EINVAL),
    (dict(logits=None), EINVAL), (dict(u=None), EINVAL), (dict(tokens=None), EINVAL), (dict(ws=None), EINVAL),
    (dict(per=0), EINVAL), (dict(ld=999), EINVAL), (dict(logits=PTR + 2), EINVAL), (dict(dtype=1, logits=PTR + 1), EINVAL),
    (dict(ws=(1 << 30) + 128), EINVAL), (dict(wsb=100), ECAP), (dict(probs=PTR + 4), EINVAL), (dict(probs=PTR, dtype=1), EINVAL),
    (dict(probs=PTR, ld=1004), EINVAL), (dict(probs=(1 << 28) + 2), EINVAL), (dict(tokens=PTR + 64), EINVAL),
    (dict(chosen=1 << 25), EINVAL), (dict(tokens=1 << 24), EINVAL), (dict(t=1 << 25), EINVAL), (dict(ld=(1 << 40) + 1), EINVAL),
])
def test_sample_refuses(lib, kw, want):
    d = dict(rows=4, V=1000, dtype=0, logits=PTR, ld=1000, per=1, t=None, u=1 << 24, tokens=1 << 25, chosen=None, probs=None,
             ws=1 << 30, wsb=1 << 30)
    d.update(kw)
    assert lib.spade_sample(d["rows"], d["V"], d["dtype"], d["logits"], d["ld"], d["per"], None, d["t"], None, None, None,
                            d["u"], d["tokens"], d["chosen"], d["probs"], d["ws"], d["wsb"], None, None) == want
    assert lib.spade_last_error().decode()


def test_sample_workspace(lib):
    n = [lib.spade_sample_workspace_bytes(r, v) for r, v in ((1, 2), (1, 128256), (64, 128256))]
    assert 0 < n[0] < n[1] < n[2]
    for r, v in ((0, 10), (1, 1), (1, (1 << 20) + 1), (1 << 30, 10)):
        assert lib.spade_sample_workspace_bytes(r, v) == 0


# --- the rotation's frequencies ---------------------------------------------


def test_frequencies():
    f, a = tree.rotary_frequencies(64, 10000.0, device="cpu")
    assert a == 1.0 and f[0] == 1.0 and abs(float(f[-1]) - 10000.0 ** (-62 / 64)) < 1e-15
    g, _ = tree.rotary_frequencies(64, 10000.0, "linear", 8.0, device="cpu")
    assert torch.equal(g, f / 8)
    g, _ = tree.rotary_frequencies(64, 10000.0, "base", 8.0, device="cpu")
    assert g[0] == f[0] and abs(float(g[-1] / f[-1]) - 1 / 8) < 1e-12
    for kind in ("bands", "ramp"):
        g, a = tree.rotary_frequencies(64, 10000.0, kind, 8.0, trained=4096, device="cpu")
        turns = 4096 * f / (2 * math.pi)
        r = g / f
        assert torch.equal(r[turns > 33], torch.ones_like(r[turns > 33]))
        assert torch.allclose(r[turns < 0.7], torch.full_like(r[turns < 0.7], 1 / 8), rtol=1e-14)
        assert (r[1:] <= r[:-1] + 1e-15).all()
        assert abs(a - (1.0 if kind == "bands" else 0.1 * math.log(8.0) + 1.0)) < 1e-15
    # a pair of 16.5 turns: half way between 1 and 32 on the line over the turns
    g, _ = tree.rotary_frequencies(2, 10000.0, "bands", 4.0, trained=1, slow=0.5 / math.pi * 0.5, fast=0.5 / math.pi * 1.5,
                                   device="cpu")
    assert abs(float(g[0]) - (0.5 + 0.5 / 4)) < 1e-12


@pytest.mark.parametrize("kw", [dict(rot_dim=7), dict(rot_dim=0), dict(rot_dim=8, theta=0.0), dict(rot_dim=8, factor=0.0),
                                dict(rot_dim=8, scaling="what"), dict(rot_dim=8, scaling="ramp", slow=2.0, fast=1.0),
                                dict(rot_dim=8, scaling="bands", trained=0)])
def test_frequencies_refuse(kw):
    with pytest.raises(ValueError):
        tree.rotary_frequencies(device="cpu", **kw)


@pytest.mark.parametrize("theta,rot", [(10000.0, 128), (500000.0, 64), (10000.0, 16)])
@pytest.mark.parametrize("factor", [4.0, 8.0])
@pytest.mark.parametrize("trained", [64, 4096, 8192, 65536, 131072, 1 << 20, 1 << 23])
def test_ramp_where_the_slowest_pairs_turn_often(trained, factor, theta, rot):
    """The line over the pairs' numbers, written out pair by pair: from the last whole
    number where a pair makes 32 turns or more to the first where it makes one or fewer,
    also where that is behind the last pair.  (In double: a power of up to 14 natural
    logarithms, 14 * 2^-53 by its argument's rounding, and a few roundings: below 1e-13.)"""
    n = rot // 2
    turns = [trained * theta ** (-2.0 * j / rot) / (2.0 * math.pi) for j in range(-8 * rot, 8 * rot)]
    lo = max(max(j for j, t in zip(range(-8 * rot, 8 * rot), turns) if t >= 32.0), 0)
    hi = min(min(j for j, t in zip(range(-8 * rot, 8 * rot), turns) if t <= 1.0), rot - 1)
    g, _ = tree.rotary_frequencies(rot, theta, "ramp", factor, trained=trained, device="cpu")
    for j in range(n):
        keep = 1.0 if j <= lo else 0.0 if j >= hi else (hi - j) / (hi - lo)
        f = theta ** (-2.0 * j / rot)
        want = f * keep + f / factor * (1.0 - keep)
        assert abs(float(g[j]) - want) <= 1e-13 * want, (j, lo, hi)
        if turns[8 * rot + j] > 1.0:  # only pairs of at most `slow` turns are divided in full
            assert float(g[j]) > f / factor * (1.0 + 1e-12)


@pytest.mark.parametrize("theta", [1.0, 0.5])
def test_ramp_refuses_frequencies_that_do_not_fall(theta):
    with pytest.raises(ValueError):
        tree.rotary_frequencies(64, theta, "ramp", 4.0, device="cpu")
    f, _ = tree.rotary_frequencies(64, theta, "bands", 4.0, device="cpu")  # (a band of turns needs no order)
    assert torch.isfinite(f).all()


# --- the oracle's pins -------------------------------------------------------


def test_oracle_rotation_is_a_complex_product():
    rng = np.random.default_rng(0)
    x, ang = rng.normal(size=(3, 64)), rng.normal(size=24)
    y = otree.rotate(x, ang, False, 1.5)
    z = (x[:, :24] + 1j * x[:, 24:48]) * 1.5 * np.exp(1j * ang)
    np.testing.assert_allclose(y, np.concatenate([z.real, z.imag, x[:, 48:]], -1), rtol=1e-13, atol=1e-13)
    y = otree.rotate(x, ang, True)
    z = (x[:, 0:48:2] + 1j * x[:, 1:48:2]) * np.exp(1j * ang)
    np.testing.assert_allclose(y[:, 0:48:2] + 1j * y[:, 1:48:2], z, rtol=1e-13, atol=1e-13)


def test_oracle_walk():
    tokens, parents = [9, 5, 6, 6, 7, 7], [-1, 0, 0, 2, 2, 2]
    assert otree.walk(tokens, parents, [6, 0, 7, 0, 3, 4], 6) == (2, [0, 2, 4], 3)
    assert otree.walk(tokens, parents, [6, 0, 7, 0, 3, 4], 4) == (1, [0, 2], 7)
    assert otree.walk(tokens, parents, [1] * 6, 6) == (0, [0], 1)
    assert otree.walk(tokens, parents, [1] * 6, 0) == (-1, [], -1)


def test_oracle_sample_distributions():
    l = np.log(np.array([0.1, 0.4, 0.05, 0.25, 0.2]))
    t, p = otree.sample(l, 0.3)
    np.testing.assert_allclose(p, [0.1, 0.4, 0.05, 0.25, 0.2], rtol=1e-12)
    np.testing.assert_allclose(otree.sample(l, 0.3, top_k=2)[1], [0, 0.4 / 0.65, 0, 0.25 / 0.65, 0], rtol=1e-12)
    np.testing.assert_allclose(otree.sample(l, 0.3, top_p=0.7)[1], np.array([0, 0.4, 0, 0.25, 0.2]) / 0.85, rtol=1e-12)
    np.testing.assert_allclose(otree.sample(l, 0.3, top_k=3, top_p=0.7)[1], np.array([0, 0.4, 0, 0.25, 0]) / 0.65, rtol=1e-12)
    np.testing.assert_allclose(otree.sample(l, 0.3, min_p=0.3)[1], np.array([0, 0.4, 0, 0.25, 0.2]) / 0.85, rtol=1e-12)
    assert otree.sample(l, 0.3, temperature=0.0)[0] == 1
    # ties go to the lowest ids
    assert otree.sample(np.zeros(8), 0.5, top_p=0.5)[1].tolist() == [0.25] * 4 + [0] * 4
    assert otree.sample(np.zeros(8), 0.5, top_k=3)[1].tolist() == [1 / 3] * 3 + [0] * 5
    # frequencies of the draw
    draws = np.bincount([otree.sample(l, u, top_k=3)[0] for u in np.random.default_rng(1).random(4000, np.float32)], minlength=5)
    want = 4000 * np.array([0, 0.4, 0, 0.25, 0.2]) / 0.85
    ok = want > 0
    assert draws[~ok].sum() == 0 and ((draws - want)[ok] ** 2 / want[ok]).sum() < 13.8  # chi-squared, 2 degrees, 0.001
