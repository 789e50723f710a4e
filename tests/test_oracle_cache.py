"""Pins of the paged cache's oracle: closed forms and second formulations."""
import numpy as np
import pytest

from oracle import cache_oracle as O


def _cache(rng, b, hkv, dh, page, per, lens, evicts=False):
    n = b * per
    c = {"k": rng.standard_normal((n, hkv, page, dh)), "v": rng.standard_normal((n, hkv, page, dh)),
         "table": rng.permutation(n).reshape(b, per), "lens": np.array(lens)}
    if evicts:
        cap = per * page
        c["seen"] = np.array(lens) + 10
        c["slot_pos"] = np.stack([np.stack([rng.permutation(cap + 10)[:cap] for _ in range(hkv)]) for _ in range(b)])
        c["weights"] = rng.random((b, hkv, cap))
    return c


def _dense(c, name, b, h):
    return np.concatenate([c[name][p, h] for p in c["table"][b]])


def test_rows_land_behind_the_last_slot():
    rng = np.random.default_rng(0)
    c = _cache(rng, 2, 2, 4, 4, 3, [3, 0], evicts=True)
    before = [_dense(c, "k", b, 1).copy() for b in range(2)]
    k, v = rng.standard_normal((7, 2, 4)), rng.standard_normal((7, 2, 4))
    O.append(c, k, v, [5, 2], [[0, 1, 2, 3, 4], [6, 5]])
    want = before[0]
    want[3:8] = k[:5, 1]
    assert np.array_equal(_dense(c, "k", 0, 1), want)
    assert np.array_equal(_dense(c, "v", 1, 0)[:2], v[[6, 5], 0])
    assert list(c["lens"]) == [8, 2] and list(c["seen"]) == [18, 12]
    assert list(c["slot_pos"][0, 0, 3:8]) == [13, 14, 15, 16, 17] and not c["weights"][0, :, 3:8].any()
    O.append(c, k, v, [7, 0], [list(range(7)), []])     # only four slots are left
    assert c["lens"][0] == 12 and c["seen"][0] == 22


@pytest.mark.parametrize("window,sinks", [(0, 0), (3, 0), (3, 2), (1, 0), (50, 1)])
def test_attention_against_a_masked_softmax(window, sinks):
    rng = np.random.default_rng(1)
    n, m, hq, hkv, dh = 11, 6, 4, 2, 8
    c = _cache(rng, 1, hkv, dh, 4, 3, [n])
    q = rng.standard_normal((m, hq, dh))
    ref = O.attend(c, q, [0], [m], 0.3, window, sinks)
    total = np.zeros((hkv, 12))
    for h in range(hq):
        k, v = _dense(c, "k", 0, h // 2)[:n], _dense(c, "v", 0, h // 2)[:n]
        x = 0.3 * q[:, h] @ k.T
        t, s = np.arange(n - m, n)[:, None], np.arange(n)[None]
        see = s <= t
        if window:
            see = see & ((t - s < window) | (s < sinks))
        x = np.where(see, x, -np.inf)
        a = np.exp(x) / np.exp(x).sum(1, keepdims=True)
        assert np.allclose(ref["out"][:, h], a @ v, atol=1e-12)
        assert np.allclose(ref["lse"][:, h], np.log(np.exp(x).sum(1)), atol=1e-12)
        total[h // 2, :n] += a.sum(0)
    assert np.allclose(ref["probs"][0], total, atol=1e-12)
    assert np.isclose(ref["probs"].sum(), m * hq)


def test_positions_take_the_slots_place():
    """Shuffling a cache's rows with their positions changes nothing."""
    rng = np.random.default_rng(2)
    n, hkv, dh = 12, 2, 4
    c = _cache(rng, 1, hkv, dh, 4, 3, [n])
    q = rng.standard_normal((1, 4, dh))
    ref = O.attend(c, q, [0], [1], 0.5, 5, 2)
    perm = np.concatenate([rng.permutation(n - 1), [n - 1]])
    d = {**c, "seen": np.array([n]), "slot_pos": np.tile(perm, (1, hkv, 1)), "k": c["k"].copy(), "v": c["v"].copy()}
    for h in range(hkv):
        for name in "kv":
            x = _dense(c, name, 0, h)[perm]
            for s in range(n):
                p, r = O.row_of(d, 0, h, s)
                d[name][p, h, r] = x[s]
    got = O.attend(d, q, [0], [1], 0.5, 5, 2)
    assert np.allclose(got["out"], ref["out"], atol=1e-12) and np.allclose(got["lse"], ref["lse"], atol=1e-12)


def test_nothing_to_see():
    rng = np.random.default_rng(3)
    c = _cache(rng, 2, 1, 4, 4, 1, [0, 2])
    ref = O.attend(c, rng.standard_normal((4, 1, 4)), [0, 1], [1, 3], 1.0)
    assert np.isneginf(ref["lse"][[0, 1], 0]).all() and not ref["out"][:2].any()
    assert np.isfinite(ref["lse"][2:]).all()
    c["table"][1, 0] = 99
    assert np.isneginf(O.attend(c, rng.standard_normal((2, 1, 4)), [0, 1], [1, 1], 1.0)["lse"]).all()


def test_eviction_keeps_the_heaviest_and_the_protected():
    rng = np.random.default_rng(4)
    b, hkv, n, budget = 2, 3, 12, 7
    c = _cache(rng, b, hkv, 4, 4, 3, [n, 5], evicts=True)
    c["slot_pos"] = np.stack([np.stack([rng.permutation(n) for _ in range(hkv)]) for _ in range(b)])
    c["seen"][:] = n
    rows = {(h, int(c["slot_pos"][0, h, s])): (_dense(c, "k", 0, h)[s], _dense(c, "v", 0, h)[s], c["weights"][0, h, s])
            for h in range(hkv) for s in range(n)}
    untouched = c["weights"][1].copy()
    O.evict(c, budget, sinks=2, recent=2)
    assert list(c["lens"]) == [budget, 5] and np.array_equal(c["weights"][1], untouched)
    for h in range(hkv):
        left = {int(p) for p in c["slot_pos"][0, h, :budget]}
        assert len(left) == budget and {0, 1, 10, 11} <= left
        free = sorted((rows[h, p][2] for p in range(2, 10)), reverse=True)
        assert sorted((rows[h, p][2] for p in left - {0, 1, 10, 11}), reverse=True) == free[:3]
        for s in range(budget):
            k, v, w = rows[h, int(c["slot_pos"][0, h, s])]
            assert np.array_equal(_dense(c, "k", 0, h)[s], k) and np.array_equal(_dense(c, "v", 0, h)[s], v)
            assert c["weights"][0, h, s] == w


def test_eviction_ties_go_to_the_lower_slot_and_nan_goes_first():
    c = _cache(np.random.default_rng(5), 1, 1, 4, 4, 2, [8], evicts=True)
    c["slot_pos"][0, 0] = np.arange(100, 108)
    c["seen"][0] = 1000
    c["weights"][0, 0] = [1, np.nan, 1, 0, 2, -0.0, 1, np.inf]
    O.evict(c, 4)
    # kept: 7 (inf), 4 (2), 0 and 2 (the lower of the ones); holes 1 and 3 take 4 and 7
    assert list(c["slot_pos"][0, 0, :4]) == [100, 104, 102, 107]
