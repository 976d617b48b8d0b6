"""The oracle of the long-history operators against closed forms, the tree attention and invariants."""
import numpy as np
import pytest

import oracle


def _case(rng, H, Hkv, P, L, N, dh):
    f = lambda *s: rng.standard_normal(s)  # noqa: E731
    return f(H, N, dh), f(Hkv, P, dh), f(Hkv, P, dh), f(Hkv, L, dh), f(Hkv, L, dh), f(Hkv, N, dh), f(Hkv, N, dh)


@pytest.mark.parametrize("H,Hkv,P,L,N", [(2, 2, 5, 3, 4), (4, 2, 0, 6, 3), (6, 1, 9, 0, 5), (3, 3, 0, 0, 2)])
def test_prefix_attention_is_tree_attention_over_the_joined_keys(H, Hkv, P, L, N):
    rng = np.random.default_rng(P + L)
    q, kp, vp, kc, vc, kt, vt = _case(rng, H, Hkv, P, L, N, 8)
    seen = np.tril(rng.random((N, N)) < 0.6) | np.eye(N, dtype=bool)
    out, lse = oracle.prefix_attention(q, kp, vp, kc, vc, kt, vt, N, seen, 0.3)
    of = np.arange(H) // (H // Hkv)
    k, v = np.concatenate([kp, kc], 1)[of], np.concatenate([vp, vc], 1)[of]
    assert np.allclose(out, oracle.tree_attention(q, k, v, P + L, kt[of], vt[of], N, seen, 0.3), atol=1e-13)
    for h in range(H):
        s = 0.3 * (np.concatenate([k[h], kt[of][h]]) @ q[h].T)  # [keys, rows]
        s[P + L:][~seen.T] = -np.inf
        assert np.allclose(lse[h], np.log(np.exp(s).sum(0)))


def test_a_row_without_keys():
    rng = np.random.default_rng(0)
    q, kp, vp, kc, vc, kt, vt = _case(rng, 2, 1, 0, 0, 2, 4)
    out, lse = oracle.prefix_attention(q, kp, vp, kc, vc, kt, vt, 2, np.array([[False, False], [True, False]]), 1.0)
    assert np.all(out[:, 0] == 0) and np.all(np.isneginf(lse[:, 0]))
    assert np.allclose(out[:, 1], vt[0, 0]) and np.all(np.isfinite(lse[:, 1]))  # one key: its value


def test_weights_of_a_row_add_up_to_one():
    """With the lse of the same keys and no prefix, every accepted row hands out a weight of 1 per head."""
    rng = np.random.default_rng(3)
    H, Hkv, L, N = 4, 2, 7, 5
    q, kp, vp, kc, vc, kt, vt = _case(rng, H, Hkv, 0, L, N, 8)
    path = [0, 2, 4]
    seen = np.zeros((N, N), dtype=bool)
    for r, i in enumerate(path):
        seen[i, path[:r + 1]] = True
    _, lse = oracle.prefix_attention(q, kp, vp, kc, vc, kt, vt, N, seen, 0.5)
    added, fresh = oracle.weight_update(q, lse, kc, kt, path, 0.5)
    assert np.allclose(added.sum(1) + fresh.sum(1), len(path) * H // Hkv)
    assert np.all(added > 0) and fresh.shape == (Hkv, 3)


def test_evict_by_hand():
    # budget 4 of 7 rows: position 0 and the last two positions stay, then the heaviest of the others (row 1)
    weight, pos = [0.1, 0.9, 0.5, 0.2, 0.8, 0.0, 0.3], [0, 3, 4, 5, 1, 11, 10]
    assert list(oracle.evict(np.array(weight), np.array(pos), 12, 4, 1, 2)) == [0, 1, 5, 6]
    assert list(oracle.evict(np.array(weight), None, 0, 3, 0, 0)) == [4, 1, 2]
    assert list(oracle.evict(np.array(weight), None, 0, 9, 0, 0)) == list(range(7))


def test_evict_ties_and_numbers_that_are_none():
    assert list(oracle.evict(np.array([1.0, 1.0, 1.0, 2.0]), None, 0, 2, 0, 0)) == [0, 3]
    assert list(oracle.evict(np.array([np.nan, -np.inf, 0.0, np.nan]), None, 0, 3, 0, 0)) == [0, 1, 2]
    assert list(oracle.evict(np.array([np.nan, 5.0, np.inf]), None, 0, 1, 0, 0)) == [2]
    assert list(oracle.evict(np.array([-0.0, 0.0, 1.0]), None, 0, 2, 0, 0)) == [0, 2]


@pytest.mark.parametrize("seed", range(20))
def test_evict_keeps_a_set_that_nothing_beats(seed):
    rng = np.random.default_rng(seed)
    L, budget = int(rng.integers(1, 60)), int(rng.integers(3, 40))
    w = np.round(rng.random(L) * 8)
    kept = oracle.evict(w, rng.permutation(L), L, budget, 1, 2)
    n = min(L, budget)
    assert len(kept) == n and len(set(kept)) == n
    assert all(k == j or (k >= n and j not in kept) for j, k in enumerate(kept))
    rows = [k for j, k in enumerate(kept) if k >= n]
    assert rows == sorted(rows)
