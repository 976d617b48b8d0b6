"""The oracle of the 4-bit cache against hand cases, its error bound, the tree attention and masks written out."""
import numpy as np
import pytest

import oracle


def test_codes_by_hand():
    x = np.zeros(40)
    x[:12] = [0.0, 6.0, -6.0, 0.25, 0.26, -0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.01]  # ties go to the even code
    x[12:16] = [7.0, -0.2, 4.9, -3.49]
    x[32:34] = [7.01, -1.0]                                                        # in the second block the scale is 2
    codes, scales = oracle.q4_encode(x)
    assert scales.tolist() == [127, 128] and codes.shape == (32,)
    nibbles = np.stack([codes & 15, codes >> 4], -1).reshape(-1)
    assert nibbles[:16].tolist() == [0, 7, 15, 0, 1, 10, 2, 4, 4, 6, 6, 7, 7, 0, 6, 13]
    assert nibbles[32:34].tolist() == [6, 9] and not nibbles[34:].any()
    assert oracle.q4_decode(codes, scales, 40)[[1, 2, 5, 12, 15, 32, 33]].tolist() == [6, -6, -1, 6, -3, 8, -1]


@pytest.mark.parametrize("dh", [8, 32, 80, 128])
def test_error_bound_and_idempotence(dh):
    rng = np.random.default_rng(dh)
    x = rng.standard_normal((50, dh)) * 2.0 ** rng.integers(-20, 20, (50, 1))
    codes, scales = oracle.q4_encode(x)
    back = oracle.q4_decode(codes, scales, dh)
    step = np.repeat(2.0 ** (scales.astype(float) - 127), 32, -1)[:, :dh]
    assert np.all(np.abs(back - x) <= step) and codes.shape == (50, 16 * -(-dh // 32))
    assert np.array_equal(oracle.q4_decode(*oracle.q4_encode(back), dh), back)


def test_ends_of_the_range():
    for v, s in ((0.0, 2), (1e-45, 2), (2.0 ** -126, 2), (7 * 2.0 ** -125, 2), (8 * 2.0 ** -125, 3), (7 * 2.0 ** 125, 252), (3.4e38, 252),
                 (np.inf, 255), (-np.inf, 255), (np.nan, 255)):
        x = np.zeros(32)
        x[3] = v
        codes, scales = oracle.q4_encode(x)
        assert scales[0] == s, v
        back = oracle.q4_decode(codes, scales, 32)
        assert np.isnan(back).all() if s == 255 else np.isfinite(back).all()
    assert not codes.any()


def _case(rng, H, Hkv, L, N, dh=8):
    f = lambda *s: rng.standard_normal(s)  # noqa: E731
    return f(H, N, dh), f(Hkv, L, dh), f(Hkv, L, dh), f(Hkv, N, dh), f(Hkv, N, dh)


def test_without_a_window_it_is_the_tree_attention():
    rng = np.random.default_rng(1)
    q, kc, vc, kt, vt = _case(rng, 4, 2, 7, 5)
    seen = np.tril(rng.random((5, 5)) < 0.6) | np.eye(5, dtype=bool)
    out, lse = oracle.window_attention(q, kc, vc, kt, vt, 5, seen, np.zeros(5, int), 0.3)
    of = np.arange(4) // 2
    assert np.allclose(out, oracle.tree_attention(q, kc[of], vc[of], 7, kt[of], vt[of], 5, seen, 0.3), atol=1e-13)
    want, want_lse = oracle.prefix_attention(q, kc[:, :0], vc[:, :0], kc, vc, kt, vt, 5, seen, 0.3)
    assert np.allclose(out, want) and np.allclose(lse, want_lse)
    wide, _ = oracle.window_attention(q, kc, vc, kt, vt, 5, seen, np.arange(5), 0.3, window=12)
    assert np.allclose(out, wide)


def test_a_window_by_hand():
    """Six cached rows, a chain of three nodes; a window of 3 and a sink of 1."""
    rng = np.random.default_rng(2)
    q, kc, vc, kt, vt = _case(rng, 1, 1, 6, 3)
    chain = np.tril(np.ones((3, 3), dtype=bool))
    out, _ = oracle.window_attention(q, kc, vc, kt, vt, 3, chain, np.arange(3), 1.0, window=3, sink=1)
    keys, values = np.concatenate([kc[0], kt[0]]), np.concatenate([vc[0], vt[0]])
    for i, sees in enumerate(([0, 4, 5, 6], [0, 5, 6, 7], [0, 6, 7, 8])):
        p = np.exp(keys[sees] @ q[0, i])
        assert np.allclose(out[0, i], p @ values[sees] / p.sum())
    out, _ = oracle.window_attention(q, kc, vc, kt, vt, 3, chain, np.arange(3), 1.0, window=1, sink=0)
    assert np.allclose(out[0], vt[0])  # every row its own key
