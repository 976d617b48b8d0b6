"""The oracle of the sampling filters against hand cases and the unfiltered draw."""
import numpy as np
import pytest

import oracle

LOGITS = np.log([0.1, 0.4, 0.05, 0.25, 0.2])  # order 1 3 4 0 2


@pytest.mark.parametrize("more,kept", [
    (dict(), [0, 1, 2, 3, 4]), (dict(top_k=2), [1, 3]), (dict(top_k=9), [0, 1, 2, 3, 4]), (dict(top_k=-1), [0, 1, 2, 3, 4]),
    (dict(top_p=0.39), [1]), (dict(top_p=0.41), [1, 3]), (dict(top_p=0.66), [1, 3, 4]), (dict(top_p=0.0), [1]), (dict(top_p=-1.0), [1]),
    (dict(top_k=2, top_p=0.6), [1]),               # 0.4 of 0.65 is 0.615
    (dict(top_k=3, top_p=0.7), [1, 3]),
    (dict(min_p=0.3), [1, 3, 4]), (dict(min_p=2.0), [1]), (dict(min_p=0.3, top_k=2), [1, 3]), (dict(top_p=float("nan"), min_p=float("nan")), [0, 1, 2, 3, 4]),
])
def test_filters_by_hand(more, kept):
    assert oracle.filter_tokens(LOGITS, 1.0, **more)[0].tolist() == kept


def test_ties_go_to_the_smaller_index():
    assert oracle.filter_tokens([1.0, 2.0, 2.0, 1.0, 2.0], 1.0, top_k=2)[0].tolist() == [1, 2]
    assert oracle.filter_tokens([0.0] * 10, 0.5, top_p=0.25)[0].tolist() == [0, 1, 2]
    assert oracle.filter_tokens([3.0, 3.0], 0.0)[0].tolist() == [0]


def test_draw_by_hand():
    assert oracle.sample_filtered(LOGITS, 0.0, 1.0, top_k=2) == (1, 2, pytest.approx(np.log(0.4 / 0.65)))
    assert oracle.sample_filtered(LOGITS, 0.62, 1.0, top_k=2)[0] == 3
    assert oracle.sample_filtered(LOGITS, 0.999999, -1.0) == (1, 1, 0.0)
    assert oracle.sample_filtered([-np.inf, np.nan], 0.5, 1.0) == (-1, 0, -np.inf)
    assert oracle.sample_filtered([5.0, np.inf, -np.inf, np.inf], 0.5, 1.0) == (3, 2, pytest.approx(np.log(0.5)))


def test_without_filters_it_is_the_plain_draw():
    rng = np.random.default_rng(0)
    for _ in range(200):
        z, u, t = rng.standard_normal(37) * 3, rng.random(), rng.uniform(0.2, 2)
        token, kept, logp = oracle.sample_filtered(z, u, t)
        assert token == oracle.sample_token(z, u, t) and kept == 37
        assert logp == pytest.approx(np.log(oracle.target_probs(z, t)[token]))
