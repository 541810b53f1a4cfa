"""The selections' oracle against hand-made cases, and its gradient against
central differences."""
import numpy as np
import pytest

import oracle.selection_oracle as S


def test_best_orders_ties_and_skips_what_is_no_number():
    assert S.best(np.array([1.0, np.nan, 3.0, 3.0, -np.inf, 0.0, -0.0]), 9) == [2, 3, 0, 5, 6]


def test_groups_choose_by_their_two_best():
    x = np.array([3.0, -9.0, 2.0, 2.0, 1.0, 1.0])
    c = S.route_values(x, "sigmoid", np.zeros(6), groups=3, topk_groups=1, group_top=2)
    assert np.isfinite(c).tolist() == [False, False, True, True, False, False]
    c = S.route_values(x, "sigmoid", np.zeros(6), groups=3, topk_groups=1, group_top=1)
    assert np.isfinite(c).tolist() == [True, True, False, False, False, False]


def test_a_masked_row_has_no_expert():
    x = np.full(5, -np.inf)
    for score in ("softmax", "sigmoid"):
        assert S.best(S.route_values(x, score), 3) == []


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_gradient_against_differences(score, renorm):
    rng = np.random.default_rng(3)
    x = rng.normal(size=9)
    chosen = S.best(S.route_values(x, score), 4)
    g = rng.normal(size=4)
    grad = S.route_gradient(x, chosen, g, score, renorm, 1.5)
    h = 1e-5
    for e in range(9):
        d = np.zeros(9)
        d[e] = h
        up = S.route_weights(x + d, chosen, score, renorm, 1.5) @ g
        down = S.route_weights(x - d, chosen, score, renorm, 1.5) @ g
        # error of a central difference: h^2 / 6 of a third derivative below
        # 10, and the cancellation of 1e-16 over 2 h
        assert abs((up - down) / (2 * h) - grad[e]) < 1e-9


def test_beam_scores_are_a_distribution():
    rng = np.random.default_rng(4)
    s = S.beam_scores(rng.normal(size=(3, 50)), np.array([0.0, -1.0, -np.inf]))
    assert np.allclose(np.exp(s[0]).sum(), 1.0) and np.allclose(np.exp(s[1] + 1.0).sum(), 1.0)
    assert np.all(s[2] == -np.inf)


def test_kept_slots_and_step_slot():
    acc = np.array([5.0, 1.0, 3.0, 3.0, np.nan, 9.0, 0.0])
    pos = np.arange(7)
    assert S.kept_slots(acc, pos, 7, 4, 1, 1) == [0, 2, 5, 6]
    assert S.kept_slots(acc, pos, 7, 7, 0, 0) == list(range(7))
    assert S.kept_slots(acc, np.array([3, -1, 1, 0, 2, -1, 4]), 5, 2, 0, 1) == [0, 6]
    assert S.step_slot(acc, pos, 7, 1, 2) == 4
    assert S.step_slot(np.array([5.0, 1.0, 1.0]), np.array([0, 1, 2]), 3, 0, 1) == 1
    assert S.step_slot(acc, np.array([0, 1, 2, -1, 4, -1, 6]), 7, 0, 1) == 3
    assert S.step_slot(np.ones(3), np.array([0, 5, 6]), 7, 1, 3) == 0
