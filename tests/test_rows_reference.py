"""The plain forms that the row operators are tested against, pinned by hand-worked cases and by differences (no GPU)."""
import math

import numpy as np
import pytest

import rows_reference as ref


def test_route_by_hand():
    l = np.log(np.array([[1.0, 4.0, 2.0, 4.0], [3.0, 1.0, 1.0, 1.0]]))
    l[1, 2] = -math.inf
    w, ids = ref.route(l, 3, False)
    assert ids.tolist() == [[1, 3, 2], [0, 1, 3]]
    np.testing.assert_allclose(w, [[4 / 11, 4 / 11, 2 / 11], [3 / 5, 1 / 5, 1 / 5]], rtol=1e-14)
    w, ids = ref.route(l, 2, True)
    np.testing.assert_allclose(w, [[0.5, 0.5], [0.75, 0.25]], rtol=1e-14)
    w, ids = ref.route(np.array([[-math.inf, 2.0]]), 2, True)
    assert ids.tolist() == [[1, -1]] and w.tolist() == [[1.0, 0.0]]
    assert ref.route(np.full((1, 3), -math.inf), 2, False)[1].tolist() == [[-1, -1]]


@pytest.mark.parametrize("over_chosen", [False, True])
def test_route_gradient_by_differences(over_chosen):
    rng = np.random.default_rng(3)
    T, E, k, h = 4, 7, 3, 1e-6
    l, dw = rng.standard_normal((T, E)), rng.standard_normal((T, k))
    w, ids = ref.route(l, k, over_chosen)
    got = ref.route_grad(l, w, ids, dw, over_chosen, E)
    for t in range(T):
        for e in range(E):
            up, down = l.copy(), l.copy()
            up[t, e] += h
            down[t, e] -= h
            slope = ((ref.route(up, k, over_chosen)[0] - ref.route(down, k, over_chosen)[0]) * dw).sum() / (2 * h)
            assert abs(slope - got[t, e]) < 1e-8


def test_sort_by_hand():
    offsets, order, place = ref.sort(np.array([2, 0, -1, 2, 1, 0, 5]), 4)
    assert offsets.tolist() == [0, 2, 3, 5, 5]
    assert order.tolist() == [1, 5, 4, 0, 3]
    assert place.tolist() == [3, 0, -1, 4, 2, 1, -1]


def test_combine_gradient_by_differences():
    rng = np.random.default_rng(4)
    T, k, D, h = 3, 2, 4, 1e-6
    place = np.array([[0, 3], [-1, 1], [2, -1]])
    z, w, dy = rng.standard_normal((4, D)), rng.standard_normal((T, k)), rng.standard_normal((T, D))
    dz, dw, _ = ref.combine_grad(dy, z, place, w)
    for array, slope in ((z, dz), (w, dw)):
        for at in np.ndindex(array.shape):
            keep = array[at]
            array[at] = keep + h
            up = (ref.combine(z, place, w)[0] * dy).sum()
            array[at] = keep - h
            down = (ref.combine(z, place, w)[0] * dy).sum()
            array[at] = keep
            assert abs((up - down) / (2 * h) - slope[at]) < 1e-8


def test_selection_by_hand():
    logits = np.log(np.array([[1.0, 1.0, 2.0], [1.0, 2.0, 1.0], [1.0, 1.0, 1.0]]))
    scores = np.array([math.log(0.5), math.log(0.25), -0.125])
    done = np.array([0, 0, 1])
    lists = ref.offers(logits, scores, done, 9)
    assert [t for _, t in lists[0]] == [2, 0, 1] and [t for _, t in lists[1]] == [1, 0, 2] and lists[2] == [(-0.125, 9)]
    # totals: beam 2 at e^-0.125 = 0.88; beam 0 at 1/4, 1/8, 1/8; beam 1 at 1/8, 1/16, 1/16
    ref.check_selection(np.array([-0.125, math.log(0.25)], np.float32), np.array([2, 0]), np.array([9, 2]), logits, scores, done, 9, 2)
    with pytest.raises(AssertionError):
        ref.check_selection(np.array([-0.125, math.log(0.25)], np.float32), np.array([2, 0]), np.array([9, 0]), logits, scores, done, 9, 2)
    with pytest.raises(AssertionError):
        ref.check_selection(np.array([math.log(0.25), -0.125], np.float32), np.array([0, 2]), np.array([2, 9]), logits, scores, done, 9, 2)
