"""The plain 64-bit implementations that the GPU tests of routed products compare with, against what is known otherwise (no GPU)."""
import itertools

import numpy as np

import routed_util as ru


def test_gradient_of_the_weights_against_differences():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((4, 9))
    dw = rng.standard_normal((4, 3))
    for softmax, renormalise in itertools.product((True, False), repeat=2):
        _, at = ru.route(x, softmax, 3, renormalise=renormalise, scale=1.5)
        got = ru.route_backward(x, softmax, at, dw, renormalise, 1.5)

        def loss(y):
            s = np.take_along_axis(ru.scores(y, softmax), at, 1)
            return 1.5 * ((s / s.sum(axis=1, keepdims=True) if renormalise else s) * dw).sum()
        for t, e in itertools.product(range(4), range(9)):
            up, down = x.copy(), x.copy()
            up[t, e] += 1e-5
            down[t, e] -= 1e-5
            assert abs((loss(up) - loss(down)) / 2e-5 - got[t, e]) < 1e-8    # third derivatives of size one, times (1e-5)^2


def test_plan_by_hand():
    offsets, token_of, slot_of = ru.plan(np.array([[2, 0], [0, 5], [2, -1]]), 3)
    assert offsets.tolist() == [0, 2, 2, 4]
    assert token_of.tolist() == [0, 1, 0, 2, -1, -1]
    assert slot_of.tolist() == [[2, 0], [1, -1], [3, -1]]


def test_choice_by_hand():
    x = np.log(np.array([[1.0, 4.0, 2.0, 4.0, 3.0, 2.0]]))
    w, i = ru.route(x, True, 3)
    assert i.tolist() == [[1, 3, 4]] and np.allclose(w, [[4 / 11, 4 / 11, 3 / 11]])
    w, i = ru.route(x, True, 2, groups=3, top_groups=1, group_top=2)        # groups (1 4) (2 4) (3 2): sums 5, 6, 5
    assert i.tolist() == [[3, 2]]
    w, i = ru.route(x, True, 2, groups=3, top_groups=1, group_top=1)        # best 4, 4, 3: the first of the equal ones
    assert i.tolist() == [[1, 0]]
    w, i = ru.route(x, True, 1, bias=[0.0, 0, 0, 0, 0, 1.0], renormalise=False, scale=2.0)
    assert i.tolist() == [[5]] and np.allclose(w, 2.0 * 2 / 16)


def test_gradients_of_the_products_against_differences():
    rng = np.random.default_rng(2)
    A, B = rng.standard_normal((5, 4)), rng.standard_normal((3, 4, 6))
    offsets, rmap = np.array([0, 2, 2, 7]), np.array([4, 0, 0, 3, 1, 2, 9])
    dC = rng.standard_normal((7, 6))

    def loss(a, b):
        return (ru.grouped(a, offsets, 7, rmap, b)[0] * dC).sum()
    dB = ru.wgrad(A, offsets, 7, rmap, dC)[0]
    dA = ru.grouped(dC, offsets, 7, None, B.transpose(0, 2, 1))[0]
    slots = np.array([[np.nonzero(rmap == t)[0][j] if j < (rmap == t).sum() else -1 for j in range(2)] for t in range(5)])
    dA = ru.combine(dA, slots, None)[0]
    for i in np.ndindex(*A.shape):
        d = np.zeros_like(A)
        d[i] = 0.5
        assert abs(loss(A + d, B) - loss(A - d, B) - dA[i]) < 1e-12      # linear: differences are exact
    for i in np.ndindex(*B.shape):
        d = np.zeros_like(B)
        d[i] = 0.5
        assert abs(loss(A, B + d) - loss(A, B - d) - dB[i]) < 1e-12


def test_rounding_to_bfloat16():
    import gemm_inputs as gi
    rng = np.random.default_rng(3)
    x = rng.standard_normal(1000).astype(np.float32)
    assert np.array_equal(ru.rounded(x, "bf16"), gi.round_to_bfloat16(x).astype(np.float64))
