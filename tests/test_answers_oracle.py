"""The oracle of the answers (log-probabilities, entropy, top classes) and of distillation: closed forms, brute force, differences."""
import numpy as np
import pytest

from oracle import oracle as orc


def rows(n, C, seed, scale=2.0):
    return np.random.default_rng(seed).standard_normal((n, C)) * scale


def test_uniform_rows_and_barred_classes():
    Z = np.zeros((3, 8))
    Z[1, 4:] = -np.inf
    Z[2] = -np.inf
    r = orc.logprobs(Z, [[0, 5, -1], [0, 5, 8], [0, 1, 2]], 3)
    np.testing.assert_allclose(r["logp"][0], [-np.log(8), -np.log(8), 0.0])
    assert r["logp"][1, 0] == pytest.approx(-np.log(4)) and np.isneginf(r["logp"][1, 1]) and r["logp"][1, 2] == 0.0
    assert np.isneginf(r["logp"][2]).all()
    np.testing.assert_allclose(r["entropy"], [np.log(8), np.log(4), 0.0])
    np.testing.assert_array_equal(r["top_ids"], [[0, 1, 2]] * 3)


def test_order_of_ties_and_nan():
    Z = np.array([[1.0, 3.0, 3.0, 0.0], [-0.0, 0.0, -1.0, 0.0], [1.0, np.nan, 5.0, np.nan], [1.0, np.inf, np.nan, np.inf]])
    r = orc.logprobs(Z, np.zeros((4, 0)), 4)
    np.testing.assert_array_equal(r["top_ids"], [[1, 2, 0, 3], [0, 1, 3, 2], [1, 3, 2, 0], [2, 1, 3, 0]])


@pytest.mark.parametrize("T", [1.0, 0.5, 3.0])
def test_logprobs_gradient_is_the_difference_quotient(T):
    rng = np.random.default_rng(3)
    Z, ids = rows(4, 7, 1), rng.integers(-1, 7, (4, 5))
    g, h, mask = rng.standard_normal((4, 5)), rng.standard_normal(4), np.array([1, 1, 0, 1], np.uint8)
    Z[1, 2] = -np.inf

    def f(x):
        r = orc.logprobs(x, ids, 0, T, mask)
        return np.where(np.isfinite(r["logp"]), g * r["logp"], 0.0).sum() + (h * r["entropy"]).sum()

    dZ = orc.logprobs_bwd(Z, ids, np.where((ids == 2) & (np.arange(4)[:, None] == 1), 0.0, g), h, T, mask)
    for i in range(4):
        for j in range(7):
            if np.isneginf(Z[i, j]):
                assert dZ[i, j] == 0.0
                continue
            a, b = Z.copy(), Z.copy()
            a[i, j] += 1e-5
            b[i, j] -= 1e-5
            assert (f(a) - f(b)) / 2e-5 == pytest.approx(dZ[i, j], abs=2e-9 / T ** 2)


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("T", [1.0, 2.0])
def test_distill_gradient_is_the_difference_quotient(rest, T):
    rng = np.random.default_rng(5)
    Z = rows(5, 9, 2)
    ids = np.array([[0, 3, 5], [2, 2, 8], [-1, 9, 4], [-1, -1, 9], [1, 0, 7]])
    val = np.log(rng.dirichlet(np.ones(4), 5)[:, :3])
    val[4, 1] = -np.inf
    mask = np.array([1, 1, 1, 1, 0], np.uint8)
    loss, row, dZ, _ = orc.distill(Z, ids, val, rest, T, mask, weight=1.7)
    assert row[3] == 0.0 and (dZ[3] == 0.0).all() and (dZ[4] == 0.0).all()
    for i in range(5):
        for j in range(9):
            a, b = Z.copy(), Z.copy()
            a[i, j] += 1e-5
            b[i, j] -= 1e-5
            num = (orc.distill(a, ids, val, rest, T, mask, weight=1.7)[0] - orc.distill(b, ids, val, rest, T, mask, weight=1.7)[0]) / 2e-5
            assert num == pytest.approx(dZ[i, j], abs=1e-9)


def test_distill_from_itself_is_zero_and_from_one_class_is_cross_entropy():
    Z = rows(6, 11, 4)
    lp = orc.row_softmax(Z, 2.0)[0]
    ids = np.argsort(-Z, 1)[:, :4]
    val = np.take_along_axis(lp, ids, 1)
    loss, row, dZ, _ = orc.distill(Z, ids, val, True, 2.0)        # the same distribution: no divergence, no gradient
    assert abs(loss) < 1e-14 and np.abs(dZ).max() < 1e-15
    y = ids[:, :1]
    loss, _, dZ, _ = orc.distill(Z, y, np.zeros((6, 1)))
    ref, dref = orc.softmax_ce(Z, y[:, 0])
    assert loss == pytest.approx(ref) and np.allclose(dZ, dref, atol=1e-15)
