"""capgnn_distill with the teacher's remaining probability as one more outcome, where the classes that are not listed lie far from the row's
maximum, where there are none, and where the student is close to its teacher; and the divergence of equal logits without it.

EPS = 2^-24 is one float rounding; bounds are formed from the operations as in test_answers.py.
"""
import numpy as np
import pytest

from oracle import oracle as orc
from tests.test_answers import EPS, check, device, distill_tol, run_distill, sum_err, to_dtype

# (n, C, k, dtype): few classes, one to eight lanes a row; a wave, 256 and 512 threads a row; rows read twice; rows in parts
KERNELS = [(5, 2, 1, "f32"), (70, 40, 4, "f32"), (33, 47, 8, "bf16"), (9, 256, 100, "f32"), (7, 200, 20, "bf16"), (5, 600, 6, "f32"), (4, 3000, 70, "bf16"),
           (5, 7000, 8, "f32"), (3, 9001, 8, "bf16"), (3, 10_007, 8, "f32"), (2, 20_000, 8, "bf16"), (3, 30_001, 30, "f32"), (3, 40_003, 9, "bf16"),
           (45, 44_001, 8, "f32"), (90, 70_001, 5, "bf16"), (3, 60_001, 8, "f32"), (2, 131_077, 8, "bf16")]


def far_rows(n, C, k, dtype, T, gap, rng):
    """logits whose k listed classes lie gap * T above the others, a fifth of which is barred"""
    ids = np.stack([rng.permutation(C)[:k] for _ in range(n)]).astype(np.int32)
    Z = rng.standard_normal((n, C)) * T
    if C > 8:
        Z[rng.random((n, C)) < 0.2] = -np.inf
    np.put_along_axis(Z, ids.astype(np.int64), gap * T + rng.standard_normal((n, k)) * T, 1)
    return to_dtype(Z, dtype), ids


@pytest.mark.gpu
@pytest.mark.parametrize("gap,T", [(80.0, 1.0), (86.0, 1.0), (88.0, 0.5), (110.0, 2.0), (300.0, 1.0), (300.0, 0.125), (600.0, 0.5), (-120.0, 1.0)])
@pytest.mark.parametrize("n,C,k,dtype", KERNELS)
def test_others_far_from_the_listed_classes(n, C, k, dtype, gap, T):
    """p of the others leaves float's range: ln P is linear in their distance all the same, and their share of what the teacher leaves stays"""
    rng = np.random.default_rng(C + 1000 + int(gap))
    Z, ids = far_rows(n, C, k, dtype, T, gap, rng)
    q = 0.9 * rng.dirichlet(np.ones(k), n)
    val = np.log(q).astype(np.float32)
    val[0] += np.float32(np.log(1.0 / 0.9) - 1e-7)              # a row with hardly a remainder
    with np.errstate(divide="ignore", invalid="ignore"):
        ref_loss, ref_row, dref, ex = orc.distill(Z, ids, val, True, T, weight=T * T)
        row_tol, dz_tol = distill_tol(Z, ex, ref_row, dref, T, C, k, T * T, dtype)
    assert np.isfinite(ref_row).all() and (ex["r"][1:] > 0.05).all()
    # the gap itself carries one rounding of each of its operations, with all of q or r
    row_tol = row_tol + 4 * EPS * abs(gap)
    loss, row, dZ = run_distill(device(Z, dtype, C), C, dtype, dtype, T, None, ids, val, 1, 0.0, T * T, C)
    check("row_loss", row, ref_row, row_tol)
    check("dZ", dZ, dref, dz_tol)
    check("loss", loss, ref_loss, T * T / n * row_tol.sum() + 4 * EPS * abs(ref_loss))


@pytest.mark.gpu
@pytest.mark.parametrize("n,C,k,dtype", [c for c in KERNELS if c[1] > 8])
def test_a_large_factor_next_to_far_others_leaves_barred_classes_alone(n, C, k, dtype):
    """gradients of 2^40 and others of 2^-120: no product on the way leaves float's range, and a barred class keeps a gradient of 0"""
    rng = np.random.default_rng(C)
    Z, ids = far_rows(n, C, k, dtype, 1.0, 83.0, rng)
    val = np.log(np.full((n, k), 0.9 / k)).astype(np.float32)
    weight = 2.0 ** 40
    ref_loss, ref_row, dref, ex = orc.distill(Z, ids, val, True, 1.0, norm=1.0, weight=weight)
    row_tol, dz_tol = distill_tol(Z, ex, ref_row, dref, 1.0, C, k, weight, dtype)
    loss, row, dZ = run_distill(device(Z, dtype, C), C, dtype, dtype, 1.0, None, ids, val, 1, 1.0, weight, C)
    assert (dZ[np.isneginf(Z)] == 0.0).all()
    check("row_loss", row, ref_row, row_tol + 4 * EPS * 83)
    check("dZ", dZ, dref, dz_tol)


@pytest.mark.gpu
@pytest.mark.parametrize("noise", [0.02, 0.001])
@pytest.mark.parametrize("T", [1.0, 2.25])
@pytest.mark.parametrize("n,C,k,dtype", [(70, 40, 4, "f32"), (33, 47, 8, "bf16"), (9, 256, 100, "f32"), (9, 200, 20, "bf16"), (5, 600, 6, "f32"),
                                         (4, 3000, 70, "bf16"), (5, 7000, 8, "f32"), (3, 10_007, 64, "f32"), (3, 30_001, 64, "f32"),
                                         (45, 44_001, 64, "f32"), (3, 60_001, 64, "f32"), (2, 131_077, 64, "bf16")])
def test_small_divergences_with_most_of_the_mass_listed(n, C, k, dtype, T, noise):
    """A student close to its teacher, four fifths and more of both on the listed classes: the terms cancel to `noise` squared.  A listed
    class's q counts with its own ln q - ln p, the others' sum with P - r, and another temperature (T's reciprocal is a float) with q - p."""
    rng = np.random.default_rng(C + k)
    Z = rng.standard_normal((n, C)) * T
    ids = np.stack([rng.permutation(C)[:k] for _ in range(n)]).astype(np.int32)
    np.put_along_axis(Z, ids.astype(np.int64), T * (np.log(C / k) + 3.0 + rng.standard_normal((n, k))), 1)
    Z = to_dtype(Z, dtype)
    at = lambda v: np.take_along_axis(v, ids.astype(np.int64), 1)
    lp = at(orc.row_softmax(Z, T)[0])
    P = 1.0 - np.exp(lp).sum(1, keepdims=True)
    val = (lp + P * noise * (rng.standard_normal((n, k)) - 1.0)).astype(np.float32)
    _, ref, dref, ex = orc.distill(Z, ids, val, True, T)
    assert (ex["P"] < 0.5).all() and ref.max() < 3 * noise ** 2 and (ex["r"] > 2.0 ** -20).all()
    x = (Z.max(1, keepdims=True) - Z) / T
    p, q = at(ex["p"]), at(ex["q"])
    tol = EPS * (q * np.abs(np.log(q / p)) + np.abs(q - p) * at(x)).sum(1)
    tol += np.abs(ex["P"] - ex["r"]) * (sum_err(C) + EPS * x.max(1)) + 2 * EPS * ref + 1e-13
    _, row, _ = run_distill(device(Z, dtype, C), C, dtype, dtype, T, None, ids, val, 1, 0.0, 1.0, C)
    check("row_loss", row, ref, tol)


@pytest.mark.gpu
@pytest.mark.parametrize("z,T", [(0.0, 1.0), (3.75, 0.7), (-200.0, 3.0)])
@pytest.mark.parametrize("C,k", [(8, 4), (3, 3), (31, 31), (47, 8), (47, 47), (100, 33), (200, 128), (200, 200), (256, 256), (700, 7), (700, 200), (5000, 11),
                                 (10_007, 32), (30_000, 255), (60_001, 64), (150_000, 3)])
def test_equal_logits_without_a_remainder(C, k, z, T):
    """Equal logits on both sides: every exponential is 1 and every sum a whole number, so the divergence is ln(C / k) but for the roundings of
    q = 1/k, which count with it, and the result's own; 0 where every class is listed."""
    for n in (1, 300 if C <= 5000 else 60):
        Z = np.full((n, C), z)
        ids = np.tile(np.random.default_rng(C + k).permutation(C)[:k].astype(np.int32), (n, 1))
        val = np.full((n, k), -1.5, np.float32)
        ref = np.full(n, np.log(C / k))
        for dtype in ("f32", "bf16"):
            loss, row, dZ = run_distill(device(Z, dtype, C), C, dtype, "f32", T, None, ids, val, 0, 0.0, 1.0, C)
            check("row_loss", row, ref, 3 * EPS * ref + 1e-13)
            check("loss", loss, ref[0], 4 * EPS * ref[0] + 1e-13)


def listed_everywhere(C, k, scale, seed):
    """rows whose teacher lists every allowed class (some of the student's others are barred), log-probabilities formed in float as z / T - ln sum"""
    n, T = 40, 0.5
    rng = np.random.default_rng(seed)
    Z = scale * rng.standard_normal((n, C))
    ids = np.stack([rng.permutation(C)[:k] for _ in range(n)]).astype(np.int32)
    out = np.full((n, C), -np.inf)
    np.put_along_axis(out, ids.astype(np.int64), np.take_along_axis(Z, ids.astype(np.int64), 1), 1)
    Z = to_dtype(out, "f32")
    t = (np.take_along_axis(Z, ids.astype(np.int64), 1) + 0.1 * scale * rng.standard_normal((n, k))).astype(np.float32) / np.float32(T)
    top = t.max(1, keepdims=True)
    lse = np.log(np.exp(t - top).sum(1, keepdims=True, dtype=np.float32)) + top
    val = t - lse
    assert val.dtype == np.float32
    return Z, ids, val, T, 1.0 - np.exp(val.astype(np.float64)).sum(1)


LISTED_EVERYWHERE = [(8, 8), (47, 47), (100, 100), (200, 200), (47, 20), (700, 150), (9001, 64), (40_003, 100), (131_077, 30)]


def test_oracle_a_remainder_of_roundings_counts_as_none_where_there_is_no_other_class():
    Z, ids, val, T, r = listed_everywhere(8, 8, 100.0, 8)
    assert ((r >= 2.0 ** -20) & (r < 2.0 ** -13)).any()
    loss, row, dZ, ex = orc.distill(Z, ids, val, True, T)
    assert np.isfinite(row).all() and (ex["r"] == 0.0).all()
    val[:, 0] -= 0.5                                    # a teacher that does leave something: there the student has nothing to give
    loss, row, dZ, ex = orc.distill(Z, ids, val, True, T)
    big = 1.0 - np.exp(val.astype(np.float64)).sum(1) >= 2.0 ** -13
    assert big.any() and np.isposinf(row[big]).all() and np.isfinite(row[~big]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [3.0, 100.0, 300.0])
@pytest.mark.parametrize("C,k", LISTED_EVERYWHERE)
def test_a_remainder_of_roundings_counts_as_none_where_there_is_no_other_class(C, k, scale):
    Z, ids, val, T, r = listed_everywhere(C, k, scale, C + k)
    assert r.max() < 2.0 ** -13
    with np.errstate(divide="ignore", invalid="ignore"):
        ref_loss, ref_row, dref, ex = orc.distill(Z, ids, val, True, T)
        row_tol, dz_tol = distill_tol(Z, ex, ref_row, dref, T, C, k, 1.0, "f32")
    assert np.isfinite(ref_row).all()
    for rows in (slice(0, 1), slice(0, 40)):
        loss, row, dZ = run_distill(device(Z[rows], "f32", C), C, "f32", "f32", T, None, ids[rows], val[rows], 1, 40.0, 1.0, C)
        check("row_loss", row, ref_row[rows], row_tol[rows])
        check("dZ", dZ, dref[rows], dz_tol[rows])


@pytest.mark.gpu
@pytest.mark.parametrize("rest", [0, 1])
@pytest.mark.parametrize("C,k", [(1, 1), (1, 41), (1, 256), (2, 41), (5, 64), (7, 40), (7, 41), (9, 200), (250, 40), (250, 41)])
def test_lists_longer_than_rows_of_a_few_classes(C, k, rest):
    """rows shorter than 16 bytes next to lists of which most entries repeat a class or are none, on both sides of the longest list of few classes"""
    n = 70
    for dtype in ("f32", "bf16"):
        rng = np.random.default_rng(1000 * C + k + rest)
        Z = to_dtype(2 * rng.standard_normal((n, C)), dtype)
        ids = rng.integers(-1, C + 1, (n, k)).astype(np.int32)
        val = (np.log(0.9 / k) + 0.1 * rng.standard_normal((n, k)) - 0.2).astype(np.float32)
        with np.errstate(divide="ignore", invalid="ignore"):
            ref_loss, ref_row, dref, ex = orc.distill(Z, ids, val, bool(rest), 1.5)
            row_tol, dz_tol = distill_tol(Z, ex, ref_row, dref, 1.5, C, k, 1.0, dtype)
        loss, row, dZ = run_distill(device(Z, dtype, C + 1), C, dtype, dtype, 1.5, None, ids, val, rest, 0.0, 1.0, C + 2)
        check("row_loss", row, ref_row, row_tol)
        check("dZ", dZ[:, :C], dref, dz_tol)
        assert (dZ[:, C:] == 9.0).all()
