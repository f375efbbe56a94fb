"""The answers and distillation at the sizes whose kernels the other tests do not reach, each against the float64 oracle: rows of several tiles
by one wave each, bf16 rows that are read twice, listed classes that share their bits, and rows whose mass lies in one vector wherever a
tile or a part of a row begins or ends.

A few rows are computed by the oracle and laid out many times over where a kernel is chosen by the number of rows.  Bounds as in test_answers.py.
"""
import numpy as np
import pytest

from oracle import oracle as orc
from paper_2508_13716_amd import binding as B
from tests.test_answers import (EPS, bwd_tol, check, check_logprobs, device, distill_tol, given, hard_rows, run_bwd, run_distill, run_logprobs, stream, sum_err,
                                teacher_of, to_dtype)


def times_over(n, *arrays):
    """n rows of each array, its own rows in turn"""
    return [a[np.arange(n) % len(a)] for a in arrays]


def only(res, rows):
    return {key: v[rows] for key, v in res.items()}


# ----------------------------------------------------------------------------- answers: a wave a row, several tiles (2048 fp32, 4096 bf16 classes)
WAVES = [("f32", 2100, 5000, 5), ("f32", 2049, 8191, 64), ("f32", 2048, 16_384, 20), ("bf16", 2050, 9001, 10), ("bf16", 2048, 8192, 64), ("bf16", 2060, 16_001, 32)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n,C,k", WAVES)
def test_answers_of_several_tiles_by_one_wave(dtype, n, C, k):
    import torch
    rng = np.random.default_rng(C)
    base = hard_rows(40, C, dtype, C)
    mask40 = (rng.random(40) < 0.8).astype(np.uint8)
    for m, mk, T in ((3, None, 1.0), (70, mask40, 0.7)):
        ids = given(rng, 40, C, m)
        ref = orc.logprobs(base, ids, k, T, mk)
        Z, idn, = times_over(n, base, ids)
        mask = None if mk is None else times_over(n, mk)[0]
        if mask is not None:
            Z = Z.copy()
            Z[mask == 0] = np.nan
        Zd = device(Z, dtype, C + 3)
        res = run_logprobs(Zd, C, dtype, T, mask, idn, k)
        check_logprobs(res, {key: times_over(n, v)[0] for key, v in ref.items()}, Z, C, T)
        if mask is None:                                # without entropy: another kernel, the same numbers
            logp, top, top_logp = (torch.zeros(n, w, device="cuda", dtype=t) for w, t in ((m, torch.float32), (k, torch.int32), (k, torch.float32)))
            stats = torch.zeros(n, 2, device="cuda")
            B.logprobs(n, C, Zd, C + 3, B.BF16 if dtype == "bf16" else B.F32, T, None, torch.from_numpy(idn.copy()).cuda(), m, m, logp, m, None, stats, k, top, top_logp,
                       k, None, 0, stream=stream())
            torch.cuda.synchronize()
            for key, t in (("logp", logp), ("stats", stats), ("top_ids", top), ("top_logp", top_logp)):
                assert np.array_equal(t.cpu().numpy(), res[key], equal_nan=True), key


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n,C,k", WAVES)
def test_one_waves_rows_with_nan_and_infinity(dtype, n, C, k):
    base = hard_rows(12, C, dtype, 11)
    base[0, C // 3], base[0, C // 2] = np.nan, np.inf
    base[1, [1, C - 1, C // 2]] = np.inf
    base[4] = np.nan
    base[3, -1] = np.nan
    base[5, ::3] = np.nan
    ids = np.tile(np.array([[0, C // 2, C - 1, -1]], np.int32), (12, 1))
    with np.errstate(invalid="ignore", over="ignore"):
        ref = orc.logprobs(base, ids, k)
    Z, idn = times_over(n, base, ids)
    res = run_logprobs(device(Z, dtype, C + 1), C, dtype, 1.0, None, idn, k)
    np.testing.assert_array_equal(res["top_ids"], times_over(n, ref["top_ids"])[0])
    broken = np.isin(np.arange(n) % 12, [0, 1, 3, 4, 5])
    for key in ("logp", "top_logp", "entropy"):
        got = res[key][broken]
        assert np.isnan(got[..., :3] if key == "logp" else got).all(), key
    pick = np.flatnonzero(~broken)
    check_logprobs(only(res, pick), {key: v[pick % 12] for key, v in ref.items()}, Z[pick], C, 1.0)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["equal", "ascending", "descending", "two values", "late", "every 64th"])
@pytest.mark.parametrize("dtype,n,C", [("f32", 2048, 8000), ("bf16", 2049, 8200), ("f32", 2048, 16_001)])
def test_one_waves_rows_that_defeat_a_threshold(dtype, n, C, kind):
    rng = np.random.default_rng(7)
    j = np.arange(C)
    r = {"equal": np.full(C, 2.5), "ascending": j / C, "descending": -j / C, "two values": rng.integers(0, 2, C).astype(float),
         "late": np.where(j >= C - 700, 1.0 + j / C, 0.0), "every 64th": np.where(j % 64 == 5, 3.0 - j / C, 0.0)}[kind]
    Z = to_dtype(np.tile(r, (n, 1)), dtype)
    for k in (1, 17, 64) if C <= 8200 else (1, 17, 32):
        res = run_logprobs(device(Z, dtype, C), C, dtype, 1.0, None, np.zeros((n, 0), np.int32), k, ids_pad=1)
        ref = np.argsort(-Z[0], kind="stable")[:k]
        np.testing.assert_array_equal(res["top_ids"], np.tile(ref, (n, 1)))


# ----------------------------------------------------------------------------- distillation
@pytest.mark.gpu
@pytest.mark.parametrize("rest", [0, 1])
@pytest.mark.parametrize("dtype,dz_dtype,n,C,k", [("bf16", "bf16", 80, 70_001, 20), ("bf16", "f32", 140, 131_075, 5), ("bf16", "bf16", 40, 20_000, 30),
                                                  ("bf16", "f32", 35, 24_573, 9), ("f32", "f32", 70, 60_011, 20), ("f32", "bf16", 33, 36_000, 200)])
def test_distill_of_long_rows(dtype, dz_dtype, n, C, k, rest):
    """rows read twice (bf16 from 65537 classes on), and bf16 rows of 256 threads with twelve vectors each"""
    rng = np.random.default_rng(C + k)
    base = hard_rows(31, C, dtype, C)
    ids31, val31 = teacher_of(base, k, rest, 2.0, rng)
    mask31 = (rng.random(31) < 0.8).astype(np.uint8)
    weight = 2.0
    with np.errstate(divide="ignore", invalid="ignore"):
        _, row, dref, ex = orc.distill(base, ids31, val31, bool(rest), 2.0, mask31, 50.0, weight)
        row_tol, dz_tol = distill_tol(base, ex, row, dref, 2.0, C, k, weight, dz_dtype)
    Z, ids, val, mask, ref_row, rtol, dz, ztol = times_over(n, base, ids31, val31, mask31, row, row_tol, dref, dz_tol)
    Zd = device(Z, dtype, C + 3)
    loss, got, dZ = run_distill(Zd, C, dtype, dz_dtype, 2.0, mask, ids, val, rest, 50.0, weight, C + 1)
    check("row_loss", got, ref_row, rtol)
    check("dZ", dZ[:, :C], dz, ztol)
    base_dz = to_dtype(rng.standard_normal((n, C)), dz_dtype)
    _, _, acc = run_distill(Zd, C, dtype, dz_dtype, 2.0, mask, ids, val, rest, 50.0, weight, C + 2, base=base_dz)
    check("accumulated", acc[:, :C], base_dz + dz, ztol + np.abs(base_dz + dz) * (2.0 ** -8 if dz_dtype == "bf16" else 2 * EPS))
    if dtype == dz_dtype:
        got = run_distill(device(Z, dtype, C + 3, fill=5.0, offset=1), C, dtype, dz_dtype, 2.0, mask, ids, val, rest, 50.0, weight, 0, in_place=True)
        check("dZ in place", got[2][:, :C], dz, ztol)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n,C", [("f32", 1, 262_144 + 4099), ("bf16", 2, 262_144 + 4099), ("f32", 270, 262_144 + 4099), ("bf16", 270, 262_144 + 4099),
                                       ("f32", 600, 600_001), ("bf16", 500, 600_001), ("f32", 500, 600_001)])
def test_listed_classes_that_share_their_bits(dtype, n, C):
    """More classes than there are bits for: a class that is not listed and has all the mass lies exactly as far behind a listed one as the bits
    repeat (196608 classes in rows read twice, 262144 in parts); listed ones lie in the row's last vector, too."""
    rng = np.random.default_rng(C)
    T, rows = 1.0, 3
    base = rng.standard_normal((rows, C))
    ids = np.stack([rng.permutation(C)[:20] for _ in range(rows)]).astype(np.int32)
    ids[:, :8] = [5, 4097, C - 1, C - 2, 70_000, C - 196_608 - 1, 12, 65_543]
    for period in (196_608, 262_144, 1 << 18):
        for r in range(rows):
            for c in ids[r]:
                if c + period < C and c + period not in ids[r]:
                    base[r, c + period] = 9.0 + r
    base = to_dtype(base, dtype)
    val = np.log(np.full((rows, 20), 0.8 / 20)).astype(np.float32)
    _, row, dref, ex = orc.distill(base, ids, val, True, T, norm=50.0)
    assert (ex["P"] > 0.8).all()
    row_tol, dz_tol = distill_tol(base, ex, row, dref, T, C, 20, 1.0, dtype)
    import torch
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    Zd = torch.from_numpy(base).to(t).cuda()[torch.arange(n, device="cuda") % rows].contiguous()
    loss = torch.zeros(1, device="cuda")
    got, dZ = torch.zeros(n, device="cuda"), torch.full((n, C), 9.0, dtype=t, device="cuda")
    idd, vd = (torch.from_numpy(np.ascontiguousarray(times_over(n, x)[0])).cuda() for x in (ids, val))
    ws = torch.empty(B.distill_workspace_bytes(n, C), dtype=torch.uint8, device="cuda")
    dt = B.F32 if dtype == "f32" else B.BF16
    B.distill(n, C, Zd, C, dt, idd, vd, 20, 20, 1, T, None, 50.0, 1.0, loss, got, dZ, C, dt, 0, ws, ws.numel(), stream=stream())
    torch.cuda.synchronize()
    check("row_loss", got.cpu().numpy(), times_over(n, row)[0], times_over(n, row_tol)[0])
    for r in range(min(rows, n)):                       # the rows laid out again have the very bits
        assert bool((dZ[r::rows] == dZ[r]).all())
    m = min(rows, n)
    check("dZ", dZ[:m].float().cpu().numpy(), dref[:m], dz_tol[:m])


# ----------------------------------------------------------------------------- all of a row's mass in one vector
def spikes(C, dtype, at, rng):
    """rows with nearly all of their mass on the vector of classes that begins at `at[i]`"""
    V = 4 if dtype == "f32" else 8
    Z = 0.5 * rng.standard_normal((len(at), C))
    for i, p in enumerate(at):
        Z[i, p: p + V] += 15.0
    return to_dtype(Z, dtype)


def check_spikes(Z, at, dtype, T=1.0):
    n, C = Z.shape
    rng = np.random.default_rng(n)
    ids = np.stack([np.asarray(at), np.full(n, C - 1), rng.integers(0, C, n)], 1).astype(np.int32)
    k = 9
    ref = orc.logprobs(Z, ids, k, T)
    Zd = device(Z, dtype, C)
    res = run_logprobs(Zd, C, dtype, T, None, ids, k)
    check_logprobs(res, ref, Z, C, T)
    g, h = rng.standard_normal((n, 3)).astype(np.float32).astype(np.float64), rng.standard_normal(n).astype(np.float32).astype(np.float64)
    dref = orc.logprobs_bwd(Z, ids, g, h, T)
    check("dlogp", run_bwd(Zd, C, dtype, dtype, T, None, ref, ids, g, h, C), dref, bwd_tol(Z, ref, dref, ids, g, h, T, C, dtype))
    lists = np.stack([(np.asarray(at) + 97) % C, np.full(n, C // 2 + 1), (np.asarray(at) + 2000) % C], 1).astype(np.int32)
    val = np.log(np.full((n, 3), 0.2)).astype(np.float32)
    for rest in (0, 1):
        _, row, dref, ex = orc.distill(Z, lists, val, bool(rest), T)
        row_tol, dz_tol = distill_tol(Z, ex, row, dref, T, C, 3, 1.0, dtype)
        _, got, dZ = run_distill(Zd, C, dtype, dtype, T, None, lists, val, rest, 0.0, 1.0, C)
        check("row_loss", got, row, row_tol)
        check("dZ", dZ, dref, dz_tol)


def edges(C, dtype):
    """first vectors, last vectors and what is left of them at every multiple of 512 (every tile and every part begins at one), and at the row's end"""
    V = 4 if dtype == "f32" else 8
    return sorted({p for b in range(0, C, 512) for p in (b, b - V) if p >= 0} | {C - V, C // V * V if C % V else C - V, C - 1})


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,C", [("f32", 60_005), ("bf16", 70_003), ("bf16", 50_001), ("f32", 33_001), ("f32", 9_003), ("bf16", 20_005)])
def test_one_vector_holds_the_mass_of_each_of_many_rows(dtype, C):
    at = edges(C, dtype)
    rng = np.random.default_rng(C)
    for a in range(0, len(at), 120):
        part = at[a: a + 120] if len(at) - a >= 120 or a == 0 else at[-120:]
        check_spikes(spikes(C, dtype, part, rng), part, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,C", [("f32", 60_005), ("bf16", 70_003), ("f32", 131_075)])
def test_one_vector_holds_the_mass_of_a_few_rows(dtype, C):
    """one and three rows in parts: every vector next to the border of a part in one of the rows"""
    at = edges(C, dtype)
    rng = np.random.default_rng(C + 1)
    step = 3 if C < 100_000 else 9
    for a in range(0, len(at) - 2, step):
        part = at[a: a + 3]
        check_spikes(spikes(C, dtype, part, rng), part, dtype)
    for p in at[-4:] + at[:4] + at[len(at) // 2: len(at) // 2 + 4]:
        check_spikes(spikes(C, dtype, [p], rng), [p], dtype)


# ----------------------------------------------------------------------------- barred classes that are given or listed
@pytest.mark.gpu
@pytest.mark.parametrize("C", [11, 300, 9001])
def test_a_barred_class_that_is_given_or_listed_has_its_own_term_alone(C):
    T = 2.0
    Z = to_dtype(np.random.default_rng(C).standard_normal((2, C)), "f32")
    Z[:, 3] = -np.inf
    Z[:, 5] = -np.inf
    ids, g = np.array([[3, 1], [1, 3]], np.int32), np.array([[0.75, 0.5], [-1.0, 0.25]])
    ref = orc.logprobs(Z, ids, 0, T)
    dZ = run_bwd(device(Z, "f32", C), C, "f32", "f32", T, None, ref, ids, g, None, C)
    assert dZ[0, 3] == 0.375 and dZ[1, 3] == 0.125 and (dZ[:, 5] == 0.0).all()
    val = np.zeros((2, 2), np.float32)                  # q = 1/2 each
    loss, row, dZ = run_distill(device(Z, "f32", C), C, "f32", "f32", T, None, ids, val, 0, 2.0, 1.0, C)
    assert np.isposinf(row).all() and np.isposinf(loss) and (dZ[:, 3] == -0.125).all() and (dZ[:, 5] == 0.0).all()
