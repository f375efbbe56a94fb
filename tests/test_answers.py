"""capgnn_logprobs, capgnn_logprobs_bwd and capgnn_distill against the float64 oracle, and what they refuse.

Tolerances, all from the operations.  EPS = 2^-24 is one float rounding.  A float sum of C positive terms, at least 64 partial sums wide,
is off by at most (C / 64 + 32) EPS of itself, and each term by 8 EPS + |its exponent| EPS: `sum_err`.  What is formed from the sum carries
that error; every further operation adds one rounding of its operands.  Results stored in bf16 add half a step, 2^-8 of the value.
"""
import numpy as np
import pytest

from oracle import oracle as orc
from paper_2508_13716_amd import binding as B
from paper_2508_13716_amd import synth

EPS = 2.0 ** -24
LOW = {"f32": -3.4028234663852886e38, "bf16": -3.3895313892515355e38}


# ----------------------------------------------------------------------------- refusals (no GPU: arguments are checked first)
def refuse(code, f, *a, **k):
    with pytest.raises(B.CapgnnError) as e:
        f(*a, **k)
    assert e.value.code == code, e.value


FAKE = 1 << 20          # an address that nothing reads


def logprobs_args(**kw):
    a = dict(n=4, n_classes=10, Z=FAKE, ldz=10, z_dtype=B.F32, temperature=1.0, mask=None, ids=FAKE, ldi=2, m=2, logp=FAKE, ldp=2,
             entropy=None, stats=None, k=3, top_ids=FAKE, top_logp=FAKE, ldt=3, ws=FAKE, ws_bytes=1 << 30)
    a.update(kw)
    return a


@pytest.mark.parametrize("bad", [
    dict(n=-1), dict(n_classes=0), dict(n_classes=-3), dict(z_dtype=2), dict(ldz=9), dict(Z=None), dict(Z=FAKE + 2), dict(Z=FAKE + 1, z_dtype=B.BF16),
    dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("inf")), dict(temperature=float("nan")), dict(temperature=1e-39), dict(temperature=1e20),
    dict(m=-1), dict(m=257, ldi=257, ldp=257), dict(ldi=1), dict(ldp=1), dict(ids=None), dict(logp=None),
    dict(k=-1), dict(k=11, ldt=11), dict(k=65, ldt=65, n_classes=100, ldz=100), dict(ldt=2), dict(top_ids=None, top_logp=None)])
def test_logprobs_refuses(bad):
    refuse(B.EINVAL, B.logprobs, **logprobs_args(**bad))


def bwd_args(**kw):
    a = dict(n=4, n_classes=10, Z=FAKE, ldz=10, z_dtype=B.F32, temperature=1.0, mask=None, stats=FAKE, entropy=FAKE, ids=FAKE, ldi=2, m=2,
             dlogp=FAKE, lddp=2, dentropy=FAKE, dZ=2 * FAKE, lddz=10, dz_dtype=B.F32)
    a.update(kw)
    return a


@pytest.mark.parametrize("bad", [
    dict(n=-1), dict(n_classes=0), dict(z_dtype=-1), dict(dz_dtype=7), dict(ldz=9), dict(lddz=9), dict(Z=None), dict(stats=None), dict(dZ=None),
    dict(entropy=None), dict(ids=None), dict(dlogp=None), dict(m=-1), dict(m=300, ldi=300, lddp=300), dict(ldi=1), dict(lddp=1), dict(temperature=0.0),
    dict(Z=FAKE + 2), dict(dZ=FAKE + 1, dz_dtype=B.BF16), dict(dZ=FAKE, lddz=11), dict(dZ=FAKE, dz_dtype=B.BF16)])
def test_logprobs_bwd_refuses(bad):
    refuse(B.EINVAL, B.logprobs_bwd, **bwd_args(**bad))


def distill_args(**kw):
    a = dict(n=4, n_classes=10, Z=FAKE, ldz=10, z_dtype=B.F32, teacher_ids=FAKE, teacher_val=FAKE, ldt=3, k=3, rest=0, temperature=1.0,
             mask=None, loss_norm=0.0, weight=1.0, loss_dev=FAKE, row_loss=None, dZ=2 * FAKE, lddz=10, dz_dtype=B.F32, accumulate=0, ws=FAKE,
             ws_bytes=1 << 30)
    a.update(kw)
    return a


@pytest.mark.parametrize("bad", [
    dict(n=-1), dict(n_classes=0), dict(z_dtype=3), dict(dz_dtype=3), dict(ldz=9), dict(lddz=9), dict(ldt=2), dict(Z=None), dict(teacher_ids=None),
    dict(teacher_val=None), dict(loss_dev=None), dict(k=0), dict(k=257, ldt=257), dict(rest=2), dict(temperature=0.0), dict(weight=float("nan")),
    dict(weight=float("inf")), dict(loss_norm=float("nan")), dict(Z=FAKE + 1), dict(dZ=FAKE, accumulate=1), dict(dZ=FAKE, lddz=12),
    dict(dZ=FAKE, dz_dtype=B.BF16), dict(ws=FAKE + 16)])
def test_distill_refuses(bad):
    refuse(B.EINVAL, B.distill, **distill_args(**bad))


def test_too_little_workspace_is_refused():
    refuse(B.ENOMEM, B.distill, **distill_args(ws=None))
    refuse(B.ENOMEM, B.distill, **distill_args(ws_bytes=B.distill_workspace_bytes(4, 10) - 1))
    for n, C in ((1, 200_000), (3, 1 << 20), (60, 50_000)):
        need = B.logprobs_workspace_bytes(n, C, 20)
        if need:
            a = logprobs_args(n=n, n_classes=C, ldz=C, k=20, ldt=20)
            refuse(B.ENOMEM, B.logprobs, **dict(a, ws_bytes=need - 1))
            refuse(B.ENOMEM, B.logprobs, **dict(a, ws=None))
            refuse(B.EINVAL, B.logprobs, **dict(a, ws=FAKE + 8))


def test_more_classes_than_offsets_hold_are_refused():
    C = (1 << 30) + 1
    refuse(B.EUNSUPPORTED, B.logprobs, **logprobs_args(n_classes=C, ldz=C))
    refuse(B.EUNSUPPORTED, B.logprobs_bwd, **bwd_args(n_classes=C, ldz=C, lddz=C))
    refuse(B.EUNSUPPORTED, B.distill, **distill_args(n_classes=C, ldz=C, lddz=C))


def test_no_rows_is_no_work():
    B.logprobs(**logprobs_args(n=0, Z=None, ids=None, logp=None))
    B.logprobs_bwd(**bwd_args(n=0, Z=None, dZ=None, stats=None))


# ----------------------------------------------------------------------------- inputs
def to_dtype(x, dtype):
    """float64 values that the type holds exactly"""
    x = np.asarray(x, np.float64)
    if dtype == "f32":
        return x.astype(np.float32).astype(np.float64)
    return synth.bf16_to_f32(synth.f32_to_bf16_rne(x.astype(np.float32)).reshape(x.shape)).reshape(x.shape).astype(np.float64)


def device(x, dtype, ld, fill=float("nan"), offset=0):
    """[n x ld] on the GPU, padding columns `fill`, starting `offset` elements into its allocation"""
    import torch
    n, C = x.shape
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    flat = torch.full((n * ld + offset,), fill, dtype=t, device="cuda")
    v = flat[offset:].view(n, ld)
    v[:, :C] = torch.from_numpy(np.ascontiguousarray(x)).to(t).cuda()
    return v


def hard_rows(n, C, dtype, seed, scale=2.0):
    """random rows, and among them (as far as n goes): an empty one, one of the type's lowest value, lowest values in barred places, equal logits
    throughout, ascending, descending, one class allowed, large offsets"""
    rng = np.random.default_rng(seed)
    Z = rng.standard_normal((n, C)) * scale
    Z[np.arange(n), rng.integers(0, C, n)] += 5.0
    special = [lambda r: np.full(C, -np.inf), lambda r: np.full(C, LOW[dtype]), lambda r: np.where(np.arange(C) % 3 == 1, LOW[dtype], r),
               lambda r: np.zeros(C), lambda r: np.arange(C) * (8.0 / C), lambda r: -np.arange(C) * (8.0 / C),
               lambda r: np.where(np.arange(C) == C // 2, 1.5, -np.inf), lambda r: r + 300.0, lambda r: np.where(np.arange(C) % 2, 0.0, -0.0),
               lambda r: np.where(np.arange(C) < C // 2, -np.inf, r)]
    for i, f in enumerate(special):
        if 1 + 3 * i < n:
            Z[1 + 3 * i] = f(Z[1 + 3 * i])
    return to_dtype(Z, dtype)


def sum_err(C):
    """relative error of a float sum of C exponentials (exponents up to 40 in base 2 where it matters: below that a term is 2^-40)"""
    return EPS * (C / 64 + 32 + 8 + 40)


def check(name, got, ref, tol):
    got, ref = np.asarray(got, np.float64), np.asarray(ref, np.float64)
    ref = np.where(np.abs(ref) > 3.4028235e38, np.copysign(np.inf, ref), ref)       # no float holds it: lowest value / 0.5 is -infinity
    same = (np.isnan(got) & np.isnan(ref)) | (got == ref)
    with np.errstate(invalid="ignore"):
        bad = ~(same | (np.abs(got - ref) <= tol))
    assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3], ref[bad][:3], np.broadcast_to(tol, ref.shape)[bad][:3])


def finite(x):
    return np.where(np.isfinite(x), x, 0.0)


# (n, C, pad, T): every size class of the kernels - a row per thread, several threads, a wave, a workgroup, several workgroups - and odd sizes
SIZES = [(1, 1, 0, 1.0), (70, 1, 2, 0.7), (333, 2, 0, 1.0), (257, 5, 0, 2.0), (1237, 8, 0, 1.0), (1030, 41, 0, 1.0), (515, 47, 1, 2.0), (300, 64, 0, 1.0),
         (200, 65, 0, 0.5), (130, 100, 28, 1.0), (77, 128, 0, 1.0), (90, 129, 0, 3.0), (65, 256, 0, 1.0), (41, 300, 1, 1.0), (33, 513, 0, 1.0),
         (35, 1000, 0, 0.7), (37, 2047, 0, 1.0), (34, 4096, 0, 1.0), (33, 4099, 5, 2.0), (31, 8200, 0, 1.0), (40, 10007, 5, 1.0), (1, 16384, 0, 1.0),
         (3, 40001, 0, 0.7), (2, 131072, 0, 1.0), (1, 150011, 3, 1.0), (300, 33000, 0, 1.0)]


def stream():
    import torch
    return torch.cuda.current_stream()


def run_logprobs(Zd, C, dtype, T, mask, ids, k, ids_pad=1):
    import torch
    n, ld = Zd.shape[0], Zd.stride(0)
    m = ids.shape[1]
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
    idd = np.full((n, m + ids_pad), 7, np.int32)
    idd[:, :m] = ids
    out = dict(logp=torch.full((n, m + 2), 77.0, device="cuda"), entropy=torch.full((n + 1,), 77.0, device="cuda"),
               stats=torch.full((n, 2), 77.0, device="cuda"), top_ids=torch.full((n, k + 3), 77, dtype=torch.int32, device="cuda"),
               top_logp=torch.full((n, k + 3), 77.0, device="cuda"))
    wb = B.logprobs_workspace_bytes(n, C, k)
    ws = torch.full((max(wb, 256),), 0xA5, dtype=torch.uint8, device="cuda")
    md, idd = (None if mask is None else dev(mask)), dev(idd)
    B.logprobs(n, C, Zd, ld, B.BF16 if dtype == "bf16" else B.F32, T, md, idd, m + ids_pad, m, out["logp"], m + 2, out["entropy"], out["stats"], k,
               out["top_ids"], out["top_logp"], k + 3, ws, wb, stream=stream())
    torch.cuda.synchronize()
    res = {key: v.cpu().numpy() for key, v in out.items()}
    assert (res["logp"][:, m:] == 77.0).all() and (res["entropy"][n:] == 77.0).all()
    assert (res["top_ids"][:, k:] == 77).all() and (res["top_logp"][:, k:] == 77.0).all()
    res["logp"], res["entropy"], res["top_ids"], res["top_logp"] = res["logp"][:, :m], res["entropy"][:n], res["top_ids"][:, :k], res["top_logp"][:, :k]
    return res


def check_logprobs(res, ref, Z, C, T):
    with np.errstate(invalid="ignore"):
        se = sum_err(C)
        tol = lambda lp: se + 8 * EPS * (np.abs(finite(lp)) + np.abs(finite(ref["stats"][:, 1:])))
        np.testing.assert_array_equal(res["top_ids"], ref["top_ids"])
        check("logp", res["logp"], ref["logp"], tol(ref["logp"]))
        check("top_logp", res["top_logp"], ref["top_logp"], tol(ref["top_logp"]))
        check("max", res["stats"][:, 0], ref["stats"][:, 0], 0.0)
        check("ln sum", res["stats"][:, 1], ref["stats"][:, 1], se + 2 * EPS * np.abs(finite(ref["stats"][:, 1])))
        # sum of e and of e * u, u to 160: both carry the sum's error, and the quotient two roundings
        check("entropy", res["entropy"], ref["entropy"], 2 * se * (1 + np.abs(finite(ref["entropy"]))) + 4 * EPS * np.abs(finite(ref["stats"][:, 1])))


def given(rng, n, C, m):
    ids = rng.integers(0, C, (n, m)).astype(np.int32)
    ids[rng.random((n, m)) < 0.1] = -1
    ids[rng.random((n, m)) < 0.05] = C
    if m > 1:
        ids[::3, 1] = ids[::3, 0]
    return ids


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,C,pad,T", SIZES)
def test_logprobs_vs_oracle(n, C, pad, T, dtype):
    rng = np.random.default_rng(1000 * C + n)
    Z = hard_rows(n, C, dtype, C + n)
    for k, m, use_mask in ((min(C, 5), 1, False), (min(C, 64), 3, True), (0, 0, False), (min(C, 9), 70, True), (1, 2, False)):
        mask = (rng.random(n) < 0.7).astype(np.uint8) if use_mask else None
        Zm = Z.copy()
        if mask is not None:
            Zm[mask == 0] = np.nan                  # rows that are not read
        ids = given(rng, n, C, m)
        res = run_logprobs(device(Zm, dtype, C + pad), C, dtype, T, mask, ids, k)
        check_logprobs(res, orc.logprobs(Z, ids, k, T, mask), Z, C, T)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,C", [(7, 47), (9, 300), (5, 5000), (5, 9001), (2, 140_000)])
def test_logprobs_rows_with_nan_and_infinity(n, C, dtype):
    Z = hard_rows(n, C, dtype, 11)
    Z[0, C // 3] = np.nan
    Z[0, C // 2] = np.inf
    Z[1, [1, C - 1, C // 2]] = np.inf
    if n > 4:
        Z[4] = np.nan
        Z[3, -1] = np.nan
    for k in (min(C, 8), min(C, 40)):
        ids = np.tile(np.array([[0, C // 2, C - 1, -1]], np.int32), (n, 1))
        res = run_logprobs(device(Z, dtype, C + 1), C, dtype, 1.0, None, ids, k)
        with np.errstate(invalid="ignore", over="ignore"):
            ref = orc.logprobs(Z, ids, k)
        np.testing.assert_array_equal(res["top_ids"], ref["top_ids"])
        broken = [0, 1] + ([3, 4] if n > 4 else [])
        for key in ("logp", "top_logp", "entropy"):
            got = res[key][broken]
            assert np.isnan(got[..., :3] if key == "logp" else got).all(), (key, got)
        assert (res["logp"][:, 3] == 0.0).all()
        ok = [i for i in range(n) if i not in broken]
        part = {key: v[ok] for key, v in ref.items()}
        check_logprobs({key: v[ok] for key, v in res.items()}, part, Z[ok], C, 1.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["equal", "ascending", "descending", "two values", "last wave", "first wave"])
def test_top_classes_of_rows_that_defeat_a_threshold(kind, dtype):
    rng = np.random.default_rng(7)
    for n, C in ((2, 3000), (3, 20_001), (1, 90_000), (600, 17_000)):
        r = {"equal": np.full(C, 2.5), "ascending": np.arange(C) / C, "descending": -np.arange(C) / C, "two values": rng.integers(0, 2, C).astype(float),
             "last wave": np.where(np.arange(C) >= C - 500, 1.0 + np.arange(C) / C, 0.0),
             "first wave": np.where(np.arange(C) % 8192 < 256, 5.0 - np.arange(C) / C, 0.0)}[kind]
        Z = to_dtype(np.tile(r, (n, 1)), dtype)
        for k in (1, 17, 64):
            res = run_logprobs(device(Z, dtype, C), C, dtype, 1.0, None, np.zeros((n, 0), np.int32), k, ids_pad=1)
            ref = np.argsort(-Z[0], kind="stable")[:k]
            np.testing.assert_array_equal(res["top_ids"], np.tile(ref, (n, 1)))


# ----------------------------------------------------------------------------- gradient of the answers
def run_bwd(Zd, C, dtype, dz_dtype, T, mask, ref, ids, g, h, lddz, in_place=False, offset=0):
    import torch
    n, ld, m = Zd.shape[0], Zd.stride(0), ids.shape[1]
    dev = lambda x, t=np.float32: torch.from_numpy(np.ascontiguousarray(x, t)).cuda()
    dt = {"f32": (B.F32, torch.float32), "bf16": (B.BF16, torch.bfloat16)}
    dZ = Zd if in_place else torch.full((n * lddz + offset,), 9.0, dtype=dt[dz_dtype][1], device="cuda")[offset:].view(n, lddz)
    args = [dev(ref["stats"]), dev(ref["entropy"]) if h is not None else None, dev(ids, np.int32), m, m, dev(g), m, None if h is None else dev(h)]
    md = None if mask is None else dev(mask, np.uint8)
    B.logprobs_bwd(n, C, Zd, ld, dt[dtype][0], T, md, *args, dZ, dZ.stride(0), dt[dz_dtype][0], stream=stream())
    torch.cuda.synchronize()
    return dZ.float().cpu().numpy()


def bwd_tol(Z, ref, dref, ids, g, h, T, C, dz_dtype):
    """p carries the error of ln sum; the factor G + h (ln p + H) one rounding of each part and the errors of ln p and H; the given
    classes' sum one rounding a term"""
    lp, p, _, ln_s = orc.row_softmax(Z, T)
    p = np.where(np.isneginf(ln_s)[:, None], 0.0, p)
    se = sum_err(C)
    inside = (ids >= 0) & (ids < C)
    G = np.where(inside, np.abs(g), 0.0).sum(1, keepdims=True)
    hh = np.zeros((len(Z), 1)) if h is None else np.abs(h)[:, None]
    lpf = np.abs(finite(np.where(p == 0, 0.0, lp)))
    H = np.abs(finite(ref["entropy"]))[:, None]
    factor = G + hh * (lpf + H)
    err = p * (factor * (se + 16 * EPS + 2 * EPS * lpf) + (ids.shape[1] + 4) * EPS * G + hh * (2 * se * (1 + H) + 8 * EPS * (lpf + H + np.abs(finite(ln_s))[:, None])))
    onto = np.zeros_like(p)
    for a in range(ids.shape[1]):
        ok = np.flatnonzero(inside[:, a])
        np.add.at(onto, (ok, ids[ok, a]), np.abs(g[ok, a]))
    err = (err + onto * (ids.shape[1] + 4) * EPS) / T
    return err * 2 + np.abs(dref) * (2.0 ** -8 if dz_dtype == "bf16" else 2 * EPS) + 1e-38


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,dz_dtype", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("n,C,pad,T", SIZES)
def test_logprobs_bwd_vs_oracle(n, C, pad, T, dtype, dz_dtype):
    rng = np.random.default_rng(77 * C + n)
    Z = hard_rows(n, C, dtype, C + 2 * n)
    for m, use_mask, use_h in ((1, False, True), (3, True, True), (70, False, False), (0, True, True), (2, True, False)):
        mask = (rng.random(n) < 0.7).astype(np.uint8) if use_mask else None
        Zm = Z.copy()
        if mask is not None:
            Zm[mask == 0] = np.nan
        ids, g = given(rng, n, C, m), rng.standard_normal((n, m)).astype(np.float32).astype(np.float64)
        h = rng.standard_normal(n).astype(np.float32).astype(np.float64) if use_h else None
        ref = orc.logprobs(Z, ids, 0, T, mask)
        dref = orc.logprobs_bwd(Z, ids, g, h, T, mask)
        tol = bwd_tol(Z, ref, dref, ids, g, h, T, C, dz_dtype)
        got = run_bwd(device(Zm, dtype, C + pad), C, dtype, dz_dtype, T, mask, ref, ids, g, h, C + 3)
        assert (got[:, C:] == 9.0).all()
        check("dZ", got[:, :C], dref, tol)
        if dtype == dz_dtype:                       # in place, from an odd address
            Zd = device(Zm, dtype, C + pad, fill=5.0, offset=1)
            got = run_bwd(Zd, C, dtype, dz_dtype, T, mask, ref, ids, g, h, 0, in_place=True)
            assert (got[:, C:] == 5.0).all()
            check("dZ in place", got[:, :C], dref, tol)


# ----------------------------------------------------------------------------- distillation
def run_distill(Zd, C, dtype, dz_dtype, T, mask, ids, val, rest, norm, weight, lddz, base=None, in_place=False, want_dz=True):
    import torch
    n, ld, k = Zd.shape[0], Zd.stride(0), ids.shape[1]
    dt = {"f32": (B.F32, torch.float32), "bf16": (B.BF16, torch.bfloat16)}
    dev = lambda x, t: torch.from_numpy(np.ascontiguousarray(x, t)).cuda()
    ti, tv = np.full((n, k + 1), 3, np.int32), np.full((n, k + 1), np.nan, np.float32)
    ti[:, :k], tv[:, :k] = ids, val
    dZ = Zd if in_place else torch.full((n, lddz), 9.0, dtype=dt[dz_dtype][1], device="cuda") if want_dz else None
    if base is not None:
        dZ[:, :C] = torch.from_numpy(base).to(dt[dz_dtype][1]).cuda()
    loss, row = torch.full((2,), 77.0, device="cuda"), torch.full((n + 1,), 77.0, device="cuda")
    wb = B.distill_workspace_bytes(n, C)
    ws = torch.full((wb,), 0xA5, dtype=torch.uint8, device="cuda")
    ti, tv, md = dev(ti, np.int32), dev(tv, np.float32), None if mask is None else dev(mask, np.uint8)
    B.distill(n, C, Zd, ld, dt[dtype][0], ti, tv, k + 1, k, rest, T, md, norm, weight, loss, row, dZ, dZ.stride(0) if dZ is not None else 0,
              dt[dz_dtype][0], int(base is not None), ws, wb, stream=stream())
    torch.cuda.synchronize()
    loss, row = loss.cpu().numpy(), row.cpu().numpy()
    assert loss[1] == 77.0 and row[n] == 77.0
    return float(loss[0]), row[:n], None if dZ is None else dZ.float().cpu().numpy()


def teacher_of(Z, k, rest, T, rng):
    """a teacher that sees the rows a little differently: its k best classes, as log-probabilities at T or as logits; with short lists, a class
    listed twice and entries of no mass"""
    n, C = Z.shape
    S = np.where(np.isfinite(Z) & (np.abs(Z) < 1e4), Z, -20.0) + 0.5 * rng.standard_normal(Z.shape)
    ids = np.argsort(-S, 1, kind="stable")[:, :k].astype(np.int32)
    val = np.take_along_axis(orc.row_softmax(S, T)[0] if rest else S, ids, 1)
    if k >= 3:
        ids[::4, 2] = ids[::4, 1]                    # (less mass on the two: it stays a distribution)
        val[::4, 1:3] -= 1.0
        val[1::4, 0] = -np.inf
        ids[2::4, 1] = -1
        ids[2::8, 2] = C
    ids[5::11] = -1                                  # rows without a teacher
    return ids, val.astype(np.float32)


def distill_tol(Z, ex, row, dref, T, C, k, weight, dz_dtype):
    se, q, p, r, P = sum_err(C), ex["q"], ex["p"], ex["r"], ex["P"]
    with np.errstate(divide="ignore", invalid="ignore"):
        lq, lp = np.abs(finite(np.where(q > 0, np.log(q), 0.0))), np.abs(finite(np.where(q > 0, ex["lp"], 0.0)))
        ln_s = np.log(C) + 1
        lnP = np.abs(finite(np.log(P)))
        inv = np.where(r > 0, finite(1.0 / P), 0.0)
    # a few roundings of every part; the sum's error once per unit of mass.  r is the teacher's log-probabilities' own rounding away from what
    # their exact values leave, in both computations alike (formed in doubles): no term
    row_tol = (q * (se + 8 * EPS * (1 + lq + lp + ln_s))).sum(1) + r * (2 * se + 8 * EPS * (1 + lnP + np.abs(finite(np.log(np.where(r > 0, r, 1)))))) + 4 * EPS * np.abs(finite(row))
    dz = p * (2 * se + 32 * EPS) + p * (r * inv)[:, None] * (4 * se + 16 * EPS) + q * (k + 8) * EPS
    dz = dz * abs(weight) / (ex["norm"] * T) * 2
    return row_tol, dz + np.abs(dref) * (2.0 ** -8 if dz_dtype == "bf16" else 4 * EPS) + 1e-38


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1.0, 2.25, 3.0])
@pytest.mark.parametrize("n,C,k", [(40, 200, 2), (30, 250, 1), (30, 2000, 4), (9, 5000, 8), (5, 40001, 8), (2, 131072, 20)])
def test_small_divergences_keep_their_digits(n, C, k, T):
    """A student close to its teacher, nearly all mass in what is not listed: the divergence is the small difference of terms that cancel.
    The sum of the others counts with P - r, a listed exponential with p, a listed q with q; nothing counts with r."""
    rng = np.random.default_rng(C + k)
    Z = to_dtype(0.1 * rng.standard_normal((n, C)), "f32")
    ids = np.stack([rng.permutation(C)[:k] for _ in range(n)]).astype(np.int32)
    at = lambda v: np.take_along_axis(v, ids.astype(np.int64), 1)
    val = (at(orc.row_softmax(Z, T)[0]) + 0.05 * rng.standard_normal((n, k))).astype(np.float32)
    _, ref, _, ex = orc.distill(Z, ids, val, True, T)
    u = 2.0 ** -24
    x = (Z.max(1, keepdims=True) - Z) / T
    p, q, lq, ln0 = at(ex["p"]), at(ex["q"]), -np.log(at(ex["q"])), np.log(C)
    # q: its rounding and its exponential (2 u) times ln(q/p) + 1, the logarithms of q and of the others (each 2 u, their sum u); a listed
    # exponential (x + 3) u, its sum, quotient and logarithm (k + 5) u; the logarithm of r 3 u of 1 - r; the others' sum: sum_err; another
    # temperature: u times the derivative by it; row_loss: u
    tol = (q * u * (2 * (1 + np.abs(np.log(q / p))) + 3 * (lq + ln0) + 3) + p * u * (at(x) + k + 8) + u * np.abs(q - p) * at(x)).sum(1)
    tol += np.abs(ex["P"] - ex["r"]) * (sum_err(C) + u * x.max(1)) + u * ref + 1e-14
    _, row, _ = run_distill(device(Z, "f32", C), C, "f32", "f32", T, None, ids, val, 1, 0.0, 1.0, C)
    check("row_loss", row, ref, tol)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,dz_dtype", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("n,C,pad,T", SIZES)
def test_distill_vs_oracle(n, C, pad, T, dtype, dz_dtype):
    rng = np.random.default_rng(5 * C + n)
    Z = hard_rows(n, C, dtype, 3 * C + n)
    for k, rest, use_mask, norm, weight in ((min(C, 4), 0, False, 0.0, 1.0), (min(C, 8), 1, True, 0.0, T * T), (min(C, 64), 1, False, 13.0, 0.5),
                                            (min(C, 200), 0, True, 0.0, -1.0), (1, 0, False, 0.0, 1.0)):
        mask = (rng.random(n) < 0.7).astype(np.uint8) if use_mask else None
        Zm = Z.copy()
        if mask is not None:
            Zm[mask == 0] = np.nan
        ids, val = teacher_of(Z, k, rest, T, rng)
        with np.errstate(divide="ignore", invalid="ignore"):
            ref_loss, ref_row, dref, ex = orc.distill(Z, ids, val, bool(rest), T, mask, norm, weight)
            row_tol, dz_tol = distill_tol(Z, ex, ref_row, dref, T, C, k, weight, dz_dtype)
        loss, row, dZ = run_distill(device(Zm, dtype, C + pad), C, dtype, dz_dtype, T, mask, ids, val, rest, norm, weight, C + 3)
        assert (dZ[:, C:] == 9.0).all()
        check("row_loss", row, ref_row, row_tol)
        check("dZ", dZ[:, :C], dref, dz_tol)
        if np.isfinite(ref_loss):
            check("loss", loss, ref_loss, abs(weight) / ex["norm"] * row_tol.sum() + 4 * EPS * abs(ref_loss))
        else:
            assert loss == ref_loss or (np.isnan(loss) and np.isnan(ref_loss))
        only = run_distill(device(Zm, dtype, C + pad), C, dtype, dz_dtype, T, mask, ids, val, rest, norm, weight, 0, want_dz=False)
        assert only[2] is None and np.array_equal(only[1], row) and (only[0] == loss or np.isnan(loss))
        base = to_dtype(rng.standard_normal((n, C)), dz_dtype)      # next to another loss's gradient: one more rounding, of the sum
        _, _, acc = run_distill(device(Zm, dtype, C + pad), C, dtype, dz_dtype, T, mask, ids, val, rest, norm, weight, C + 2, base=base)
        check("accumulated", acc[:, :C], base + dref, dz_tol + np.abs(base + dref) * (2.0 ** -8 if dz_dtype == "bf16" else 2 * EPS))
        if dtype == dz_dtype:
            Zd = device(Zm, dtype, C + pad, fill=5.0, offset=1)
            got = run_distill(Zd, C, dtype, dz_dtype, T, mask, ids, val, rest, norm, weight, 0, in_place=True)
            assert (got[2][:, C:] == 5.0).all()
            check("dZ in place", got[2][:, :C], dref, dz_tol)


@pytest.mark.gpu
@pytest.mark.parametrize("rest", [0, 1])
@pytest.mark.parametrize("n,C,k", [(67, 200, 127), (50, 256, 113), (131, 90, 63), (90, 129, 99), (200, 33, 31), (301, 20, 16), (140, 3, 16), (140, 3, 17),
                                   (70, 7, 150), (45, 200, 129), (40, 400, 256)])
def test_distill_lists_of_many_lengths(n, C, k, rest):
    """as many entries as a lane of few classes takes, one more, odd numbers of them, more than there are classes"""
    rng = np.random.default_rng(C + k)
    for dtype in ("f32", "bf16"):
        Z = hard_rows(n, C, dtype, C + k)
        ids, val = teacher_of(Z, min(C, k), rest, 1.0, rng)
        if k > C:                                    # behind the classes: nothing, and classes again with little mass
            more = rng.integers(-1, C, (n, k - C)).astype(np.int32)
            ids, val = np.concatenate([ids, more], 1), np.concatenate([val - 0.5, np.full((n, k - C), -9.0, np.float32)], 1).astype(np.float32)
        perm = rng.permutation(k)
        ids, val = ids[:, perm], val[:, perm]
        mask = (rng.random(n) < 0.8).astype(np.uint8)
        with np.errstate(divide="ignore", invalid="ignore"):
            ref_loss, ref_row, dref, ex = orc.distill(Z, ids, val, bool(rest), 1.0, mask)
            row_tol, dz_tol = distill_tol(Z, ex, ref_row, dref, 1.0, C, k, 1.0, dtype)
        loss, row, dZ = run_distill(device(Z, dtype, C + 1), C, dtype, dtype, 1.0, mask, ids, val, rest, 0.0, 1.0, C + 3)
        check("row_loss", row, ref_row, row_tol)
        check("dZ", dZ[:, :C], dref, dz_tol)


@pytest.mark.gpu
@pytest.mark.parametrize("C", [30, 700, 9000, 150_000])
def test_distill_student_sure_of_the_listed_classes(C):
    """P far below the rounding of a sum that holds the listed classes: it has to be formed without them"""
    n, k = 3, 4
    rng = np.random.default_rng(C)
    Z = to_dtype(rng.standard_normal((n, C)), "f32")
    Z[:, :k] += 30.0
    ids = np.tile(np.arange(k, dtype=np.int32), (n, 1))
    val = np.log(np.full((n, k), 0.9 / k)).astype(np.float32)
    ref_loss, ref_row, dref, ex = orc.distill(Z, ids, val, True)
    assert ex["P"].max() < 1e-7
    row_tol, dz_tol = distill_tol(Z, ex, ref_row, dref, 1.0, C, k, 1.0, "f32")
    loss, row, dZ = run_distill(device(Z, "f32", C), C, "f32", "f32", 1.0, None, ids, val, 1, 0.0, 1.0, C)
    check("row_loss", row, ref_row, row_tol)
    check("dZ", dZ, dref, dz_tol)


@pytest.mark.gpu
@pytest.mark.parametrize("rest", [0, 1])
@pytest.mark.parametrize("n,C", [(9, 40), (9, 600), (9, 9000), (9, 80_000), (700, 70_000)])
def test_distill_nan_stays_in_its_row(n, C, rest):
    """a NaN or an infinite logit, a NaN among the teacher's values: that row's numbers are NaN, the others' what they are without"""
    rng = np.random.default_rng(C)
    Z = to_dtype(rng.standard_normal((n, C)), "f32")
    ids, val = teacher_of(Z, 6, rest, 1.0, rng)
    clean = run_distill(device(Z, "f32", C), C, "f32", "f32", 1.0, None, ids, val, rest, 3.0, 1.0, C)
    Z[1, C // 2], Z[2, 0] = np.nan, np.inf
    val[6, 3] = np.nan
    loss, row, dZ = run_distill(device(Z, "f32", C), C, "f32", "f32", 1.0, None, ids, val, rest, 3.0, 1.0, C)
    broken = np.zeros(n, bool)
    broken[[1, 2, 6]] = True
    assert np.isnan(loss) and np.isnan(row[broken]).all() and np.isnan(dZ[broken]).all()
    assert np.array_equal(row[~broken], clean[1][~broken]) and np.array_equal(dZ[~broken], clean[2][~broken])


@pytest.mark.gpu
def test_distill_without_rows_leaves_a_loss_of_zero():
    import torch
    loss = torch.full((1,), 5.0, device="cuda")
    ws = torch.empty(B.distill_workspace_bytes(0, 4), dtype=torch.uint8, device="cuda")
    B.distill(0, 4, None, 4, B.F32, None, None, 2, 2, 0, 1.0, None, 0.0, 1.0, loss, None, None, 4, B.F32, 0, ws, ws.numel(), stream=stream())
    torch.cuda.synchronize()
    assert float(loss) == 0.0


# ----------------------------------------------------------------------------- together, as they are used
def chain_on_gpu(Zt, Zs, y, k, T, rest, mask, ws, out, st):
    """a teacher's top classes, a student's loss on labels and, next to it, on the teacher: one gradient"""
    n, C = Zs.shape
    B.logprobs(n, C, Zt, C, B.F32, T, None, None, 0, 0, None, 0, None, None, k, out["top"], out["top_logp"], k, ws["lp"], ws["lp"].numel(), stream=st)
    B.softmax_ce(n, C, Zs, C, y, mask, 0.0, out["ce"], out["dZ"], C, B.F32, ws["ce"], ws["ce"].numel(), stream=st)
    B.distill(n, C, Zs, C, B.F32, out["top"], out["top_logp"], k, k, rest, T, mask, 0.0, 0.5 * T * T, out["kd"], out["row"], out["dZ"], C, B.F32, 1,
              ws["kd"], ws["kd"].numel(), stream=st)
    B.logprobs(n, C, Zs, C, B.F32, 1.0, mask, y, 1, 1, out["logp"], 1, out["ent"], out["stats"], 0, None, None, 0, ws["lp"], ws["lp"].numel(), stream=st)
    B.logprobs_bwd(n, C, Zs, C, B.F32, 1.0, mask, out["stats"], out["ent"], y, 1, 1, out["g"], 1, out["h"], out["dZ2"], C, B.F32, stream=st)


def chain_buffers(n, C, k):
    import torch
    f = lambda *s: torch.full(s, 55.0, device="cuda")
    size = lambda b: torch.empty(max(b, 256), dtype=torch.uint8, device="cuda")
    out = dict(top=torch.empty(n, k, dtype=torch.int32, device="cuda"), top_logp=f(n, k), ce=f(1), kd=f(1), row=f(n), dZ=f(n, C), logp=f(n, 1), ent=f(n),
               stats=f(n, 2), g=torch.linspace(-1, 1, n, device="cuda").view(n, 1).contiguous(), h=torch.linspace(1, -2, n, device="cuda"), dZ2=f(n, C))
    ws = dict(lp=size(B.logprobs_workspace_bytes(n, C, k)), ce=size(B.loss_workspace_bytes(n)), kd=size(B.distill_workspace_bytes(n, C)))
    return out, ws


CHAIN = [(700, 47, 8), (130, 1500, 20), (6, 30_011, 64), (260, 12_000, 33)]


@pytest.mark.gpu
@pytest.mark.parametrize("rest", [0, 1])
@pytest.mark.parametrize("n,C,k", CHAIN)
def test_teacher_to_student_chain_vs_oracle(n, C, k, rest):
    import torch
    rng = np.random.default_rng(n)
    T = 2.0
    Zt = to_dtype(rng.standard_normal((n, C)) * 2, "f32")
    Zs = to_dtype(Zt * 0.7 + rng.standard_normal((n, C)), "f32")
    y, mask = rng.integers(0, C, n).astype(np.int32), (rng.random(n) < 0.6).astype(np.uint8)
    dev = lambda x, t: torch.from_numpy(np.ascontiguousarray(x, t)).cuda()
    out, ws = chain_buffers(n, C, k)
    chain_on_gpu(dev(Zt, np.float32), dev(Zs, np.float32), dev(y, np.int32), k, T, rest, dev(mask, np.uint8), ws, out, stream())
    torch.cuda.synchronize()
    t = orc.logprobs(Zt, np.zeros((n, 0)), k, T)
    np.testing.assert_array_equal(out["top"].cpu().numpy(), t["top_ids"])
    val = out["top_logp"].cpu().numpy()              # what the student is given
    ce, dce = orc.softmax_ce(Zs, y, mask)
    kd, row, dkd, ex = orc.distill(Zs, t["top_ids"], val, bool(rest), T, mask, 0.0, 0.5 * T * T)
    row_tol, dz_tol = distill_tol(Zs, ex, row, dkd, T, C, k, 0.5 * T * T, "f32")
    check("row", out["row"].cpu().numpy(), row, row_tol)
    # softmax_ce's own gradient: a probability with the sum's error, expf and three roundings, twice for the sum of the two
    p = np.exp(orc.row_softmax(Zs)[0])
    check("dZ", out["dZ"].cpu().numpy(), dce + dkd, dz_tol + mask[:, None] * (p * 2 * sum_err(C) + 8 * EPS * (np.arange(C) == y[:, None])) / max(mask.sum(), 1) +
          2 * EPS * np.abs(dce + dkd))
    g, h = out["g"].cpu().numpy().astype(np.float64), out["h"].cpu().numpy().astype(np.float64)
    ref = orc.logprobs(Zs, y[:, None], 0, 1.0, mask)
    dref = orc.logprobs_bwd(Zs, y[:, None], g, h, 1.0, mask)
    check("dZ2", out["dZ2"].cpu().numpy(), dref, bwd_tol(Zs, ref, dref, y[:, None], g, h, 1.0, C, "f32"))


@pytest.mark.gpu
@pytest.mark.parametrize("n,C,k", CHAIN)
def test_chain_recorded_and_replayed_gives_the_eager_bits(n, C, k):
    import torch
    rng = np.random.default_rng(C)
    st = torch.cuda.Stream()
    y, mask = rng.integers(0, C, n).astype(np.int32), (rng.random(n) < 0.6).astype(np.uint8)
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
    y, mask = dev(y), dev(mask)
    Zt, Zs = torch.empty(n, C, device="cuda"), torch.empty(n, C, device="cuda")
    out, ws = chain_buffers(n, C, k)
    eager, ews = chain_buffers(n, C, k)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        chain_on_gpu(Zt, Zs, y, k, 1.5, 1, mask, ws, out, torch.cuda.current_stream())
    for replay in range(4):
        Zt.copy_(dev((rng.standard_normal((n, C)) * 2).astype(np.float32)))
        Zs.copy_(dev(rng.standard_normal((n, C)).astype(np.float32)))
        chain_on_gpu(Zt, Zs, y, k, 1.5, 1, mask, ews, eager, torch.cuda.current_stream())
        torch.cuda.synchronize()
        for w in ws.values():
            w.fill_(replay * 37 + 1)                 # a workspace's contents do not matter
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for key in out:
            a, b = out[key].cpu().numpy(), eager[key].cpu().numpy()
            assert np.array_equal(a, b, equal_nan=True), (replay, key)


@pytest.mark.gpu
def test_two_streams_with_a_workspace_each():
    import torch
    n, C, k = 5, 60_001, 17
    rng = np.random.default_rng(1)
    sets = []
    for i in range(2):
        st = torch.cuda.Stream()
        Zt, Zs = (torch.from_numpy(rng.standard_normal((n, C)).astype(np.float32)).cuda() for _ in range(2))
        y = torch.from_numpy(rng.integers(0, C, n).astype(np.int32)).cuda()
        sets.append((Zt, Zs, y, st, *chain_buffers(n, C, k)))
    alone = []
    for Zt, Zs, y, st, out, ws in sets:
        o, w = chain_buffers(n, C, k)
        chain_on_gpu(Zt, Zs, y, k, 1.0, 1, None, w, o, torch.cuda.current_stream())
        alone.append(o)
    torch.cuda.synchronize()
    for _ in range(3):
        for Zt, Zs, y, st, out, ws in sets:
            chain_on_gpu(Zt, Zs, y, k, 1.0, 1, None, ws, out, st)
    torch.cuda.synchronize()
    for (_, _, _, _, out, _), o in zip(sets, alone):
        for key in out:
            assert torch.equal(out[key], o[key]), key


@pytest.mark.gpu
@pytest.mark.parametrize("C", [40, 3000, 20_000])
def test_rows_far_apart(C):
    """row offsets beyond 2^31 elements and 2^32 bytes"""
    import torch
    n, ld, k = 3, (1 << 30) + 40_007, 5
    rng = np.random.default_rng(C)
    Z = to_dtype(rng.standard_normal((n, C)) * 2, "bf16")
    big = torch.empty((n - 1) * ld + C, dtype=torch.bfloat16, device="cuda")
    rows = torch.as_strided(big, (n, C), (ld, 1))
    rows.copy_(torch.from_numpy(Z).to(torch.bfloat16).cuda())
    ids = np.tile(np.array([[0, C - 1]], np.int32), (n, 1))
    res = run_logprobs(rows, C, "bf16", 1.0, None, ids, k)
    ref = orc.logprobs(Z, ids, k)
    check_logprobs(res, ref, Z, C, 1.0)
    tids, val = teacher_of(Z, 4, 0, 1.0, rng)
    _, ref_row, dref, ex = orc.distill(Z, tids, val)
    row_tol, dz_tol = distill_tol(Z, ex, ref_row, dref, 1.0, C, 4, 1.0, "bf16")
    got = run_distill(rows, C, "bf16", "bf16", 1.0, None, tids, val, 0, 0.0, 1.0, 0, in_place=True)
    check("row_loss", got[1], ref_row, row_tol)
    check("dZ", got[2], dref, dz_tol)
    rows.copy_(torch.from_numpy(Z).to(torch.bfloat16).cuda())
    g, h = rng.standard_normal((n, 2)), rng.standard_normal(n)
    g, h = to_dtype(g, "f32"), to_dtype(h, "f32")
    dref = orc.logprobs_bwd(Z, ids, g, h)
    got = run_bwd(rows, C, "bf16", "bf16", 1.0, None, ref, ids, g, h, 0, in_place=True)
    check("dZ", got, dref, bwd_tol(Z, ref, dref, ids, g, h, 1.0, C, "bf16"))


@pytest.mark.gpu
@pytest.mark.parametrize("n,C", [(3, 11), (2, 700), (2, 9000)])
def test_gradients_are_the_difference_quotients_of_the_kernels_own_values(n, C):
    """a step of 2^-5 each way along random directions, values as double sums of the row losses / log-probabilities; a third derivative of at
    most ~1 times step^2 / 6, and the float values' rounding over the step, bound the difference"""
    import torch
    rng = np.random.default_rng(C)
    Z, D = rng.standard_normal((n, C)), rng.standard_normal((n, C))
    D /= np.abs(D).max()
    step = 2.0 ** -5
    ids, val = teacher_of(Z, 3, 1, 1.0, rng)
    given_ids, g, h = rng.integers(0, C, (n, 2)).astype(np.int32), rng.standard_normal((n, 2)), rng.standard_normal(n)

    def values(x):
        x = to_dtype(x, "f32")
        _, row, dz = run_distill(device(x, "f32", C), C, "f32", "f32", 1.0, None, ids, val, 1, 1.0, 1.0, C)
        r = run_logprobs(device(x, "f32", C), C, "f32", 1.0, None, given_ids, 0)
        return row.astype(np.float64).sum(), (g * r["logp"]).sum() + (h * r["entropy"]).sum(), dz[:, :C], r

    _, _, dz, r = values(Z)
    dlp = run_bwd(device(to_dtype(Z, "f32"), "f32", C), C, "f32", "f32", 1.0, None, r, given_ids, g, h, C)[:, :C]
    up, down = values(Z + step * D), values(Z - step * D)
    for i, grad in ((0, dz), (1, dlp)):
        quotient, slope = (up[i] - down[i]) / (2 * step), (grad.astype(np.float64) * D).sum()
        weight = n * (2.0 + (np.abs(g).sum() + 12 * np.abs(h).sum() if i else 0.0))
        assert abs(quotient - slope) <= weight * (step ** 2 + sum_err(C) * 20 / step), (quotient, slope)
