"""capgnn_rmsnorm, its gradient and capgnn_quantize_rows against float64, and what they refuse.

Tolerances, by counting roundings of EPS.  A lane adds at most 32 squares, its wave 6 levels of partial sums and a workgroup 16 waves: the
sum of squares (all positive) is off by at most 54 + 4 roundings of itself (the squares' and h's own among them), the mean by 2 more,
rstd by half of that and three of its own: under 40.  y is three products of it: 44.  An 8-bit row's scale is one division more, and a value is
off by half a step of the type (2^-4 of it, or half of the smallest step, 2^-10, near 0).  The gradient's mean of products is off by 58
roundings of the terms' magnitudes; dw sums n rows in some order."""
import numpy as np
import pytest

from paper_2508_13716_amd import binding as B
from tests.row_ops import CODE, EPS, FAKE, HALF, Mat, close, held, new, p, refuse, replayed, vec, ws_of

RSTD, Y = 40 * EPS, 44 * EPS


# ----------------------------------------------------------------------------- refusals
def fwd_args(**kw):
    a = dict(n=4, F=8, X=FAKE, ldx=8, R=2 * FAKE, ldr=8, H=3 * FAKE, ldh=8, dtype=B.F32, w=FAKE, eps=1e-6, Y=4 * FAKE, ldy=8, y_dtype=B.F32,
             y_scale=None, rstd=None)
    a.update(kw)
    return a


@pytest.mark.parametrize("bad", [
    dict(n=-1), dict(F=0), dict(dtype=2), dict(dtype=-1), dict(y_dtype=3), dict(X=None), dict(Y=None), dict(ldx=7), dict(ldr=7), dict(ldh=7), dict(ldy=7),
    dict(eps=-1e-9), dict(eps=float("nan")), dict(eps=float("inf")), dict(y_scale=FAKE), dict(y_dtype=B.E4M3), dict(X=FAKE + 2), dict(R=FAKE + 1, dtype=B.BF16),
    dict(w=FAKE + 2), dict(rstd=FAKE + 2), dict(H=FAKE, ldh=9), dict(H=2 * FAKE, ldh=9), dict(Y=3 * FAKE), dict(Y=FAKE, ldy=9), dict(Y=FAKE, y_dtype=B.BF16),
    dict(Y=FAKE, H=FAKE), dict(Y=2 * FAKE, y_dtype=B.BF16)])
def test_rmsnorm_refuses(bad):
    refuse(B.EINVAL, B.rmsnorm, **fwd_args(**bad))


def bwd_args(**kw):
    a = dict(n=4, F=8, dY=FAKE, lddy=8, dy_dtype=B.F32, H=2 * FAKE, ldh=8, dtype=B.F32, w=FAKE, rstd=FAKE, dH=3 * FAKE, lddh=8, dX=4 * FAKE, lddx=8,
             dw=FAKE, ws=FAKE, ws_bytes=1 << 30)
    a.update(kw)
    return a


@pytest.mark.parametrize("bad", [
    dict(n=-1), dict(F=0), dict(dtype=2), dict(dy_dtype=2), dict(dY=None), dict(H=None), dict(rstd=None), dict(dX=None), dict(lddy=7), dict(ldh=7), dict(lddh=7),
    dict(lddx=7), dict(dY=FAKE + 2), dict(dX=FAKE + 1, dtype=B.BF16), dict(dw=FAKE + 2), dict(dX=FAKE, lddx=9), dict(dX=FAKE, dtype=B.BF16), dict(dX=2 * FAKE, lddx=9),
    dict(dX=3 * FAKE, lddx=9), dict(n=4000, ws=FAKE + 16)])
def test_rmsnorm_bwd_refuses(bad):
    refuse(B.EINVAL, B.rmsnorm_bwd, **bwd_args(**bad))


@pytest.mark.parametrize("bad", [dict(n=-1), dict(F=0), dict(dtype=2), dict(X=None), dict(Q=None), dict(q_scale=None), dict(ldx=7), dict(ldq=7), dict(X=FAKE + 2),
                                 dict(q_scale=FAKE + 2), dict(Q=FAKE)])
def test_quantize_rows_refuses(bad):
    a = dict(n=4, F=8, X=FAKE, ldx=8, dtype=B.F32, Q=2 * FAKE, ldq=8, q_scale=FAKE)
    a.update(bad)
    refuse(B.EINVAL, B.quantize_rows, **a)


def test_too_wide_and_too_little_are_refused():
    wide = B.NORM_MAX + 1
    refuse(B.EUNSUPPORTED, B.rmsnorm, **fwd_args(F=wide, ldx=wide, ldr=wide, ldh=wide, ldy=wide))
    refuse(B.EUNSUPPORTED, B.rmsnorm_bwd, **bwd_args(F=wide, lddy=wide, ldh=wide, lddh=wide, lddx=wide))
    refuse(B.EUNSUPPORTED, B.quantize_rows, 1, wide, FAKE, wide, B.F32, 2 * FAKE, wide, FAKE)
    need = B.rmsnorm_bwd_workspace_bytes(4000, 8)
    refuse(B.ENOMEM, B.rmsnorm_bwd, **bwd_args(n=4000, ws_bytes=need - 1))
    refuse(B.ENOMEM, B.rmsnorm_bwd, **bwd_args(n=4000, ws=None))
    B.rmsnorm(**fwd_args(n=0, X=None, Y=None))
    B.quantize_rows(0, 8, None, 8, B.F32, None, 8, None)
    B.rmsnorm_bwd(**bwd_args(n=0, dY=None, H=None, dX=None, rstd=None, dw=None, ws=None, ws_bytes=0))


# ----------------------------------------------------------------------------- the GPU
WIDTHS = [1, 2, 3, 4, 5, 7, 8, 9, 12, 17, 41, 64, 100, 255, 256, 257, 513, 602, 1000, 1024, 2047, 2048, 2049, 4100, 8192, 8193, 16_385, 32_768]


def rows_for(F):
    return 67 if F <= 2048 else 5


def rms(h, eps):
    return 1.0 / np.sqrt((h * h).mean(1) + eps)


def check_q(q, s, y, what=""):
    """8-bit values q and their scales s against y"""
    want_s = np.maximum(np.abs(y).max(1), 2.0 ** -100) / 448.0
    close(s, want_s, want_s * (Y + 2 * EPS), what + " scale")
    z = y / want_s[:, None]
    close(q, z, np.maximum(np.abs(z) * HALF["e4m3"], 2.0 ** -10) + np.abs(z) * 100 * EPS + 2.0 ** -30, what + " values")


@pytest.mark.gpu
@pytest.mark.parametrize("F", WIDTHS)
@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("to", ["f32", "bf16", "e4m3"])
def test_norm(F, t, to):
    import torch
    rng = np.random.default_rng(F)
    n, eps = rows_for(F), 1e-5
    x, r = held(rng.standard_normal((n, F)) * np.exp(rng.standard_normal((n, 1))), t), held(rng.standard_normal((n, F)), t)
    w = held(1 + 0.3 * rng.standard_normal((1, F)), "f32")
    for residual, weight, pad in ((True, True, 0), (False, True, 3), (True, False, 5), (False, False, 8)):
        ld = F + pad
        X, R = Mat(x, t, ld, pad % 2), Mat(r, t, ld, pad % 3) if residual else None
        H, out, rstd = new(n, F, t, ld, pad % 2) if residual else None, new(n, F, to, ld, pad % 5), new(1, n, "f32")
        scale = new(1, n, "f32") if to == "e4m3" else None
        wd = vec(w) if weight else None
        B.rmsnorm(n, F, X.p, ld, p(R), ld, p(H), ld, CODE[t], p(wd), eps, out.p, ld, CODE[to], p(scale), rstd.p)
        torch.cuda.synchronize()
        h = x + r if residual else x
        s = rms(h, np.float64(np.float32(eps)))
        close(rstd.get()[0], s, s * RSTD, "rstd")
        y = h * s[:, None] * (w if weight else 1.0)
        if residual:
            close(H.get(), h, np.abs(h) * (EPS + HALF[t]) * 1.001, "H")
        if to == "e4m3":
            check_q(out.get(), scale.get()[0], y)
        else:
            close(out.get(), y, np.abs(y) * (Y + HALF[to]) * 1.001, "Y")
        X.get()


@pytest.mark.gpu
@pytest.mark.parametrize("F", [1, 3, 8, 41, 100, 602, 2049, 8193, 32_768])
@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_norm_in_place(F, t):
    """the residual stream updated where it lies, in each of the ways that are allowed"""
    import torch
    rng = np.random.default_rng(F + 1)
    n, ld = rows_for(F), F + 3
    x, r = held(rng.standard_normal((n, F)), t), held(rng.standard_normal((n, F)), t)
    h = x + r
    y = h * rms(h, 1e-5)[:, None]
    for way in ("H=X", "H=R", "H=X,Y=R", "H=R,Y=X", "Y=X", "Y=R"):
        X, R = Mat(x, t, ld, 1), Mat(r, t, ld, 1)
        H = X if "H=X" in way else R if "H=R" in way else None
        out = X if "Y=X" in way else R if "Y=R" in way else new(n, F, t, ld)
        B.rmsnorm(n, F, X.p, ld, R.p, ld, p(H), ld, CODE[t], None, 1e-5, out.p, ld, CODE[t])
        torch.cuda.synchronize()
        close(out.get(), y, np.abs(y) * (Y + HALF[t]) * 1.001, way)
        if H is not None:
            close(H.get(), h, np.abs(h) * (EPS + HALF[t]) * 1.001, way)


@pytest.mark.gpu
@pytest.mark.parametrize("F", WIDTHS)
@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_quantize_rows(F, t):
    import torch
    rng = np.random.default_rng(F + 2)
    n = rows_for(F)
    x = held(rng.standard_normal((n, F)) * np.exp(4 * rng.standard_normal((n, 1))), t)
    x[n // 2] = 0.0
    Q, s = new(n, F, "e4m3", F + 3, 1), new(1, n, "f32")
    B.quantize_rows(n, F, Mat(x, t, F + 1, 1).p, F + 1, CODE[t], Q.p, F + 3, s.p)
    torch.cuda.synchronize()
    check_q(Q.get(), s.get()[0], x)
    assert (Q.get()[n // 2] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("F", [6, 100, 5000])
def test_rows_of_zeros_infinities_and_nan(F):
    import torch
    x = np.ones((6, F))
    x[1] = 0.0
    x[2, F - 1] = np.nan
    x[3, 0] = np.inf
    x[4] = 1e-30
    for t in ("f32", "bf16"):
        out, q, s, rstd = new(6, F, "f32"), new(6, F, "e4m3"), new(1, 6, "f32"), new(1, 6, "f32")
        X = Mat(x, t)
        B.rmsnorm(6, F, X.p, F, None, 0, None, 0, CODE[t], None, 1e-6, out.p, F, B.F32, None, rstd.p)
        B.rmsnorm(6, F, X.p, F, None, 0, None, 0, CODE[t], None, 1e-6, q.p, F, B.E4M3, s.p)
        torch.cuda.synchronize()
        y, z, scale = out.get(), q.get(), s.get()[0]
        for k in (0, 5):
            assert np.abs(y[k] - 1).max() < 1e-5 and (z[k] == 448).all()
        assert (y[1] == 0).all() and (z[1] == 0).all() and scale[1] == np.float32(2.0 ** -100) / np.float32(448)
        assert np.isnan(y[2]).all() and np.isnan(z[2]).all() and np.isnan(scale[2])
        assert np.isnan(y[3, 0]) and (y[3, 1:] == 0).all() and rstd.get()[0, 3] == 0
        close(y[4], held(np.array([1e-30]), t) * 1e3 * np.ones(F), 1e-27 * 1e-4 * np.ones(F))
        assert (z[4] == 448).all()                  # (above 2^-100)
        B.rmsnorm(1, F, Mat(np.zeros((1, F)), t).p, F, None, 0, None, 0, CODE[t], None, 0.0, out.p, F, B.F32)
        torch.cuda.synchronize()
        assert np.isnan(out.get()[0]).all()         # eps = 0: 0 * infinity


def grad_ref(dy, h, w, rstd, dh):
    F = h.shape[1]
    hat, g = h * rstd[:, None], dy * w
    mean = (g * hat).mean(1)[:, None]
    dx = rstd[:, None] * (g - hat * mean) + dh
    err = rstd[:, None] * (3 * EPS * np.abs(g) + np.abs(hat) * 60 * EPS * np.abs(g * hat).mean(1)[:, None] + 5 * EPS * np.abs(hat * mean)) + 3 * EPS * (np.abs(dx) + np.abs(dh))
    return dx, err, (dy * hat).sum(0), np.abs(dy * hat).sum(0) * (len(h) + 24) * EPS


@pytest.mark.gpu
@pytest.mark.parametrize("F", WIDTHS)
@pytest.mark.parametrize("t,dt", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
def test_gradient(F, t, dt):
    import torch
    rng = np.random.default_rng(F + 3)
    n = rows_for(F)
    h, dy, dh = held(rng.standard_normal((n, F)), t), held(rng.standard_normal((n, F)), dt), held(rng.standard_normal((n, F)), t)
    w = held(1 + 0.3 * rng.standard_normal((1, F)), "f32")
    rstd = held(rms(h, 1e-6), "f32")
    for residual, weight, pad in ((True, True, 0), (False, False, 3), (True, True, 5)):
        ld = F + pad
        dx, err, dw, dw_err = grad_ref(dy, h, w if weight else 1.0, rstd, dh if residual else 0.0 * dh)
        H, dY, dH = Mat(h, t, ld, pad % 2), Mat(dy, dt, ld, pad % 3), Mat(dh, t, ld, pad % 2) if residual else None
        dX, dW, r = new(n, F, t, ld, 1), new(1, F, "f32") if weight else None, vec(rstd)
        ws, size = ws_of(B.rmsnorm_bwd_workspace_bytes(n, F) if weight else 0)
        wd = vec(w) if weight else None
        B.rmsnorm_bwd(n, F, dY.p, ld, CODE[dt], H.p, ld, CODE[t], p(wd), r.p, p(dH), ld, dX.p, ld, p(dW), ws if weight else None, size)
        torch.cuda.synchronize()
        close(dX.get(), dx, (err + np.abs(dx) * HALF[t]) * 1.001, "dX")
        if weight:
            close(dW.get()[0], dw, dw_err * 1.001 + 1e-30, "dw")
        # in place of each input
        ways = [("dH", dH)] if residual else []
        ways += [("H", H)] + ([("dY", dY)] if t == dt else [])
        for name, _ in ways:
            m = {"H": Mat(h, t, ld, 1), "dY": Mat(dy, dt, ld, 1), "dH": Mat(dh, t, ld, 1) if residual else None}
            B.rmsnorm_bwd(n, F, m["dY"].p, ld, CODE[dt], m["H"].p, ld, CODE[t], p(wd), r.p, p(m["dH"]), ld, m[name].p, ld, p(dW), ws if weight else None, size)
            torch.cuda.synchronize()
            close(m[name].get(), dx, (err + np.abs(dx) * HALF[t]) * 1.001, "dX is " + name)
            if weight:
                close(dW.get()[0], dw, dw_err * 1.001 + 1e-30, "dw, dX is " + name)


@pytest.mark.gpu
@pytest.mark.parametrize("F", [5, 37, 300])
def test_gradient_is_that_of_differences(F):
    import torch
    rng = np.random.default_rng(F + 4)
    n, eps, step = 6, 1e-5, 1e-5
    h, w, up = rng.standard_normal((n, F)), 1 + 0.3 * rng.standard_normal((1, F)), rng.standard_normal((n, F))
    h, w, up = held(h, "f32"), held(w, "f32"), held(up, "f32")
    loss = lambda h, w: float((h * rms(h, eps)[:, None] * w * up).sum())
    dX, dw, ws = new(n, F, "f32"), new(1, F, "f32"), ws_of(B.rmsnorm_bwd_workspace_bytes(n, F))
    B.rmsnorm_bwd(n, F, Mat(up, "f32").p, F, B.F32, Mat(h, "f32").p, F, B.F32, vec(w).p, vec(held(rms(h, eps), "f32")).p, None, 0, dX.p, F, dw.p, *ws)
    torch.cuda.synchronize()
    for _ in range(8):
        d, e = rng.standard_normal((n, F)), rng.standard_normal((1, F))
        want = (loss(h + step * d, w + step * e) - loss(h - step * d, w - step * e)) / (2 * step)
        got = float((dX.get() * d).sum() + (dw.get() * e).sum())
        size = float(np.abs(dX.get() * d).sum() + np.abs(dw.get() * e).sum())
        assert abs(got - want) <= size * 1e-5       # (differences: step^2 times the third derivative, and 1e-16 / step)


@pytest.mark.gpu
@pytest.mark.parametrize("n,F,t", [(200_001, 1, "f32"), (70_000, 8, "bf16"), (30_000, 41, "f32"), (5000, 602, "bf16"), (3000, 1024, "f32")])
def test_many_rows(n, F, t):
    import torch
    rng = np.random.default_rng(n)
    x, dy = held(rng.standard_normal((n, F)), t), held(rng.standard_normal((n, F)), t)
    X, dY, out, rstd = Mat(x, t), Mat(dy, t), new(n, F, t), new(1, n, "f32")
    B.rmsnorm(n, F, X.p, F, None, 0, None, 0, CODE[t], None, 1e-6, out.p, F, CODE[t], None, rstd.p)
    dX, dw, ws = new(n, F, t), new(1, F, "f32"), ws_of(B.rmsnorm_bwd_workspace_bytes(n, F))
    B.rmsnorm_bwd(n, F, dY.p, F, CODE[t], X.p, F, CODE[t], None, rstd.p, None, 0, dX.p, F, dw.p, *ws)
    torch.cuda.synchronize()
    s = rms(x, np.float64(np.float32(1e-6)))
    y = x * s[:, None]
    close(out.get(), y, np.abs(y) * (Y + HALF[t]) * 1.001)
    dx, err, want, want_err = grad_ref(dy, x, 1.0, rstd.get()[0], 0.0 * x)
    close(dX.get(), dx, (err + np.abs(dx) * HALF[t]) * 1.001 + 1e-30)
    # a thread's chain is n / 1024 rows, at least 256 wide after that: far fewer roundings than n
    close(dw.get()[0], want, want_err)


@pytest.mark.gpu
def test_recorded_and_replayed():
    rng = np.random.default_rng(9)
    n, F = 300, 602
    X, R, H, Q, s, rstd = Mat(rng.standard_normal((n, F)), "bf16"), Mat(rng.standard_normal((n, F)), "bf16"), new(n, F, "bf16"), new(n, F, "e4m3"), new(1, n, "f32"), new(1, n, "f32")
    dX, dw, (ws, size), w = new(n, F, "bf16"), new(1, F, "f32"), ws_of(B.rmsnorm_bwd_workspace_bytes(n, F)), vec(rng.standard_normal(F))

    def run(st):
        B.rmsnorm(n, F, X.p, F, R.p, F, H.p, F, B.BF16, w.p, 1e-6, Q.p, F, B.E4M3, s.p, rstd.p, stream=st)
        B.rmsnorm_bwd(n, F, R.p, F, B.BF16, H.p, F, B.BF16, w.p, rstd.p, X.p, F, dX.p, F, dw.p, ws, size, stream=st)
    replayed(run, lambda: [H.raw(), Q.raw(), s.raw(), rstd.raw(), dX.raw(), dw.raw()])


@pytest.mark.gpu
def test_rows_beyond_32_bit_offsets():
    import torch
    n, F = 4_200_000, 1024                           # 2^32 elements and more
    X = torch.zeros((n, F), dtype=torch.bfloat16, device="cuda")
    X[-1] = 3.0
    X[0] = 2.0
    H = torch.empty_like(X)
    out = torch.empty_like(X)
    B.rmsnorm(n, F, X, F, X, F, H, F, B.BF16, None, 1e-6, out, F, B.BF16)
    torch.cuda.synchronize()
    assert float(H[-1, -1]) == 6.0 and float(H[0, 0]) == 4.0 and float(out[-1, 0]) == 1.0 and float(out[0, -1]) == 1.0
    assert int(torch.count_nonzero(out[:, 5])) == 2


@pytest.mark.gpu
def test_the_gradient_of_no_rows_is_zero():
    import torch
    for F in (1, 41, 602):
        dw = Mat(np.full((1, F), 7.0), "f32")
        B.rmsnorm_bwd(0, F, None, F, B.F32, None, F, B.F32, None, None, None, 0, None, F, dw.p, None, 0)
        torch.cuda.synchronize()
        assert (dw.get() == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("F", [5, 6, 9, 41, 100, 602, 2049, 8193, 32_767])
@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("way", ["X", "R", "sum"])
def test_an_infinity_among_elements_that_two_vectors_share(F, t, way):
    """a row's last vector ends where the row does and repeats elements of the one before: an infinity at each of its places"""
    import torch
    places = list(range(max(F - 8, 0), F)) + [0]
    n = len(places)
    rows, sign = np.arange(n), np.where(np.arange(n) % 2, -1.0, 1.0)
    x, r = np.ones((n, F)), np.zeros((n, F))
    if way == "sum":                                 # (two numbers whose sum is none)
        x[rows, places] = r[rows, places] = sign * 3e38
    else:
        (x if way == "X" else r)[rows, places] = sign * np.inf
    X, R, H, out, rstd = Mat(x, t), Mat(r, t), new(n, F, t), new(n, F, "f32"), new(1, n, "f32")
    q, s = new(n, F, "e4m3"), new(1, n, "f32")
    B.rmsnorm(n, F, X.p, F, R.p, F, H.p, F, CODE[t], None, 1e-6, out.p, F, B.F32, None, rstd.p)
    B.rmsnorm(n, F, X.p, F, R.p, F, None, 0, CODE[t], None, 1e-6, q.p, F, B.E4M3, s.p)
    torch.cuda.synchronize()
    there = np.zeros((n, F), bool)
    there[rows, places] = True
    y = out.get()
    assert (rstd.get()[0] == 0).all()
    assert np.isnan(y[there]).all() and (y[~there] == 0).all()          # infinity * 0, and 1 * 0
    assert np.array_equal(H.get()[there], sign[np.nonzero(there)[0]] * np.inf) and (H.get()[~there] == 1).all()
    assert np.isnan(s.get()).all() and np.isnan(q.get()).all()
