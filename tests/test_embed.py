"""capgnn_embed and capgnn_embed_bwd against float64, and what they refuse.

Tolerances: a looked-up value is one float product (EPS of it) rounded to the output's type.  A row of the gradient sums m terms in
float: at most m roundings, each EPS of a partial sum, which the terms' magnitudes bound; then the product with the scale and, where it
accumulates, one more sum."""
import numpy as np
import pytest

from paper_2508_13716_amd import binding as B
from tests.row_ops import CODE, EPS, FAKE, HALF, Mat, close, held, new, refuse, replayed, ws_of


# ----------------------------------------------------------------------------- refusals (arguments are checked first: no GPU)
def fwd_args(**kw):
    a = dict(n=4, ids=FAKE, V=10, F=8, table=FAKE, ldt=8, dtype=B.F32, scale=1.0, out=2 * FAKE, ldo=8, out_dtype=B.F32)
    a.update(kw)
    return a


@pytest.mark.parametrize("bad", [dict(n=-1), dict(V=0), dict(V=-1), dict(V=1 << 31), dict(F=0), dict(ids=None), dict(table=None), dict(out=None), dict(ldt=7),
                                 dict(ldo=7), dict(dtype=2), dict(out_dtype=2), dict(dtype=-1), dict(table=FAKE + 2), dict(out=FAKE + 1, out_dtype=B.BF16),
                                 dict(ids=FAKE + 4), dict(out=FAKE)])
def test_embed_refuses(bad):
    refuse(B.EINVAL, B.embed, **fwd_args(**bad))


def bwd_args(**kw):
    a = dict(n=4, ids=FAKE, V=10, F=8, dY=FAKE, lddy=8, dy_dtype=B.F32, scale=1.0, dtable=2 * FAKE, lddt=8, accumulate=0, ws=FAKE, ws_bytes=1 << 30)
    a.update(kw)
    return a


@pytest.mark.parametrize("bad", [dict(n=-1), dict(n=1 << 31), dict(V=0), dict(V=1 << 31), dict(F=0), dict(ids=None), dict(dY=None), dict(dtable=None),
                                 dict(lddy=7), dict(lddt=7), dict(dy_dtype=2), dict(dY=FAKE + 2), dict(dtable=FAKE + 2), dict(ids=FAKE + 4),
                                 dict(dtable=FAKE), dict(ws=FAKE + 16)])
def test_embed_bwd_refuses(bad):
    refuse(B.EINVAL, B.embed_bwd, **bwd_args(**bad))


def test_too_little_workspace_and_too_wide_rows_are_refused():
    for n, V in ((4, 10), (100_000, 1 << 20)):
        need = B.embed_bwd_workspace_bytes(n, V, 8)
        assert need > 0
        refuse(B.ENOMEM, B.embed_bwd, **bwd_args(n=n, V=V, ws_bytes=need - 1))
        refuse(B.ENOMEM, B.embed_bwd, **bwd_args(n=n, V=V, ws=None))
    wide = (1 << 22) + 1
    refuse(B.EUNSUPPORTED, B.embed, **fwd_args(F=wide, ldt=wide, ldo=wide))
    refuse(B.EUNSUPPORTED, B.embed_bwd, **bwd_args(F=wide, lddy=wide, lddt=wide))
    assert B.embed_bwd_workspace_bytes(0, 10, 8) == 0 and B.embed_bwd_workspace_bytes(4, 10, wide) == 0


def test_no_rows_is_no_work():
    B.embed(**fwd_args(n=0, ids=None, table=None, out=None))
    B.embed_bwd(**bwd_args(n=0, ids=None, dY=None, accumulate=1, ws=None, ws_bytes=0))


# ----------------------------------------------------------------------------- the GPU
def some_ids(n, V, rng, kind):
    if kind == "uniform":
        return rng.integers(0, V, n)
    if kind == "power":
        return np.minimum(np.exp(rng.random(n) * np.log(V + 1)).astype(np.int64) - 1, V - 1) * 7 % V
    if kind == "one":
        return np.full(n, V // 2)
    ids = rng.integers(0, V, n)                     # "outside": a third of them name no row
    ids[rng.random(n) < 0.33] = -1
    ids[rng.random(n) < 0.1] = V
    ids[:: 17] = 1 << 40
    ids[5:: 19] = -(1 << 62)
    return ids


def dev(ids):
    import torch
    return torch.from_numpy(np.asarray(ids, np.int64)).cuda()


@pytest.mark.gpu
@pytest.mark.parametrize("n,V,F", [(1, 1, 1), (3, 5, 3), (70, 40, 7), (64, 1000, 1024), (500, 47, 100), (37, 11, 41), (33, 9, 602), (2, 3, 2051)])
@pytest.mark.parametrize("t,to", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("pad,kind", [(0, "uniform"), (5, "outside")])
def test_lookup(n, V, F, t, to, pad, kind):
    import torch
    rng = np.random.default_rng(n * F)
    x = held(rng.standard_normal((V, F)) * 3, t)
    ids = some_ids(n, V, rng, kind)
    table, out = Mat(x, t, F + pad, offset=pad % 2), new(n, F, to, F + pad, offset=pad % 3)
    scale = np.float32(1.7)
    B.embed(n, dev(ids), V, F, table.p, F + pad, CODE[t], float(scale), out.p, F + pad, CODE[to])
    torch.cuda.synchronize()
    ok = (ids >= 0) & (ids < V)
    want = np.where(ok[:, None], x[np.where(ok, ids, 0)] * np.float64(scale), 0.0)
    close(out.get(), want, np.abs(want) * (EPS + HALF[to]) * 1.001)
    if t == to:                                     # a scale of one copies
        B.embed(n, dev(ids), V, F, table.p, F + pad, CODE[t], 1.0, out.p, F + pad, CODE[to])
        torch.cuda.synchronize()
        assert np.array_equal(out.get(), np.where(ok[:, None], x[np.where(ok, ids, 0)], 0.0))


def check_gradient(n, V, F, t, pad, kind, accumulate, scale=0.75, seed=0):
    import torch
    rng = np.random.default_rng(n + 31 * F + seed)
    x = held(rng.standard_normal((n, F)), t)
    ids = some_ids(n, V, rng, kind)
    before = held(rng.standard_normal((V, F)), "f32") if accumulate else None
    dY, dtable = Mat(x, t, F + pad, offset=pad % 2), Mat(before, "f32", F + pad, pad % 3, (V, F))
    if not accumulate:
        dtable.view[:, :F] = 9.0
    ws, size = ws_of(B.embed_bwd_workspace_bytes(n, V, F))
    d_ids = dev(ids)
    B.embed_bwd(n, d_ids, V, F, dY.p, F + pad, CODE[t], scale, dtable.p, F + pad, int(accumulate), ws, size)
    torch.cuda.synchronize()
    ok = (ids >= 0) & (ids < V)
    total, mass, count = np.zeros((V, F)), np.zeros((V, F)), np.zeros(V)
    np.add.at(total, ids[ok], x[ok])
    np.add.at(mass, ids[ok], np.abs(x[ok]))
    np.add.at(count, ids[ok], 1)
    want = scale * total + (before if accumulate else 0.0)
    tol = scale * mass * (count[:, None] + 2) * EPS + np.abs(want) * 2 * EPS
    got = dtable.get()
    close(got, want, tol * 1.001, "dtable")
    untouched = count == 0
    assert np.array_equal(got[untouched], before[untouched] if accumulate else np.zeros((int(untouched.sum()), F)))
    if not accumulate:                              # the same every time
        first = dtable.raw()
        B.embed_bwd(n, d_ids, V, F, dY.p, F + pad, CODE[t], scale, dtable.p, F + pad, 0, ws, size)
        torch.cuda.synchronize()
        assert torch.equal(first, dtable.raw())


@pytest.mark.gpu
@pytest.mark.parametrize("n,V,F,kind", [
    (1, 1, 1, "one"), (1, 50, 9, "uniform"), (7, 3, 3, "uniform"), (100, 60, 7, "outside"), (513, 47, 100, "power"), (8192, 1000, 20, "power"),
    (8193, 1000, 20, "power"), (9000, 2047, 5, "uniform"), (9000, 2048, 5, "uniform"), (20_001, 70_000, 33, "power"), (10_000, 5_000_000, 1, "outside"),
    (60_000, 41, 16, "power"), (3000, 1 << 20, 12, "uniform"), (300, 20, 1029, "power"), (5000, 30, 602, "power")])
@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("accumulate,pad", [(False, 0), (True, 3)])
def test_gradient(n, V, F, kind, t, accumulate, pad):
    check_gradient(n, V, F, t, pad, kind, accumulate)


@pytest.mark.gpu
@pytest.mark.parametrize("n,F,t", [(70_000, 4, "f32"), (33_000, 64, "bf16"), (9000, 300, "f32"), (257, 8, "bf16")])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("V", [5, 5000])
def test_every_row_names_the_same_one(n, F, t, accumulate, V):
    check_gradient(n, V, F, t, 1, "one", accumulate)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [100, 20_000])
@pytest.mark.parametrize("V", [1, 2, 31, 36, 40, 41, 71, 72, 73, 120, 305])
@pytest.mark.parametrize("F,t", [(1, "f32"), (3, "f32"), (9, "bf16"), (64, "f32"), (256, "bf16"), (258, "f32"), (520, "bf16")])
def test_tables_of_a_few_rows(n, V, F, t):
    check_gradient(n, V, F, t, 2, "outside", V % 2 == 0)


@pytest.mark.gpu
@pytest.mark.parametrize("n,V,F,t", [(2000, 3, 20_001, "f32"), (2000, 70, 20_001, "bf16"), (400, 2, 100_000, "f32")])
def test_tables_of_a_few_wide_rows(n, V, F, t):
    check_gradient(n, V, F, t, 1, "outside", V == 3)


@pytest.mark.gpu
@pytest.mark.parametrize("n,V,F,t", [(8192, 20, 64, "f32"), (8192, 21, 64, "f32"), (8193, 39, 64, "f32"), (8193, 40, 64, "f32"), (9000, 156, 1, "f32"), (9000, 157, 1, "f32"),
                                     (50, 80, 1, "f32"), (50, 81, 1, "f32"), (32_768, 3, 520, "bf16"), (32_769, 3, 520, "bf16"), (9000, 18, 250, "bf16"), (9000, 20, 250, "bf16")])
def test_tables_at_the_borders_of_a_workgroups_memory(n, V, F, t):
    check_gradient(n, V, F, t, 1, "outside", False)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 127, 128, 129, 130, 1025])
@pytest.mark.parametrize("V", [200, 3_000_000])
def test_a_few_ids(n, V):
    check_gradient(n, V, 9, "f32", 1, "outside", V > 200)
    check_gradient(n, V, 9, "bf16", 0, "one", True)


@pytest.mark.gpu
@pytest.mark.parametrize("n,V,F", [(120_000, 1660, 2), (60_000, 1000, 8), (200_000, 900, 1), (150_000, 400, 40), (40_000, 300, 200)])
@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_runs_of_every_length(n, V, F, t):
    """narrow rows drawn by a power law: runs inside a tile, over a few, over what a wave adds, over more"""
    check_gradient(n, V, F, t, 1, "power", F == 8)


@pytest.mark.gpu
def test_an_infinite_scale_leaves_rows_of_zeros():
    import torch
    x = Mat(np.full((4, 40), 0.5), "f32")
    out = new(3, 40, "f32")
    B.embed(3, dev(np.array([-1, 2, 4])), 4, 40, x.p, 40, B.F32, float("inf"), out.p, 40, B.F32)
    torch.cuda.synchronize()
    assert (out.get() == np.array([[0.0], [np.inf], [0.0]])).all()


@pytest.mark.gpu
@pytest.mark.parametrize("V", [7, 900])
@pytest.mark.parametrize("n", [60, 9000])
def test_rows_that_no_id_names_keep_their_bits(V, n):
    """what is added to: signs of zero and NaN among it"""
    import torch
    bits = torch.tensor([0x80000000, 0, 0x7FC12345, 0x3F800000, 0xFF800000], dtype=torch.int64).to(torch.int32).repeat(V * 4)[: V * 4]
    dtable = bits.cuda().view(torch.float32)
    ids = dev(np.full(n, 2))
    dY = Mat(np.full((n, 4), 0.25), "f32")
    ws, size = ws_of(B.embed_bwd_workspace_bytes(n, V, 4))
    B.embed_bwd(n, ids, V, 4, dY.p, 4, B.F32, -1.0, dtable, 4, 1, ws, size)
    torch.cuda.synchronize()
    now = dtable.view(torch.int32).cpu()
    assert torch.equal(now[:8], bits[:8]) and torch.equal(now[12:], bits[12:])


@pytest.mark.gpu
@pytest.mark.parametrize("n", [40, 9000])
def test_no_id_names_a_row(n):
    import torch
    ids = dev(np.full(n, -7))
    dY = Mat(np.full((n, 12), np.nan), "f32")
    for accumulate, left in ((0, 0.0), (1, 3.0)):
        dtable = Mat(np.full((6, 12), 3.0), "f32", 13)
        ws, size = ws_of(B.embed_bwd_workspace_bytes(n, 6, 12))
        B.embed_bwd(n, ids, 6, 12, dY.p, 12, B.F32, 1.0, dtable.p, 13, accumulate, ws, size)
        torch.cuda.synchronize()
        assert (dtable.get() == left).all()


@pytest.mark.gpu
def test_no_ids_zero_the_table():
    import torch
    for V, F, ld in ((7, 3, 3), (50, 602, 602), (13, 1, 4), (9, 2, 5), (31, 130, 131)):
        dtable = Mat(np.full((V, F), 3.0), "f32", ld)
        B.embed_bwd(0, None, V, F, None, 0, B.F32, 1.0, dtable.p, ld, 0, None, 0)
        torch.cuda.synchronize()
        assert (dtable.get() == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("V", [50, 500])
def test_a_row_that_is_nan_stays_with_its_id(V):
    import torch
    x = np.ones((9000, 6))
    x[4000] = np.nan
    x[100, 2] = np.inf
    ids = np.arange(9000) % 50
    dtable = new(V, 6, "f32")
    ws, size = ws_of(B.embed_bwd_workspace_bytes(9000, V, 6))
    B.embed_bwd(9000, dev(ids), V, 6, Mat(x, "bf16").p, 6, B.BF16, 1.0, dtable.p, 6, 0, ws, size)
    torch.cuda.synchronize()
    assert (dtable.get()[50:] == 0).all()
    got = dtable.get()[:50]
    want = np.full((50, 6), 180.0)
    want[0] = np.nan
    assert np.isnan(got[0]).all() and (got[1:] == 180.0).all()


@pytest.mark.gpu
def test_rows_beyond_32_bit_offsets():
    """a table of more than 2^32 bytes, and elements"""
    import torch
    V, F = 9_000_001, 512
    table = torch.zeros((V, F), dtype=torch.bfloat16, device="cuda")
    rows = [0, 4_194_303, 4_194_304, 8_388_608, V - 1]
    for k, r in enumerate(rows):
        table[r] = k + 1
    out = new(5, F, "bf16")
    ids = dev(rows)
    B.embed(5, ids, V, F, table, F, B.BF16, 1.0, out.p, F, B.BF16)
    torch.cuda.synchronize()
    assert np.array_equal(out.get()[:, 0], np.arange(1.0, 6.0)) and (out.get() == out.get()[:, :1]).all()
    del table
    V = 4_500_001
    dtable = torch.full((V, F), 5.0, device="cuda")
    rows = [0, 4_194_303, 4_194_304, 4_300_000, V - 1]
    ids = dev(rows)
    ws, size = ws_of(B.embed_bwd_workspace_bytes(5, V, F))
    B.embed_bwd(5, ids, V, F, out.p, F, B.BF16, 1.0, dtable, F, 1, ws, size)
    torch.cuda.synchronize()
    assert [float(dtable[r, F - 1]) for r in rows] == [6.0, 7.0, 8.0, 9.0, 10.0]
    B.embed_bwd(5, ids, V, F, out.p, F, B.BF16, 1.0, dtable, F, 0, ws, size)
    torch.cuda.synchronize()
    assert [float(dtable[r, F - 1]) for r in rows] == [1.0, 2.0, 3.0, 4.0, 5.0]
    assert int(torch.count_nonzero(dtable[:, 0])) == 5 and int(torch.count_nonzero(dtable[:, F - 1])) == 5


@pytest.mark.gpu
@pytest.mark.parametrize("n,V", [(300, 90), (30_000, 5000)])
def test_recorded_and_replayed(n, V):
    rng = np.random.default_rng(5)
    ids = dev(some_ids(n, V, rng, "power"))
    table, out = Mat(rng.standard_normal((V, 40)), "f32"), new(n, 40, "f32")
    dtable = new(V, 40, "f32")
    ws, size = ws_of(B.embed_bwd_workspace_bytes(n, V, 40))

    def run(st):
        B.embed(n, ids, V, 40, table.p, 40, B.F32, 2.0, out.p, 40, B.F32, stream=st)
        B.embed_bwd(n, ids, V, 40, out.p, 40, B.F32, 2.0, dtable.p, 40, 0, ws, size, stream=st)
    replayed(run, lambda: [out.raw(), dtable.raw()])


@pytest.mark.gpu
def test_two_streams_with_a_workspace_each():
    import torch
    rng = np.random.default_rng(6)
    n, V, F = 50_000, 300, 64
    jobs = []
    for k in range(2):
        x, ids = held(rng.standard_normal((n, F)), "f32"), rng.integers(0, V, n)
        ws, size = ws_of(B.embed_bwd_workspace_bytes(n, V, F))
        jobs.append((x, ids, Mat(x, "f32"), dev(ids), new(V, F, "f32"), ws, size, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        for x, ids, dY, d_ids, dtable, ws, size, st in jobs:
            B.embed_bwd(n, d_ids, V, F, dY.p, F, B.F32, 1.0, dtable.p, F, 0, ws, size, stream=st)
    torch.cuda.synchronize()
    for x, ids, dY, d_ids, dtable, ws, size, st in jobs:
        want, mass = np.zeros((V, F)), np.zeros((V, F))
        np.add.at(want, ids, x)
        np.add.at(mass, ids, np.abs(x))
        close(dtable.get(), want, mass * (np.bincount(ids, minlength=V)[:, None] + 2) * EPS + np.abs(want) * 2 * EPS)


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("n,V", [(60, 7), (60, 900), (9000, 7), (9000, 900), (300_000, 7)])
@pytest.mark.parametrize("F,t", [(3, "f32"), (40, "f32"), (41, "bf16")])
@pytest.mark.parametrize("accumulate", [0, 1])
def test_a_scale_that_is_not_finite_leaves_the_gradient_of_rows_that_no_id_names(scale, n, V, F, t, accumulate):
    """tables in LDS and sorted ids alike: such rows are zeros, or what they were; a sum of zeros, -0 among them, is 0 * scale"""
    import torch
    ids = np.arange(n) % 5                           # 0: a sum above 0, 1: one of -0, 2: one that cancels, 3 and 4: no row
    ids = np.where(ids == 3, -1, np.where(ids == 4, V, ids))
    x = np.full((n, F), 0.5)
    x[ids == 1] = -0.0
    x[np.flatnonzero(ids == 2)[::2]] = -0.5
    assert (ids == 2).sum() % 2 == 0
    dtable = Mat(np.full((V, F), 3.0), "f32", F + 1)
    ws, size = ws_of(B.embed_bwd_workspace_bytes(n, V, F))
    B.embed_bwd(n, dev(ids), V, F, Mat(x, t).p, F, CODE[t], scale, dtable.p, F + 1, accumulate, ws, size)
    torch.cuda.synchronize()
    got = dtable.get()
    assert (got[3:] == (3.0 if accumulate else 0.0)).all()
    assert np.isnan(got[1:3]).all()
    assert np.isnan(got[0]).all() if np.isnan(scale) else (got[0] == scale).all()


@pytest.mark.gpu
@pytest.mark.parametrize("n,V,F,t", [(9000, 30, 64, "f32"), (200, 20, 16, "f32"), (20_000, 7, 200, "bf16")])
def test_tables_recorded_and_replayed(n, V, F, t):
    """tables in LDS, more and less of it than a launch has by itself"""
    rng = np.random.default_rng(11)
    ids = dev(some_ids(n, V, rng, "outside"))
    dY, dtable, more = Mat(rng.standard_normal((n, F)), t), new(V, F, "f32"), Mat(rng.standard_normal((V, F)), "f32")
    start = more.bits.clone()
    ws, size = ws_of(B.embed_bwd_workspace_bytes(n, V, F))

    def run(st):
        import torch
        with torch.cuda.stream(st):
            more.bits.copy_(start)
        B.embed_bwd(n, ids, V, F, dY.p, F, CODE[t], 2.0, dtable.p, F, 0, ws, size, stream=st)
        B.embed_bwd(n, ids, V, F, dY.p, F, CODE[t], 2.0, more.p, F, 1, ws, size, stream=st)
    replayed(run, lambda: [dtable.raw(), more.raw()])
