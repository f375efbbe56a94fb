"""capgnn_tensors_create, capgnn_grad_norm, capgnn_grad_clip and capgnn_clipped_step against float64, and what they refuse.

Tolerances: the norm is summed in double (far below a float's rounding) and rounded once.  A clipped gradient is one product with a
rounded factor (2 EPS) and one rounding to its type; a step one fused operation with a rounded factor, and one rounding."""
import ctypes as C

import numpy as np
import pytest

from paper_2508_13716_amd import binding as B
from tests.row_ops import CODE, EPS, FAKE, HALF, close, held, refuse, replayed, ttype, ws_of


def create(grads, dtypes, counts, params=None, param_dtypes=None, n=None):
    n = len(counts) if n is None else n
    arr = lambda t, v: None if v is None else (t * max(len(v), 1))(*v)
    h = C.c_void_p()
    rc = B.lib().capgnn_tensors_create(C.byref(h), n, arr(C.c_void_p, grads), arr(C.c_int32, dtypes), arr(C.c_void_p, params), arr(C.c_int32, param_dtypes),
                                       arr(C.c_int64, counts), None)
    return rc, h


@pytest.mark.parametrize("a", [
    dict(grads=[FAKE], dtypes=[0], counts=[4], n=-1), dict(grads=None, dtypes=[0], counts=[4]), dict(grads=[FAKE], dtypes=None, counts=[4]),
    dict(grads=[FAKE], dtypes=[0], counts=None, n=1), dict(grads=[FAKE], dtypes=[2], counts=[4]), dict(grads=[FAKE], dtypes=[0], counts=[-1]),
    dict(grads=[None], dtypes=[0], counts=[4]), dict(grads=[FAKE + 2], dtypes=[0], counts=[4]), dict(grads=[FAKE + 1], dtypes=[1], counts=[4]),
    dict(grads=[FAKE], dtypes=[0], counts=[1 << 50]), dict(grads=[FAKE, FAKE], dtypes=[0, 0], counts=[4, 4]), dict(grads=[FAKE, FAKE + 12], dtypes=[0, 0], counts=[4, 4]),
    dict(grads=[FAKE], dtypes=[0], counts=[4], params=[FAKE + 8], param_dtypes=[0]), dict(grads=[FAKE], dtypes=[0], counts=[4], params=[None], param_dtypes=[0]),
    dict(grads=[FAKE], dtypes=[0], counts=[4], params=[2 * FAKE], param_dtypes=None), dict(grads=[FAKE], dtypes=[0], counts=[4], params=[2 * FAKE], param_dtypes=[5]),
    dict(grads=[FAKE, 2 * FAKE], dtypes=[0, 0], counts=[4, 4], params=[3 * FAKE, 3 * FAKE + 4], param_dtypes=[0, 0])])
def test_bad_lists_are_refused(a):
    rc, h = create(**a)
    assert rc == B.EINVAL and not h


def test_calls_are_refused():
    rc, h = create([None], [0], [0])                 # an empty list needs no GPU
    assert rc == B.OK

    class L:
        pass
    t = L()
    t.h = h
    need = B.grad_workspace_bytes(t)
    assert need >= 8
    for f, extra in ((B.grad_norm, ()), (B.grad_clip, (1.0,)), (B.clipped_step, (0.1, 1.0))):
        code = B.EINVAL if f is B.clipped_step else None
        refuse(B.EINVAL, f, t, *extra, None, FAKE, need)
        refuse(B.EINVAL, f, t, *extra, FAKE + 2, FAKE, need)
        refuse(B.ENOMEM, f, t, *extra, FAKE, None, need)
        refuse(B.ENOMEM, f, t, *extra, FAKE, FAKE, need - 1)
        refuse(B.EINVAL, f, t, *extra, FAKE, FAKE + 64, need)
        if code:
            refuse(code, f, t, *extra, FAKE, FAKE, need)          # no params
    for bad in (-1.0, float("nan")):
        refuse(B.EINVAL, B.grad_clip, t, bad, FAKE, FAKE, need)
    none = L()
    none.h = None
    refuse(B.EINVAL, B.grad_norm, none, FAKE, FAKE, need)
    assert B.grad_workspace_bytes(none) == 0
    B.lib().capgnn_tensors_destroy(h)
    assert B.lib().capgnn_tensors_destroy(None) == B.OK


def test_the_list_takes_dense_float_tensors_alone():
    import torch
    with pytest.raises(ValueError):
        B.TensorList([torch.zeros(4, dtype=torch.float16)])
    with pytest.raises(ValueError):
        B.TensorList([torch.zeros(4, 4).t()[1:]])
    with pytest.raises(ValueError):
        B.TensorList([torch.zeros(4)], [torch.zeros(5)])


def test_the_list_takes_tensors_on_the_gpu_alone():
    """a host address would reach the kernels"""
    import torch
    for t in (torch.float32, torch.bfloat16):
        with pytest.raises(ValueError, match="GPU"):
            B.TensorList([torch.zeros(4, dtype=t)])
        with pytest.raises(ValueError, match="GPU"):
            B.TensorList([torch.zeros(4, dtype=t)], [torch.zeros(4, dtype=t)])
    with pytest.raises(ValueError, match="GPU"):
        B.TensorList([torch.zeros(4, device="meta")])


@pytest.mark.gpu
def test_the_list_takes_no_host_tensor_among_others():
    import torch
    on = torch.zeros(4, device="cuda")
    for grads, params in (([on, torch.zeros(4)], None), ([on], [torch.zeros(4)]), ([torch.zeros(4).pin_memory()], [on])):
        with pytest.raises(ValueError, match="GPU"):
            B.TensorList(grads, params)


# ----------------------------------------------------------------------------- the GPU
class Model:
    """tensors of given sizes, one after the other in one allocation, each `gap` elements after the last"""

    def __init__(self, sizes, gt, pt, gap=0, seed=0, spread=1.0):
        import torch
        rng = np.random.default_rng(seed)
        self.at, at = [], 1 if gap else 0
        for s in sizes:
            self.at.append((at, at + s))
            at += s + gap
        self.gt, self.pt, self.n = gt, pt, at
        self.g, self.p = held(rng.standard_normal(at) * spread, gt), held(rng.standard_normal(at), pt)
        self.G, self.P = torch.from_numpy(self.g).to(ttype(gt)).cuda(), torch.from_numpy(self.p).to(ttype(pt)).cuda()
        self.list = B.TensorList([self.G[a:b] for a, b in self.at], [self.P[a:b] for a, b in self.at])
        self.norm = torch.zeros(1, device="cuda")
        self.ws, self.size = ws_of(B.grad_workspace_bytes(self.list))
        self.inside = np.zeros(at, bool)
        for a, b in self.at:
            self.inside[a:b] = True

    def want(self):
        return float(np.sqrt((self.g[self.inside] ** 2).sum()))


LISTS = [([1], 0), ([7], 0), ([5, 1, 3], 1), ([2048], 0), ([2049, 1], 0), ([602 * 256, 256, 256 * 41, 41], 0), ([602 * 256, 256, 256 * 41, 41], 3),
         ([0, 9, 0, 100_003], 1), ([(37 * k) % 501 + 1 for k in range(700)], 1), ([6_000_001, 3, 70_000], 5)]


@pytest.mark.gpu
@pytest.mark.parametrize("sizes,gap", LISTS)
@pytest.mark.parametrize("gt,pt", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
def test_norm_clip_and_step(sizes, gap, gt, pt):
    import torch
    m = Model(sizes, gt, pt, gap, seed=len(sizes))
    want = m.want()
    B.grad_norm(m.list, m.norm, m.ws, m.size)
    torch.cuda.synchronize()
    assert abs(m.norm.item() - want) <= want * EPS * 1.01
    assert np.array_equal(m.G.double().cpu().numpy(), m.g)
    for limit in (0.3 * want, 3 * want, float("inf")):
        limit, lr = float(np.float32(limit)), float(np.float32(0.37))
        c = min(1.0, limit / want)
        m.P.copy_(torch.from_numpy(m.p).to(ttype(pt)))
        m.norm.zero_()
        B.clipped_step(m.list, lr, limit, m.norm, m.ws, m.size)
        torch.cuda.synchronize()
        step = np.where(m.inside, m.p - lr * c * m.g, m.p)
        close(m.P.double().cpu().numpy(), step, np.where(m.inside, (np.abs(lr * c * m.g) * EPS + np.abs(step) * EPS + np.abs(step) * HALF[pt]) * 1.001, 0.0), "step")
        assert abs(m.norm.item() - want) <= want * EPS * 1.01
    for limit in (3 * want, 0.3 * want):             # (the second changes the gradients)
        limit = float(np.float32(limit))
        c = min(1.0, limit / want)
        B.grad_clip(m.list, limit, m.norm, m.ws, m.size)
        torch.cuda.synchronize()
        g = np.where(m.inside, m.g * c, m.g)
        close(m.G.double().cpu().numpy(), g, np.where(m.inside & (c < 1), np.abs(g) * (2 * EPS + HALF[gt]) * 1.001, 0.0), "clip")
        assert abs(m.norm.item() - want) <= want * EPS * 1.01


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_a_norm_that_is_not_finite_changes_nothing(bad):
    import torch
    m = Model([100, 5000, 3], "f32", "f32", 1, seed=1)
    m.G[m.at[1][0] + 4000] = bad
    g, q = m.G.clone(), m.P.clone()
    B.clipped_step(m.list, 0.1, 1.0, m.norm, m.ws, m.size)
    B.grad_clip(m.list, 1.0, m.norm, m.ws, m.size)
    torch.cuda.synchronize()
    assert torch.equal(m.G.view(torch.int32), g.view(torch.int32)) and torch.equal(m.P, q)
    assert (np.isnan(m.norm.item()) if np.isnan(bad) else m.norm.item() == np.inf)


@pytest.mark.gpu
def test_a_norm_beyond_a_float_changes_nothing():
    import torch
    m = Model([100, 5000, 3], "f32", "f32", 1, seed=1)
    for at in (m.at[0][0], m.at[1][0], m.at[1][0] + 77):
        m.G[at] = 3e38                               # (each is a float; the norm, 5.2e38, is none)
    g, q = m.G.clone(), m.P.clone()
    B.clipped_step(m.list, 0.1, 1.0, m.norm, m.ws, m.size)
    B.grad_clip(m.list, 1.0, m.norm, m.ws, m.size)
    torch.cuda.synchronize()
    assert torch.equal(m.G, g) and torch.equal(m.P, q) and m.norm.item() == np.inf


@pytest.mark.gpu
def test_squares_beyond_a_float_and_far_below_it():
    import torch
    for spread in (1e30, 1e-30):
        m = Model([4000, 33], "f32", "f32", 0, seed=2, spread=spread)
        want = m.want()
        B.grad_clip(m.list, float(np.float32(0.5 * want)), m.norm, m.ws, m.size)
        torch.cuda.synchronize()
        assert abs(m.norm.item() - want) <= want * EPS * 1.01
        close(m.G.double().cpu().numpy(), 0.5 * m.g, np.abs(0.5 * m.g) * 4 * EPS)


@pytest.mark.gpu
def test_zeros_nothing_and_a_limit_of_zero():
    import torch
    m = Model([300, 4], "f32", "bf16", 0, seed=3)
    m.G.zero_()
    B.clipped_step(m.list, 1.0, 0.0, m.norm, m.ws, m.size)
    torch.cuda.synchronize()
    assert m.norm.item() == 0 and np.array_equal(m.P.double().cpu().numpy(), m.p)
    m.G.fill_(2.0)
    B.grad_clip(m.list, 0.0, m.norm, m.ws, m.size)
    torch.cuda.synchronize()
    assert int(torch.count_nonzero(m.G)) == 0
    empty = B.TensorList([], [])
    norm = torch.full((1,), 7.0, device="cuda")
    ws, size = ws_of(B.grad_workspace_bytes(empty))
    B.grad_norm(empty, norm, ws, size)
    torch.cuda.synchronize()
    assert norm.item() == 0
    norm.fill_(7.0)
    B.clipped_step(empty, 0.1, 1.0, norm, ws, size)
    torch.cuda.synchronize()
    assert norm.item() == 0


@pytest.mark.gpu
def test_recorded_and_replayed_and_on_another_stream():
    import torch
    m = Model([70_000, 256, 9], "f32", "f32", 1, seed=4)
    start = m.P.clone()

    def run(st):
        with torch.cuda.stream(st):
            m.P.copy_(start)
        B.clipped_step(m.list, 0.1, 1.0, m.norm, m.ws, m.size, stream=st)
    replayed(run, lambda: [m.P.cpu().clone(), m.norm.cpu().clone()])
    want = m.P.clone()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    run(st)
    torch.cuda.synchronize()
    assert torch.equal(m.P, want)


@pytest.mark.gpu
def test_a_tensor_beyond_32_bit_offsets():
    import torch
    n = (1 << 32) + 5
    G = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    P = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    G[0] = 3.0
    G[-1] = 4.0
    t = B.TensorList([G], [P])
    norm = torch.zeros(1, device="cuda")
    B.clipped_step(t, 1.0, 10.0, norm, *ws_of(B.grad_workspace_bytes(t)))
    torch.cuda.synchronize()
    assert norm.item() == 5.0 and float(P[0]) == -3.0 and float(P[-1]) == -4.0 and float(P[1]) == 0.0


@pytest.mark.gpu
@pytest.mark.parametrize("gt,pt", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("top,limit,lr", [(3e36, 1e-3, 1e-6), (3e36, 1e-3, -1e-2), (1e36, 1e-5, 1.0), (3e36, 1e-36, 1e5), (1e30, 1e-9, 1e-30), (1e36, 1e38, 1e-43)])
def test_factors_below_floats_normal_range(gt, pt, top, limit, lr):
    """norms that are large but finite: the factor has few bits as a float, or none, its product with a gradient all of them.  A product far
    below the least normal float is off by a step there at most"""
    import torch
    m = Model([5000, 1, 33], gt, pt, 1, seed=5, spread=top)
    m.p *= 0.0
    m.P.zero_()
    want = m.want()
    limit, lr = float(np.float32(limit)), float(np.float32(lr))
    c = min(1.0, limit / want)
    step = 2.0 ** -149 if "f32" == pt else 2.0 ** -133
    B.clipped_step(m.list, lr, limit, m.norm, m.ws, m.size)
    torch.cuda.synchronize()
    assert abs(m.norm.item() - want) <= want * EPS * 1.01
    to = np.where(m.inside, -lr * c * m.g, 0.0)
    close(m.P.double().cpu().numpy(), to, np.where(m.inside, np.abs(to) * (2 * EPS + HALF[pt]) * 1.001 + 2.0 ** -149 + step, 0.0), "step")
    step = 2.0 ** -149 if "f32" == gt else 2.0 ** -133
    B.grad_clip(m.list, limit, m.norm, m.ws, m.size)
    torch.cuda.synchronize()
    to = np.where(m.inside, m.g * c, m.g)
    close(m.G.double().cpu().numpy(), to, np.where(m.inside & (c < 1), np.abs(to) * (2 * EPS + HALF[gt]) * 1.001 + 2.0 ** -149 + step, 0.0), "clip")
