"""Learnt rows, a graph layer, the norm, products with an epilogue, the losses and the clipped step in one chain, as a residual vertex model
is trained with them, against the same model in float64 (torch's automatic differentiation on the CPU); its serving form with 8-bit rows;
and the harness's epochs with clipping.

Tolerance of the chain: 1e-4 norm-wise per tensor, the bar of this library's fp32 chains (every kernel sums in float in a fixed order; here the
longest sum has 700 terms, 700 * 2^-24 = 4e-5 if every rounding went the same way)."""
import numpy as np
import pytest

from paper_2508_13716_amd import binding as B
from tests.row_ops import EPS, HALF, Mat, close, held, new, replayed, vec, ws_of

N, V, F, HID, C, SCALE, NORM_EPS = 700, 90, 48, 96, 10, 6.9, 1e-5


def problem(seed=0):
    rng = np.random.default_rng(seed)
    f = lambda *s, k=1.0: held(rng.standard_normal(s) * k, "f32")
    cols = [np.unique(np.append(rng.integers(0, N, rng.integers(0, 9)), i)) for i in range(N)]
    rowptr = np.cumsum([0] + [len(c) for c in cols]).astype(np.int64)
    p = dict(table=f(V, F, k=F ** -0.5), W1=f(F, F, k=F ** -0.5), b1=f(1, F, k=0.1), w=1 + f(1, F, k=0.2), Wa=f(HID, F, k=F ** -0.5), ba=f(1, HID, k=0.1),
             Wb=f(F, HID, k=HID ** -0.5), bb=f(1, F, k=0.1), Wc=f(C, F, k=F ** -0.5), bc=f(1, C, k=0.1))
    ids = np.minimum(np.exp(rng.random(N) * np.log(V + 1)).astype(np.int64) - 1, V - 1)
    ids[5] = -1                                     # a vertex without a row of its own
    return p, ids, rowptr, np.concatenate(cols).astype(np.int32), rng.integers(0, C, N).astype(np.int32)


def in_float64(p, ids, rowptr, col, labels):
    import torch
    t = {k: torch.from_numpy(v.copy()).requires_grad_(True) for k, v in p.items()}
    d = np.diff(rowptr)
    A = torch.zeros(N, N, dtype=torch.float64)
    for i in range(N):
        for e in range(rowptr[i], rowptr[i + 1]):
            A[i, col[e]] += 1.0 / np.sqrt(float(d[i]) * float(d[col[e]]))
    known = torch.from_numpy(ids >= 0)[:, None]
    x0 = torch.where(known, SCALE * t["table"][torch.from_numpy(np.maximum(ids, 0))], 0.0)
    h1 = A @ x0 @ t["W1"] + t["b1"]
    s = h1 + x0
    y = s * (s.square().mean(1, keepdim=True) + NORM_EPS).rsqrt() * t["w"]
    z = torch.nn.functional.gelu(y @ t["Wa"].t() + t["ba"])
    h2 = z @ t["Wb"].t() + t["bb"] + s
    logits = h2 @ t["Wc"].t() + t["bc"]
    loss = torch.nn.functional.cross_entropy(logits, torch.from_numpy(labels).long())
    loss.backward()
    return float(loss.detach()), logits.detach().numpy(), {k: v.grad.numpy() for k, v in t.items()}


class OnGpu:
    def __init__(self, p, ids, rowptr, col, labels):
        import torch
        r, c = B.norm_scales(B.NORM_SYM, N, 0, rowptr, None)
        self.graph = B.Graph(N, 0, rowptr, col, r, c, None, 0)
        self.W = {k: Mat(v, "f32") for k, v in p.items()}
        self.g = {k: new(*v.shape, "f32") for k, v in p.items()}
        self.ids, self.labels = torch.from_numpy(ids).cuda(), torch.from_numpy(labels).cuda()
        self.layer = B.make_layer(B.GCN, F, F, B.ACT_NONE, B.F32, self.W["W1"].p, None, self.W["b1"].p, B.XFORM_FIRST)
        self.saved = torch.zeros(max(B.layer_saved_bytes(self.graph, self.layer), 256), dtype=torch.uint8, device="cuda")
        f = lambda *s: new(*s, "f32")
        self.x0, self.h1, self.s, self.y, self.rstd, self.u, self.z, self.h2, self.logits = f(N, F), f(N, F), f(N, F), f(N, F), f(1, N), f(N, HID), f(N, HID), f(N, F), f(N, C)
        self.dlogits, self.dh2, self.dz, self.du, self.dy, self.ds, self.dlayer, self.dx0 = f(N, C), f(N, F), f(N, HID), f(N, HID), f(N, F), f(N, F), f(N, F), f(N, F)
        self.loss = torch.zeros(1, device="cuda")
        sizes = [B.embed_bwd_workspace_bytes(N, V, F), B.rmsnorm_bwd_workspace_bytes(N, F), B.linear_act_bwd_workspace_bytes(N, HID), B.loss_workspace_bytes(N),
                 B.layer_workspace_bytes(self.graph, self.layer)]
        sizes += [B.linear_workspace_bytes(N, o, k, B.F32) for o, k in ((HID, F), (F, HID), (C, F))]
        sizes += [B.gemm_workspace_bytes(1, o, k, N) for o, k in ((HID, F), (F, HID), (C, F))] + [B.gemm_workspace_bytes(0, N, k, o) for o, k in ((HID, F), (F, HID), (C, F))]
        self.ws, self.size = ws_of(max(sizes))
        torch.cuda.synchronize()

    def linear(self, x, k, W, o, bias, act, R, U, Y, st):
        B.linear(N, o, k, x.p, k, None, self.W[W].p, k, None, B.F32, self.W[bias].p, act, None if R is None else R.p, o, None if U is None else U.p, o, Y.p, o, B.F32,
                 self.ws, self.size, stream=st)

    def products(self, dU, o, x, k, W, dX, st):
        """dW = dU^T x, dX = dU W"""
        B.gemm(1, 0, o, k, N, dU.p, o, x.p, k, self.g[W].p, k, B.F32, 1, 0, None, 0, None, 0, stream=st, ws=self.ws, ws_bytes=self.size)
        B.gemm(0, 0, N, k, o, dU.p, o, self.W[W].p, k, dX.p, k, B.F32, 1, 0, None, 0, None, 0, stream=st, ws=self.ws, ws_bytes=self.size)

    def run(self, st):
        W, g, ws = self.W, self.g, (self.ws, self.size)
        B.embed(N, self.ids, V, F, W["table"].p, F, B.F32, SCALE, self.x0.p, F, B.F32, stream=st)
        B.layer_fwd(self.graph, self.layer, self.x0.p, F, self.h1.p, F, self.saved, *ws, stream=st)
        B.rmsnorm(N, F, self.h1.p, F, self.x0.p, F, self.s.p, F, B.F32, W["w"].p, NORM_EPS, self.y.p, F, B.F32, None, self.rstd.p, stream=st)
        self.linear(self.y, F, "Wa", HID, "ba", B.ACT_GELU, None, self.u, self.z, st)
        self.linear(self.z, HID, "Wb", F, "bb", B.ACT_NONE, self.s, None, self.h2, st)
        self.linear(self.h2, F, "Wc", C, "bc", B.ACT_NONE, None, None, self.logits, st)
        B.softmax_ce(N, C, self.logits.p, C, self.labels, None, 0.0, self.loss, self.dlogits.p, C, B.F32, *ws, stream=st)
        # backward: each product's epilogue first (dU and the bias's gradient), then the two products
        B.linear_act_bwd(N, C, self.dlogits.p, C, None, 0, B.F32, B.ACT_NONE, None, 0, g["bc"].p, *ws, stream=st)
        self.products(self.dlogits, C, self.h2, F, "Wc", self.dh2, st)
        B.linear_act_bwd(N, F, self.dh2.p, F, None, 0, B.F32, B.ACT_NONE, None, 0, g["bb"].p, *ws, stream=st)
        self.products(self.dh2, F, self.z, HID, "Wb", self.dz, st)
        B.linear_act_bwd(N, HID, self.dz.p, HID, self.u.p, HID, B.F32, B.ACT_GELU, self.du.p, HID, g["ba"].p, *ws, stream=st)
        self.products(self.du, HID, self.y, F, "Wa", self.dy, st)
        B.rmsnorm_bwd(N, F, self.dy.p, F, B.F32, self.s.p, F, B.F32, W["w"].p, self.rstd.p, self.dh2.p, F, self.ds.p, F, g["w"].p, *ws, stream=st)
        # ds reaches x0 on the residual's way and through the layer, whose backward pass overwrites its input
        B.embed_bwd(N, self.ids, V, F, self.ds.p, F, B.F32, SCALE, g["table"].p, F, 0, *ws, stream=st)
        B.layer_bwd(self.graph, self.layer, self.x0.p, F, self.h1.p, F, self.saved, self.ds.p, F, g["W1"].p, None, g["b1"].p, self.dx0.p, F, False, *ws, stream=st)
        B.embed_bwd(N, self.ids, V, F, self.dx0.p, F, B.F32, SCALE, g["table"].p, F, 1, *ws, stream=st)


def normwise(got, want):
    return np.abs(got - want).max() / np.abs(want).max()


@pytest.mark.gpu
def test_a_training_step_of_a_residual_model():
    import torch
    data = problem()
    loss, logits, grads = in_float64(*data)
    m = OnGpu(*data)
    st = torch.cuda.Stream()
    m.run(st)
    torch.cuda.synchronize()
    assert abs(m.loss.item() - loss) <= 1e-5 * abs(loss)
    assert normwise(m.logits.get(), logits) <= 1e-4
    for k, want in grads.items():
        assert normwise(m.g[k].get(), want) <= 1e-4, k
    # the step on all of them, clipped to a third of their norm
    names = list(grads)
    tensors = B.TensorList([m.g[k].view for k in names], [m.W[k].view for k in names])
    total = float(np.sqrt(sum((grads[k] ** 2).sum() for k in names)))
    norm = torch.zeros(1, device="cuda")
    ws, size = ws_of(B.grad_workspace_bytes(tensors))
    B.clipped_step(tensors, 0.5, total / 3, norm, ws, size, stream=st)
    torch.cuda.synchronize()
    assert abs(norm.item() - total) <= 1e-4 * total
    for k in names:
        moved = m.W[k].get() - data[0][k]
        assert normwise(moved, -0.5 / 3 * grads[k]) <= 1e-4 + 2 * EPS * np.abs(data[0][k]).max() / np.abs(0.5 / 3 * grads[k]).max(), k


@pytest.mark.gpu
def test_the_training_step_recorded_and_replayed():
    m = OnGpu(*problem(1))
    replayed(m.run, lambda: [m.logits.raw(), m.loss.cpu().clone()] + [v.raw() for v in m.g.values()])


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 9, 130])
@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_serving_with_8_bit_rows(n, t):
    """residual stream -> norm into 8 bits -> 8-bit product with activation -> product back, added to the stream in place"""
    import torch
    F, HID = 200, 330
    code = {"f32": B.F32, "bf16": B.BF16}[t]
    rng = np.random.default_rng(n)
    x, r = held(rng.standard_normal((n, F)), t), held(rng.standard_normal((n, F)), t)
    wa, wb, w = held(rng.standard_normal((HID, F)) / F ** 0.5, "f32"), held(rng.standard_normal((F, HID)) / HID ** 0.5, t), held(1 + 0.1 * rng.standard_normal((1, F)), "f32")
    Wq, Ws = new(HID, F, "e4m3"), new(1, HID, "f32")
    B.quantize_rows(HID, F, Mat(wa, "f32").p, F, B.F32, Wq.p, F, Ws.p)
    X, R, Q, S, Z, Wb, wd = Mat(x, t), Mat(r, t), new(n, F, "e4m3"), new(1, n, "f32"), new(n, HID, t), Mat(wb, t), vec(w)
    ws, size = ws_of(max(B.linear_workspace_bytes(n, HID, F, B.E4M3), B.linear_workspace_bytes(n, F, HID, code)))
    B.rmsnorm(n, F, X.p, F, R.p, F, X.p, F, code, wd.p, 1e-6, Q.p, F, B.E4M3, S.p)
    B.linear(n, HID, F, Q.p, F, S.p, Wq.p, F, Ws.p, B.E4M3, None, B.ACT_SILU, None, 0, None, 0, Z.p, HID, code, ws, size)
    before = X.raw()
    B.linear(n, F, HID, Z.p, HID, None, Wb.p, HID, None, code, None, B.ACT_NONE, X.p, F, None, 0, X.p, F, code, ws, size)
    torch.cuda.synchronize()
    h = before.view(torch.float32 if t == "f32" else torch.bfloat16)[: n * F].double().numpy().reshape(n, F)
    close(h, x + r, np.abs(x + r) * (EPS + HALF[t]) * 1.001)
    # each step from what the one before left
    q, wq = Q.get() * S.get().T, Wq.get() * Ws.get().T
    y = (x + r) / np.sqrt(((x + r) ** 2).mean(1, keepdims=True) + 1e-6) * w
    close(q, y, np.maximum(np.abs(y) * HALF["e4m3"], S.get().T * 2.0 ** -10) * 1.001 + 100 * EPS * np.abs(y))
    close(wq, wa, np.maximum(np.abs(wa) * HALF["e4m3"], Ws.get().T * 2.0 ** -10) * 1.001)
    u = q @ wq.T
    largest = np.abs(q).max(1, keepdims=True) * np.abs(wq).max(1)       # of a group of eight products, at most (see test_linear)
    err = np.abs(q) @ np.abs(wq).T * (F + 12) * EPS + (7 * 2.0 ** -13 * largest * (F / 8 + 1) if t == "bf16" else 0)
    z = u / (1 + np.exp(-u))
    close(Z.get(), z, 1.13 * err + 8 * EPS * np.abs(u) + HALF[t] * np.abs(z) * 1.001)
    out = Z.get() @ wb.T + h
    close(X.get(), out, np.abs(Z.get()) @ np.abs(wb).T * (HID + 12) * EPS + (2 * EPS + HALF[t]) * np.abs(out) * 1.001)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,dtype,dims", [("gcn", "f32", [96, 64, 24]), ("sage", "bf16", [64, 32, 8])])
def test_epochs_with_clipping(kind, dtype, dims):
    """the harness's epoch with max_norm: the epoch's gradients, then the clipped step on all of a model's tensors"""
    import torch
    from paper_2508_13716_amd import harness as H, synth
    from tests import oracle_side as O
    cfg = synth.Config(f"clipped-{kind}", kind, 2500, 2000, 30_000, dims, dtype, 0.5, max_deg=300, seed=synth.BASE_SEED * 10 + 7)
    prob = H.make_problem(cfg, mask_frac=0.5)
    plain, dp = H.DeviceProblem(prob), H.DeviceProblem(prob)
    plain.run_epoch()
    want = plain.results()
    flat = [g.astype(np.float64) for g in want["dW"] + want["dW_self"] + want["db"] if g is not None]
    norm = float(np.sqrt(sum((g ** 2).sum() for g in flat)))
    tensors = lambda d: [t for t in d.W + d.W_self + d.bias if t is not None]
    before = [O.widen(H.dev_to_np(t)) for t in tensors(dp)]
    lr, limit = 0.25, float(np.float32(norm / 2))
    loss, _ = dp.run_epoch(lr=lr, max_norm=limit)
    got = dp.results()
    for a, b in zip(got["dW"] + got["db"], want["dW"] + want["db"]):
        assert np.array_equal(a, b)                  # the gradients stay
    assert abs(dp.grad_norm.item() - norm) <= norm * EPS * 1.01
    for t, p0, g in zip(tensors(dp), before, flat):
        step = lr * limit / norm * g.reshape(p0.shape)
        ref = p0 - step
        half = HALF["bf16"] if t.dtype == torch.bfloat16 else EPS
        close(O.widen(H.dev_to_np(t)), ref, (np.abs(step) * 2 * EPS + np.abs(ref) * (EPS + half)) * 1.001)
    second, _ = dp.run_epoch(lr=lr, max_norm=1e9)    # (no clipping any more)
    assert np.isfinite(second) and second != loss
    plain.close()
    dp.close()
