"""What a residual vertex model is built and trained with beside its aggregation, as timed cases: rows of learnt embeddings and their
gradient by sorted ids, the root-mean-square norm with the residual's addition (and 8-bit rows for the product that follows), the
product with bias, activation and residual in its epilogue, and the update with the gradients' global norm clipped.

Widths go from the vertex classifiers of ``paper_2508_13716_amd/synth.py`` (100, 256, 602) to wide layers; row counts from one request
to the vertices of a partition.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
E4M3_MAX = 448.0
TINY = 2.0 ** -100        # rows whose largest value is below it are brought to 8 bits as if it were this


def _case(op, name=None, **kw):
    base = {"embed": dict(n=1, V=2, F=1, dtype="f32", pad=0, scale=1.0),
            "embed_bwd": dict(n=1, V=2, F=1, dtype="f32", pad=0, scale=1.0, accumulate=False),
            "norm": dict(n=1, F=1, dtype="f32", out="f32", pad=0, residual=True, weight=True),
            "norm_bwd": dict(n=1, F=1, dtype="f32", pad=0, residual=True, weight=True),
            "linear": dict(M=1, N=1, K=1, dtype="f32", out="f32", pad=0, act="none", bias=True, residual=False, save=False),
            "linear_train": dict(M=1, N=1, K=1, dtype="f32", out="f32", pad=0, act="gelu", bias=True, residual=False, save=True),
            "step": dict(count=1, total=1, align=64, params="f32", grads="f32", max_norm=1.0, lr=0.1)}[op]
    c = dict(op=op, **{**base, **kw})
    return dict(c, name=name) if name else c


def listed():
    return [
        # a request's few rows out of a large table, scaled by the root of the width
        _case("embed", "embed_request", n=64, V=131_072, F=1_024, dtype="bf16", scale=32.0),
        # the gradient of a table with one row per class of vertices: few rows, every one of them hit thousands of times
        _case("embed_bwd", "embed_grad_classes", n=612_000, V=47, F=100),
        # ... and with a row per vertex, drawn by a power law: most rows are not hit, some very often
        _case("embed_bwd", "embed_grad_vertices", n=300_001, V=500_009, F=256, dtype="bf16", scale=16.0),
        # one row on its way into an 8-bit product
        _case("norm", "norm_one_row", n=1, F=4_096, dtype="bf16", out="e4m3"),
        # a partition's vertices between two layers, fp32 rows of a width that is no power of two
        _case("norm", "norm_vertices", n=180_000, F=602, pad=6),
        # the backward pass over a training batch of wide rows
        _case("norm_bwd", "norm_grad_wide", n=16_384, F=4_096, dtype="bf16"),
        # one row through a wide layer: the weights' bytes bound it
        _case("linear", "linear_one_row", M=1, N=4_096, K=4_096, dtype="bf16", out="bf16", act="silu", residual=True),
        # training on odd sizes: forward with the values before the activation kept, and the activation's backward pass
        _case("linear_train", "linear_ragged", M=3_001, N=1_009, K=602, pad=5, act="gelu"),
        # a wide layer over a training batch
        _case("linear", "linear_wide", M=8_192, N=8_192, K=8_192, dtype="bf16", out="bf16", act="gelu", residual=True),
        # the same layer served with 8-bit rows and weights
        _case("linear", "linear_wide_8bit", M=8_192, N=8_192, K=4_096, dtype="e4m3", out="bf16", act="silu", residual=True),
        # the few small tensors of a two-layer model (602-256-41): launches and latency
        _case("step", "step_small", count=4, total=164_905, max_norm=5.0),
        # a wide model's tensors, bf16 weights with fp32 gradients
        _case("step", "step_large", count=300, total=120_000_000, params="bf16", max_norm=100.0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["embed", "embed_bwd", "norm", "norm_bwd", "linear", "linear", "linear_train", "step"])
    pad = rng.choice([0, 0, 0, 8, 16, rng.randint(1, 31)])
    half = rng.choice(["f32", "bf16"])
    if op in ("embed", "embed_bwd"):
        F = _log_int(rng, 1, 2_048)
        kw = dict(n=_log_int(rng, 1, min(612_000, 76_800_000 // F)), V=_log_int(rng, 1, min(1_000_000, 128_000_000 // F)), F=F, dtype=half,
                  pad=pad, scale=rng.choice([1.0, round(math.sqrt(F), 3)]))
        return _case(op, **kw, **({"accumulate": rng.random() < 0.5} if op == "embed_bwd" else {}))
    if op in ("norm", "norm_bwd"):
        F = _log_int(rng, 1, 16_384)
        kw = dict(n=_log_int(rng, 1, min(1_000_000, 67_000_000 // F)), F=F, dtype=half, pad=pad, residual=rng.random() < 0.7,
                  weight=rng.random() < 0.8)
        return _case(op, **kw, **({"out": rng.choice([half, half, "e4m3"])} if op == "norm" else {}))
    if op in ("linear", "linear_train"):
        M, N = _log_int(rng, 1, 16_384), _log_int(rng, 1, 16_384)
        K = _log_int(rng, 1, min(16_384, 8_192 ** 3 // (M * N)))
        dtype = rng.choice(["f32", "bf16"] if op == "linear_train" else ["f32", "bf16", "bf16", "e4m3"])
        return _case(op, M=M, N=N, K=K, dtype=dtype, out=rng.choice([dtype, dtype, "f32"]) if dtype != "e4m3" else half, pad=pad,
                     # (the slope of relu next to 0 goes by a sign that rounding decides: training cases take the smooth ones)
                     act=rng.choice(["none", "gelu", "silu"] + ["relu"] * (op == "linear")), bias=rng.random() < 0.8, residual=rng.random() < 0.5,
                     save=op == "linear_train")
    total = _log_int(rng, 1_000, 120_000_000)
    return _case(op, count=rng.randint(1, 400), total=total, align=rng.choice([64, 64, 1]), params=half, grads=rng.choice(["f32", "f32", half]),
                 max_norm=round(0.03 * math.sqrt(total) * rng.choice([0.1, 0.5, 2.0]), 3))


# ------------------------------------------------------------------ sizes
def _distinct(n, V):
    """rows that n draws of _ids hit, as expected"""
    r = torch.arange(1, V + 1, dtype=torch.float64)
    return float((-torch.expm1(n * torch.log1p(-(torch.log1p(1 / r) / math.log(V + 1)).clamp(max=1 - 1e-12)))).sum())


def _counts(case):
    """the tensors' sizes: of every four one weight matrix, a bias, a narrow matrix and a small one"""
    share = [(1.0, 0.004, 0.07, 0.02)[i % 4] for i in range(case["count"])]
    return [max(1, int(case["total"] * s / sum(share))) for s in share]


def work(case):
    size = lambda t: TYPES[t].itemsize
    op = case["op"]
    if op in ("embed", "embed_bwd"):
        n, V, F, s = case["n"], case["V"], case["F"], size(case["dtype"])
        hit = _distinct(n, V)
        if op == "embed":
            return {"bytes": n * 8 + (hit + n) * F * s, "flops": n * F}
        return {"bytes": n * 8 + n * F * s + (2 * hit if case["accumulate"] else V) * F * 4, "flops": 2 * n * F}
    if op in ("norm", "norm_bwd"):
        n, F, s = case["n"], case["F"], size(case["dtype"])
        w = 4 * F if case["weight"] else 0
        if op == "norm":
            return {"bytes": n * F * (s * (3 if case["residual"] else 1) + size(case["out"])) + w + n * (8 if case["out"] == "e4m3" else 4),
                    "flops": 5 * n * F}
        return {"bytes": n * F * s * (4 if case["residual"] else 3) + 2 * w + 4 * n, "flops": 8 * n * F}
    if op in ("linear", "linear_train"):
        M, N, K, s, o = case["M"], case["N"], case["K"], size(case["dtype"]), size(case["out"])
        out = 1 + case["residual"] + case["save"] + (3 if op == "linear_train" else 0)
        return {"bytes": (M + N) * K * s + M * N * o * out + (4 * N if case["bias"] else 0) + (4 * N if op == "linear_train" else 0)
                + (4 * (M + N) if case["dtype"] == "e4m3" else 0), "flops": 2 * M * N * K}
    total, p, g = sum(_counts(case)), size(case["params"]), size(case["grads"])
    return {"bytes": total * (2 * g + 2 * p), "flops": 4 * total}


# ------------------------------------------------------------------ inputs
def _rows8(v):
    """rows in 8 bits with a scale each"""
    s = v.abs().amax(1).clamp(min=TINY) / E4M3_MAX
    return (v / s[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), s


def _ids(n, V, g):
    """ids by a power law (rank r with a probability of about 1/r), ranks scattered over the table"""
    rank = torch.exp(torch.rand(n, generator=g, device="cuda", dtype=torch.float64) * math.log(V + 1)).long().clamp(1, V) - 1
    return (rank * 7_368_787 + 12_345) % V


def _padded(rows, cols, pad, dtype, fill=0.0):
    return torch.full((rows, cols + pad), fill, device="cuda").to(dtype)


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")
    x, op = {"case": case}, case["op"]
    if op in ("embed", "embed_bwd"):
        n, V, F, pad, dt = case["n"], case["V"], case["F"], case["pad"], TYPES[case["dtype"]]
        x["ids"] = _ids(n, V, g)
        if op == "embed":
            x["table"] = (rand(V, F + pad) / math.sqrt(F)).to(dt)
        else:
            x["dY"] = (rand(n, F + pad) / math.sqrt(n)).to(dt)
            if case["accumulate"]:
                x["dtable"] = rand(V, F + pad) / math.sqrt(n)
    elif op in ("norm", "norm_bwd"):
        n, F, pad, dt = case["n"], case["F"], case["pad"], TYPES[case["dtype"]]
        level = torch.exp(0.5 * rand(n, 1))                     # rows differ in size as a residual stream's do
        x["X"] = (level * rand(n, F + pad)).to(dt)
        x["w"] = 1.0 + 0.2 * rand(F) if case["weight"] else None
        if op == "norm":
            x["R"] = (0.5 * rand(n, F + pad)).to(dt) if case["residual"] else None
        else:
            x["dY"] = (rand(n, F + pad) / math.sqrt(n)).to(dt)
            x["dH"] = (rand(n, F + pad) / math.sqrt(n)).to(dt) if case["residual"] else None
            x["rstd"] = (x["X"][:, :F].double().square().mean(1) + 1e-6).rsqrt().float()
    elif op in ("linear", "linear_train"):
        M, N, K, pad, dt, out = case["M"], case["N"], case["K"], case["pad"], TYPES[case["dtype"]], TYPES[case["out"]]
        A, W = rand(M, K + pad), rand(N, K + pad) / math.sqrt(K)
        x["a_scale"] = x["w_scale"] = None
        if case["dtype"] == "e4m3":
            x["A"], x["a_scale"] = _rows8(A)
            x["W"], x["w_scale"] = _rows8(W)
        else:
            x["A"], x["W"] = A.to(dt), W.to(dt)
        x["bias"] = 0.1 * rand(N) if case["bias"] else None
        x["R"] = rand(M, N + pad).to(out) if case["residual"] else None
        if op == "linear_train":
            x["dY"] = (rand(M, N + pad) / math.sqrt(M)).to(out)
    else:
        at, ends = 0, []
        for c in _counts(case):
            ends.append((at, at + c))
            at = -(-(at + c) // case["align"]) * case["align"]
        x["at"] = ends
        x["params"] = (0.02 * rand(at)).to(TYPES[case["params"]])
        x["grads"] = (0.03 * rand(at)).to(TYPES[case["grads"]])
        inside = torch.zeros(at, dtype=torch.bool, device="cuda")
        for a, b in ends:
            inside[a:b] = True
        x["params"].mul_(inside)                                # what lies between two tensors is no gradient
        x["grads"].mul_(inside)
    return x


def prepare(case, seed):
    x, op = _inputs(case, seed), case["op"]
    new = lambda *s, t=torch.float32: torch.zeros(s, dtype=t, device="cuda")
    ws = 0
    if own:
        from paper_2508_13716_amd import binding as B
    if op == "embed":
        x["out"] = _padded(case["n"], case["F"], case["pad"], TYPES[case["dtype"]])
    elif op == "embed_bwd":
        if not case["accumulate"]:
            x["dtable"] = _padded(case["V"], case["F"], case["pad"], torch.float32)
        ws = B.embed_bwd_workspace_bytes(case["n"], case["V"], case["F"]) if own else 0
    elif op == "norm":
        n, F, pad = case["n"], case["F"], case["pad"]
        x["H"] = _padded(n, F, pad, TYPES[case["dtype"]]) if case["residual"] else None
        x["Y"], x["rstd"] = _padded(n, F, pad, TYPES[case["out"]]), new(n)
        x["y_scale"] = new(n) if case["out"] == "e4m3" else None
    elif op == "norm_bwd":
        n, F, pad = case["n"], case["F"], case["pad"]
        x["dX"], x["dw"] = _padded(n, F, pad, TYPES[case["dtype"]]), new(F) if case["weight"] else None
        ws = B.rmsnorm_bwd_workspace_bytes(n, F) if own else 0
    elif op in ("linear", "linear_train"):
        M, N, pad, out = case["M"], case["N"], case["pad"], TYPES[case["out"]]
        x["Y"] = _padded(M, N, pad, out)
        x["U"] = _padded(M, N, pad, out) if case["save"] else None
        if op == "linear_train":
            x["dU"], x["dbias"] = _padded(M, N, pad, out), new(N)
        if own:
            ws = B.linear_workspace_bytes(M, N, case["K"], _code(B, case["dtype"]))
            if op == "linear_train":
                ws = max(ws, B.linear_act_bwd_workspace_bytes(M, N))
    else:
        x["norm"] = new(1)
        if own:
            view = lambda t: [t[a:b] for a, b in x["at"]]
            x["list"] = B.TensorList(view(x["grads"]), view(x["params"]))
            ws = B.grad_workspace_bytes(x["list"])
    if own:
        x["ws"], x["ws_bytes"] = torch.empty(max(ws, 256), dtype=torch.uint8, device="cuda"), ws
    return x


def run(x):
    return _run_own(x) if own else _run_plain(x)


# ------------------------------------------------------------------ the framework's calls
def _code(B, t):
    return {"f32": B.F32, "bf16": B.BF16, "e4m3": B.E4M3}[t]


def _run_own(x):
    from paper_2508_13716_amd import binding as B
    c, st = x["case"], torch.cuda.current_stream()
    op, pad = c["op"], c.get("pad", 0)
    if op in ("embed", "embed_bwd"):
        n, V, F, dt = c["n"], c["V"], c["F"], _code(B, c["dtype"])
        ld = F + pad
        if op == "embed":
            B.embed(n, x["ids"], V, F, x["table"], ld, dt, c["scale"], x["out"], ld, dt, stream=st)
            return {"out": x["out"][:, :F]}
        B.embed_bwd(n, x["ids"], V, F, x["dY"], ld, dt, c["scale"], x["dtable"], ld, int(c["accumulate"]), x["ws"], x["ws_bytes"], stream=st)
        return {"dtable": x["dtable"][:, :F]}
    if op == "norm":
        n, F, dt = c["n"], c["F"], _code(B, c["dtype"])
        ld = F + pad
        B.rmsnorm(n, F, x["X"], ld, x["R"], ld, x["H"], ld, dt, x["w"], 1e-6, x["Y"], ld, _code(B, c["out"]), x["y_scale"], x["rstd"], stream=st)
        return {"Y": x["Y"][:, :F], "H": None if x["H"] is None else x["H"][:, :F], "y_scale": x["y_scale"], "rstd": x["rstd"]}
    if op == "norm_bwd":
        n, F, dt = c["n"], c["F"], _code(B, c["dtype"])
        ld = F + pad
        B.rmsnorm_bwd(n, F, x["dY"], ld, dt, x["X"], ld, dt, x["w"], x["rstd"], x["dH"], ld, x["dX"], ld, x["dw"], x["ws"], x["ws_bytes"],
                      stream=st)
        return {"dX": x["dX"][:, :F], "dw": x["dw"]}
    if op in ("linear", "linear_train"):
        M, N, K, out = c["M"], c["N"], c["K"], _code(B, c["out"])
        ldk, ldn, act = K + pad, N + pad, {"none": B.ACT_NONE, "relu": B.ACT_RELU, "gelu": B.ACT_GELU, "silu": B.ACT_SILU}[c["act"]]
        B.linear(M, N, K, x["A"], ldk, x["a_scale"], x["W"], ldk, x["w_scale"], _code(B, c["dtype"]), x["bias"], act, x["R"], ldn, x["U"], ldn,
                 x["Y"], ldn, out, x["ws"], x["ws_bytes"], stream=st)
        got = {"Y": x["Y"][:, :N], "U": None if x["U"] is None else x["U"][:, :N]}
        if op == "linear_train":
            B.linear_act_bwd(M, N, x["dY"], ldn, x["U"], ldn, out, act, x["dU"], ldn, x["dbias"], x["ws"], x["ws_bytes"], stream=st)
            got.update(dU=x["dU"][:, :N], dbias=x["dbias"])
        return got
    B.clipped_step(x["list"], c["lr"], c["max_norm"], x["norm"], x["ws"], x["ws_bytes"], stream=st)
    return {"norm": x["norm"], "params": x["params"]}


# ------------------------------------------------------------------ the plain form: 32 bits, one torch operation after another
def _act(u, kind):
    if kind == "relu":
        return torch.where(u > 0, u, 0.0)
    if kind == "gelu":
        return 0.5 * u * (1.0 + torch.erf(u * math.sqrt(0.5)))
    if kind == "silu":
        return u / (1.0 + torch.exp(-u))
    return u


def _act_slope(u, kind):
    if kind == "relu":
        return (u > 0).to(u.dtype)
    if kind == "gelu":
        return 0.5 * (1.0 + torch.erf(u * math.sqrt(0.5))) + u * torch.exp(-0.5 * u * u) * (1.0 / math.sqrt(2.0 * math.pi))
    if kind == "silu":
        s = 1.0 / (1.0 + torch.exp(-u))
        return s * (1.0 + u * (1.0 - s))
    return torch.ones_like(u)


def _run_plain(x):
    c = x["case"]
    op = c["op"]
    if op == "embed":
        return {"out": (x["table"][:, : c["F"]][x["ids"]].float() * c["scale"]).to(x["table"].dtype)}
    if op == "embed_bwd":
        F = c["F"]
        # rows in the order of their ids, running sums in 64 bits, and what they grew by over each run of equal ids
        ids, order = torch.sort(x["ids"], stable=True)
        rows = torch.nn.functional.pad(x["dY"][:, :F][order].double(), (0, 0, 0, -len(ids) % 512)).reshape(-1, 512, F).cumsum(1)
        ends = rows[:, -1]                                       # (512 at a time: one long column keeps few threads busy)
        upto = (rows + (ends.reshape(1, -1, F).cumsum(1)[0] - ends)[:, None]).reshape(-1, F)
        row, count = torch.unique_consecutive(ids, return_counts=True)
        upto = upto[torch.cumsum(count, 0) - 1]
        total = torch.diff(upto, dim=0, prepend=torch.zeros(1, F, dtype=torch.float64, device="cuda"))
        if not c["accumulate"]:
            x["dtable"].zero_()
        x["dtable"][:, :F].index_add_(0, row, (total * c["scale"]).float())
        return {"dtable": x["dtable"][:, :F]}
    if op == "norm":
        F = c["F"]
        h = x["X"][:, :F].float()
        if x["R"] is not None:
            h = h + x["R"][:, :F].float()
        rstd = 1.0 / torch.sqrt((h * h).mean(1) + 1e-6)
        y = h * rstd[:, None]
        if x["w"] is not None:
            y = y * x["w"]
        got = {"H": h.to(x["X"].dtype) if x["R"] is not None else None, "rstd": rstd, "y_scale": None}
        if c["out"] == "e4m3":
            got["Y"], got["y_scale"] = _rows8(y)
        else:
            got["Y"] = y.to(TYPES[c["out"]])
        return got
    if op == "norm_bwd":
        F = c["F"]
        h, dy, r = x["X"][:, :F].float(), x["dY"][:, :F].float(), x["rstd"][:, None]
        xhat = h * r
        g = dy * x["w"] if x["w"] is not None else dy
        dx = r * (g - xhat * (g * xhat).mean(1, keepdim=True))
        if x["dH"] is not None:
            dx = dx + x["dH"][:, :F].float()
        return {"dX": dx.to(x["X"].dtype), "dw": (dy * xhat).sum(0, dtype=torch.float64).float() if x["w"] is not None else None}
    if op in ("linear", "linear_train"):
        N, K, out = c["N"], c["K"], TYPES[c["out"]]
        u = x["A"][:, :K].float() @ x["W"][:, :K].float().t()
        if x["a_scale"] is not None:
            u = u * x["a_scale"][:, None] * x["w_scale"]
        if x["bias"] is not None:
            u = u + x["bias"]
        y = _act(u, c["act"])
        if x["R"] is not None:
            y = y + x["R"][:, :N].float()
        got = {"Y": y.to(out), "U": u.to(out) if c["save"] else None}
        if op == "linear_train":
            du = x["dY"][:, :N].float() * _act_slope(got["U"].float(), c["act"])
            got.update(dU=du.to(out), dbias=du.sum(0, dtype=torch.float64).float())
        return got
    g = x["grads"].float()
    norm = (g * g).sum(dtype=torch.float64).sqrt()
    keep = torch.where(norm > c["max_norm"], c["max_norm"] / norm, 1.0)
    x["params"].copy_((x["params"].float() - (c["lr"] * keep).float() * g).to(x["params"].dtype))
    return {"norm": norm.float().reshape(1), "params": x["params"]}


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    x, op = _inputs(case, seed), case["op"]
    if op == "embed":
        return {"out": torch.index_select(x["table"], 0, x["ids"])[:, : case["F"]].double() * case["scale"]}
    if op == "embed_bwd":
        F, V, n = case["F"], case["V"], case["n"]
        out = x["dtable"][:, :F].double() if case["accumulate"] else torch.zeros(V, F, dtype=torch.float64, device="cuda")
        if V <= 256:                                            # few rows: a product with the rows' indicators, some at a time
            for a in range(0, n, 65_536):
                hit = (x["ids"][a: a + 65_536, None] == torch.arange(V, device="cuda")).double()
                out += case["scale"] * (hit.t().contiguous() @ x["dY"][a: a + 65_536, :F].double())
            return {"dtable": out}
        return {"dtable": out.scatter_add_(0, x["ids"][:, None].expand(n, F), x["dY"][:, :F].double() * case["scale"])}
    if op in ("norm", "norm_bwd"):
        F = case["F"]
        h, w = x["X"][:, :F].double(), torch.ones(F, dtype=torch.float64, device="cuda") if x["w"] is None else x["w"].double()
        if op == "norm":
            h = h if x["R"] is None else h.add_(x["R"][:, :F])
            size = torch.linalg.vector_norm(h, dim=1).square() / F + 1e-6
            y = torch.einsum("nf,f,n->nf", h, w, size ** -0.5)
            got = {"H": h if x["R"] is not None else None, "rstd": size ** -0.5, "Y": y, "y_scale": None}
            if case["out"] == "e4m3":
                got["y_scale"] = torch.maximum(y.max(1)[0], -y.min(1)[0]).clamp(min=TINY) / E4M3_MAX
                got["Y"] = y / got["y_scale"][:, None]
            return got
        r, dy = x["rstd"].double(), x["dY"][:, :F].double()
        along = (dy * w * h).sum(1) * r ** 3 / F               # d/dh of w h r(h), r = (mean h^2 + eps)^-1/2: dr/dh = -r^3 h / F
        dx = dy * w * r[:, None] - h * along[:, None]
        return {"dX": dx if x["dH"] is None else dx + x["dH"][:, :F], "dw": r @ (dy * h) if x["w"] is not None else None}
    if op in ("linear", "linear_train"):
        N, K = case["N"], case["K"]
        A, W = x["A"][:, :K].double(), x["W"][:, :K].double()
        if x["a_scale"] is not None:
            A, W = A * x["a_scale"].double()[:, None], W * x["w_scale"].double()[:, None]
        u = torch.mm(A, W.t().contiguous())
        u = u if x["bias"] is None else u + x["bias"].double()
        normal = torch.distributions.Normal(torch.zeros((), dtype=torch.float64, device="cuda"), torch.ones((), dtype=torch.float64, device="cuda"))
        value = {"none": lambda v: v, "relu": lambda v: v.clamp(min=0.0), "gelu": lambda v: v * normal.cdf(v), "silu": lambda v: v * torch.sigmoid(v)}
        slope = {"none": torch.ones_like, "relu": lambda v: (v > 0).double(), "gelu": lambda v: normal.cdf(v) + v * normal.log_prob(v).exp(),
                 "silu": lambda v: torch.sigmoid(v) + v * torch.sigmoid(v) * torch.sigmoid(-v)}
        y = value[case["act"]](u)
        got = {"Y": y if x["R"] is None else y + x["R"][:, :N].double(), "U": u if case["save"] else None}
        if op == "linear_train":
            # the backward pass is a function of the values kept, which are rounded: theirs are the kept ones here, too
            du = x["dY"][:, :N].double() * slope[case["act"]](u.to(TYPES[case["out"]]).double())
            got.update(dU=du, dbias=du.sum(0))
        return got
    flat = torch.cat([x["grads"][a:b] for a, b in x["at"]]).double()
    norm = torch.linalg.vector_norm(flat)
    rate = case["lr"] * min(1.0, case["max_norm"] / float(norm))
    return {"norm": norm.reshape(1), "params": x["params"].double() - rate * x["grads"].double()}
