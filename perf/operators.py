"""What a classifier answers with and what it learns from a teacher, as timed cases: log-probabilities of given classes with
entropy and the most likely classes, the gradient of those, and distillation from a teacher's top logits with its gradient.

Logits are [n x C] rows of one vertex (or token) each.  The class counts go from the vertex classifiers of
``paper_2508_13716_amd/synth.py`` (8, 41, 47 classes) to output layers over a whole vocabulary.
"""
from __future__ import annotations

import math

import torch

own = False

LOGITS = {"f32": torch.float32, "bf16": torch.bfloat16}


def _case(op, name=None, **kw):
    c = dict(op=op, n=1, C=2, pad=0, dtype="f32", temp=1.0, mask=1.0, barred=0.0, m=1, k=0, entropy=True, rest=False)
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one row of a large output layer while serving: the sampled class's log-probability and 20 alternatives
        _case("logprobs", "answer_one_row", n=1, C=40_000, temp=0.7, k=20),
        # the answers of a trained vertex classifier on its partition (47 classes): latency does not count, memory does
        _case("logprobs", "answer_vertices", n=612_000, C=47, k=5),
        # a padded batch: pitch not a multiple of anything, a tenth of the classes barred, three candidates per row
        _case("logprobs", "answer_ragged", n=3_001, C=10_007, pad=5, dtype="bf16", mask=0.8, barred=0.1, m=3, k=10),
        # a teacher's pass over a training batch: 64 classes per row kept for its students
        _case("logprobs", "answer_teacher", n=4_096, C=131_072, dtype="bf16", k=64),
        # the last layer's gradient when vertices' log-probabilities are weighted and their entropy is rewarded (41 classes)
        _case("logprobs_bwd", "grad_vertices", n=60_000, C=41, mask=0.5),
        # a few long rows, several classes given in each
        _case("logprobs_bwd", "grad_few_rows", n=8, C=100_003, m=4, temp=0.7),
        # a policy step over a large output layer
        _case("logprobs_bwd", "grad_large", n=4_096, C=65_536, dtype="bf16"),
        # the smallest evaluation graph (4096 vertices, 8 classes) learning from a teacher: launches and latency
        _case("distill", "distill_tiny", n=4_096, C=8, k=4, temp=2.0),
        # a partition's vertices, half of them in the loss
        _case("distill", "distill_vertices", n=612_000, C=47, k=8, temp=2.0, mask=0.5),
        # odd sizes, padded rows, the teacher's remaining probability as one more outcome
        _case("distill", "distill_ragged", n=2_999, C=10_007, pad=5, k=32, rest=True, barred=0.1),
        # a student's training batch over a large output layer, in bf16 ...
        _case("distill", "distill_large", n=8_192, C=64_000, dtype="bf16", k=64, temp=2.0),
        # ... and in fp32 with the remaining probability
        _case("distill", "distill_long_rows", n=2_048, C=131_072, k=64, rest=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["logprobs", "logprobs_bwd", "distill"])
    C = _log_int(rng, 2, 200_000)
    n = _log_int(rng, 1, max(1, min(2_450_000, 2_000 * 131_072 // C)))
    return _case(op, n=n, C=C, pad=rng.choice([0, 0, 0, 1, 8, rng.randint(1, 31)]), dtype=rng.choice(["f32", "bf16"]),
                 temp=rng.choice([1.0, 1.0, 2.0, round(rng.uniform(0.5, 4.0), 2)]), mask=rng.choice([1.0, 1.0, 0.5, 0.9]),
                 barred=rng.choice([0.0, 0.0, 0.1]) if C > 8 else 0.0, m=rng.choice([1, 1, 2, rng.randint(1, 16)]),
                 k=min(C, rng.choice([1, 5, 8, 20, 64, rng.randint(1, 64)])), entropy=rng.random() < 0.7, rest=rng.random() < 0.5)


def work(case):
    n, C, es = case["n"], case["C"], 2 if case["dtype"] == "bf16" else 4
    m, k = case["m"], case["k"]
    on = case["mask"]
    mask = n if on < 1.0 else 0
    if case["op"] == "logprobs":       # outputs of every row, logits of the masked-in ones
        return {"bytes": n * on * C * es + mask + n * (8 * m + 12 + 8 * k), "flops": n * on * C * 4}
    if case["op"] == "logprobs_bwd":
        return {"bytes": n * on * C * es + n * C * es + mask + n * (8 * m + 8 + (8 if case["entropy"] else 0)), "flops": n * on * C * 6}
    return {"bytes": n * on * C * es + n * C * es + mask + n * (8 * k + 4), "flops": n * on * C * 6}


# ------------------------------------------------------------------ inputs
def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, C, ld, dt = case["n"], case["C"], case["C"] + case["pad"], LOGITS[case["dtype"]]
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")
    # logits as a trained output layer gives them: a spread of 2 and a class or two well above
    base = rand(n, ld).mul_(2.0)
    best = torch.randint(0, C, (n, 1), generator=g, device="cuda")
    base.scatter_add_(1, best, 6.0 + 2.0 * rand(n, 1))
    x = {"case": case}
    if case["op"] == "distill":         # the teacher: the same rows seen a little differently, its k best classes kept
        teacher = base[:, :C] + rand(n, C)
        if case["barred"]:
            teacher[:, : int(C * case["barred"])] = -math.inf
        val, ids = torch.topk(teacher, case["k"], dim=1)
        if case["rest"]:                # as log-probabilities at the temperature of the loss
            val = val / case["temp"] - torch.logsumexp(teacher / case["temp"], 1, keepdim=True)
        x["t_ids"], x["t_val"] = ids.to(torch.int32).contiguous(), val.float().contiguous()
        del teacher
    else:
        ids = torch.randint(0, C, (n, case["m"]), generator=g, device="cuda", dtype=torch.int32)
        ids[:, :1] = torch.where(rand(n, 1) > 0, best.to(torch.int32), ids[:, :1])
        ids[:, 1:][rand(n, case["m"] - 1) > 1.0] = -1          # rows with fewer candidates than columns
        x["ids"] = ids
    if case["barred"]:
        base[:, : int(C * case["barred"])] = -math.inf
    x["Z"] = base.to(dt)
    x["mask"] = (torch.rand(n, generator=g, device="cuda") < case["mask"]).to(torch.uint8) if case["mask"] < 1.0 else None
    if case["op"] == "logprobs_bwd":
        x["dlogp"] = rand(n, case["m"]) / n
        x["dent"] = rand(n).mul_(0.01).add_(0.02) / n if case["entropy"] else None
    return x


def prepare(case, seed):
    x = _inputs(case, seed)
    n, C, dt = case["n"], case["C"], LOGITS[case["dtype"]]
    ld, new = C + case["pad"], lambda *s, t=torch.float32: torch.zeros(s, dtype=t, device="cuda")
    if case["op"] == "logprobs":
        x.update(logp=new(n, case["m"]), ent=new(n), stats=new(n, 2), top=new(n, case["k"], t=torch.int32), top_logp=new(n, case["k"]))
    elif case["op"] == "logprobs_bwd":      # what the forward pass of the same rows left
        d, lse, top = _plain_rows(x)
        x["stats"] = torch.cat([top, lse], 1).contiguous()
        x["ent"] = _plain_entropy(d, lse).contiguous()
        x["dZ"] = new(n, ld, t=dt)
        del d
    else:
        x.update(loss=new(1), row_loss=new(n), dZ=new(n, ld, t=dt))
    if own:
        from paper_2508_13716_amd import binding as B
        size = (B.logprobs_workspace_bytes(n, C, case["k"]) if case["op"] == "logprobs" else
                B.distill_workspace_bytes(n, C) if case["op"] == "distill" else 0)
        x["ws"] = torch.empty(max(size, 256), dtype=torch.uint8, device="cuda")
        x["ws_bytes"] = size
    return x


def run(x):
    return _run_own(x) if own else _run_plain(x)


# ------------------------------------------------------------------ the framework's calls
def _run_own(x):
    from paper_2508_13716_amd import binding as B
    c = x["case"]
    n, C, Z, T = c["n"], c["C"], x["Z"], c["temp"]
    ld, dt, st = C + c["pad"], B.BF16 if c["dtype"] == "bf16" else B.F32, torch.cuda.current_stream()
    if c["op"] == "logprobs":
        B.logprobs(n, C, Z, ld, dt, T, x["mask"], x["ids"], c["m"], c["m"], x["logp"], c["m"], x["ent"], x["stats"], c["k"],
                   x["top"], x["top_logp"], c["k"], x["ws"], x["ws_bytes"], stream=st)
        return {"logp": x["logp"], "entropy": x["ent"], "stats": x["stats"], "top": x["top"], "top_logp": x["top_logp"]}
    if c["op"] == "logprobs_bwd":
        B.logprobs_bwd(n, C, Z, ld, dt, T, x["mask"], x["stats"], x["ent"], x["ids"], c["m"], c["m"], x["dlogp"], c["m"], x["dent"],
                       x["dZ"], ld, dt, stream=st)
        return {"dZ": x["dZ"][:, :C]}
    B.distill(n, C, Z, ld, dt, x["t_ids"], x["t_val"], c["k"], c["k"], int(c["rest"]), T, x["mask"], 0.0, T * T, x["loss"],
              x["row_loss"], x["dZ"], ld, dt, 0, x["ws"], x["ws_bytes"], stream=st)
    return {"loss": x["loss"], "row_loss": x["row_loss"], "dZ": x["dZ"][:, :C]}


# ------------------------------------------------------------------ the plain form: 32 bits, one torch operation after another
def _plain_rows(x):
    """(z - max) / T, ln of the sum of their exponentials, max"""
    c = x["case"]
    z = x["Z"][:, : c["C"]].float()
    top = z.amax(1, keepdim=True)
    d = (z - top) / c["temp"]
    return d, d.exp().sum(1, keepdim=True).log(), top


def _plain_entropy(d, lse):
    e = d.exp()
    return (lse[:, 0] - torch.where(e > 0, e * d, 0.0).sum(1) / e.sum(1))


def _given(ids, C):
    ok = (ids >= 0) & (ids < C)
    return ok, ids.clamp(0, C - 1).long()


def _run_plain(x):
    c = x["case"]
    n, C, T = c["n"], c["C"], c["temp"]
    on = x["mask"].bool()[:, None] if x["mask"] is not None else torch.ones(n, 1, dtype=torch.bool, device="cuda")
    if c["op"] == "logprobs":
        d, lse, top = _plain_rows(x)
        ok, at = _given(x["ids"], C)
        logp = torch.where(ok & on, d.gather(1, at) - lse, 0.0)
        ent = torch.where(on[:, 0], _plain_entropy(d, lse), 0.0)
        stats = torch.where(on, torch.cat([top, lse], 1), 0.0)
        # the k largest, ties to the lowest class: an integer that orders (logit, -class)
        bits = (x["Z"][:, :C].float() + 0.0).view(torch.int32)
        key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() * (1 << 32) + (0xFFFFFFFF - torch.arange(C, device="cuda"))
        best = 0xFFFFFFFF - (torch.topk(key, c["k"], dim=1)[0] & 0xFFFFFFFF)
        return {"logp": logp, "entropy": ent, "stats": stats, "top": torch.where(on, best, -1).int(),
                "top_logp": torch.where(on, d.gather(1, best) - lse, 0.0)}
    if c["op"] == "logprobs_bwd":
        d = (x["Z"][:, :C].float() - x["stats"][:, :1]) / T - x["stats"][:, 1:]
        p = d.exp()
        ok, at = _given(x["ids"], C)
        g = torch.where(ok, x["dlogp"], 0.0)
        dz = -p * g.sum(1, keepdim=True)
        if x["dent"] is not None:
            dz -= torch.where(p > 0, p * (d + x["ent"][:, None]), 0.0) * x["dent"][:, None]
        dz.scatter_add_(1, at, g)
        return {"dZ": torch.where(on, dz / T, 0.0).to(x["Z"].dtype)}
    d, lse, _ = _plain_rows(x)
    p = (d - lse).exp()
    at, v = x["t_ids"].long(), x["t_val"].double()      # (what is left of 1 in 64 bits: it is the small difference of numbers near 1)
    if c["rest"]:
        q = v.exp()
        r = 1.0 - q.sum(1, keepdim=True)
        r = torch.where(r < 2.0 ** -20, 0.0, r)
        away = p.scatter(1, at, 0.0)
        P = away.sum(1, keepdim=True).double()
        share = torch.where(r > 0, r / P, 0.0).float()
        last = torch.where(r > 0, r * (r.log() - P.log()), 0.0)
        mass = (q.sum(1, keepdim=True) + r).float()
    else:
        e = ((v - v.amax(1, keepdim=True)) / T).exp()
        q = e / e.sum(1, keepdim=True)
        away, share, last, mass = None, 0.0, 0.0, 1.0
    row = torch.where(q > 0, q * (q.log() - (d.gather(1, at) - lse)), 0.0).sum(1, keepdim=True) + last
    row, q = torch.where(on, row, 0.0).float(), q.float()
    dz = p * mass if away is None else p * mass - away * share
    dz.scatter_add_(1, at, -q)
    count = on.sum().clamp(min=1)
    return {"loss": (row.sum() * (T * T) / count).reshape(1), "row_loss": row[:, 0],
            "dZ": torch.where(on, dz * (T / count), 0.0).to(x["Z"].dtype)}


# ------------------------------------------------------------------ the definition in 64 bits, some rows at a time
def exact(case, seed):
    x = _inputs(case, seed)
    n, C, T, op = case["n"], case["C"], float(case["temp"]), case["op"]
    live = torch.ones(n, dtype=torch.bool, device="cuda") if x["mask"] is None else x["mask"] != 0
    norm = max(int(live.sum()), 1)
    step = max(1, (1 << 26) // C)
    out = []
    for a in range(0, n, step):
        rows = slice(a, min(n, a + step))
        z = x["Z"][rows, :C].double()
        on = live[rows]
        s = z / T
        lse = torch.logsumexp(s, 1)
        lp = s - lse[:, None]
        p = lp.exp()
        plogp = torch.nan_to_num(p * lp, nan=0.0)
        if op == "logprobs":
            ids = x["ids"][rows].long()
            inside = (ids >= 0) & (ids < C)
            logp = torch.take_along_dim(lp, torch.where(inside, ids, 0), 1)
            order = torch.sort(z, dim=1, descending=True, stable=True)[1][:, : case["k"]]
            zmax = z.max(1)[0]
            out.append({"logp": logp.masked_fill(~inside | ~on[:, None], 0.0), "entropy": (-plogp.sum(1)).masked_fill(~on, 0.0),
                        "stats": torch.stack([zmax, lse - zmax / T], 1).masked_fill(~on[:, None], 0.0),
                        "top": order.masked_fill(~on[:, None], -1).int(),
                        "top_logp": torch.take_along_dim(lp, order, 1).masked_fill(~on[:, None], 0.0)})
        elif op == "logprobs_bwd":
            ids, g = x["ids"][rows].long(), x["dlogp"][rows].double()
            dz = torch.zeros_like(z)
            for b in range(ids.shape[1]):
                inside = ((ids[:, b] >= 0) & (ids[:, b] < C)).double()
                dz.sub_(p * (g[:, b] * inside)[:, None])
                dz[torch.arange(len(z), device="cuda"), ids[:, b].clamp(0, C - 1)] += g[:, b] * inside
            if x["dent"] is not None:
                dz.sub_((plogp - p * plogp.sum(1, keepdim=True)) * x["dent"][rows].double()[:, None])
            out.append({"dZ": (dz / T).masked_fill(~on[:, None], 0.0)})
        else:
            ids, v = x["t_ids"][rows].long(), x["t_val"][rows].double()
            target = torch.zeros_like(z)
            target.scatter_(1, ids, v.exp() if case["rest"] else torch.softmax(v / T, 1))
            kl = torch.where(target > 0, target * (target.log() - lp), 0.0).sum(1)
            grad = p * target.sum(1, keepdim=True) - target
            if case["rest"]:
                r = (1.0 - target.sum(1)).clamp(min=0.0)
                r[r < 2.0 ** -20] = 0.0
                others = p.scatter(1, ids, 0.0)
                P = others.sum(1)
                kl += torch.where(r > 0, r * (r / P).log(), 0.0)
                grad += r[:, None] * p - torch.where(r > 0, r / P, 0.0)[:, None] * others
            out.append({"row_loss": kl.masked_fill(~on, 0.0), "dZ": (grad * (T / norm)).masked_fill(~on[:, None], 0.0)})
    whole = {key: torch.cat([o[key] for o in out]) for key in out[0]}
    if op == "distill":
        whole = {"loss": (whole["row_loss"].sum() * T * T / norm).reshape(1), **whole}
    return whole
