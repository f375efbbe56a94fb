"""capgnn_linear in its large tiles (64 to 256 rows and columns, operands straight to LDS) against float64 on the GPU.  Which tile a size takes is
asked of the library's own rule (linear_plan.h, host code alone, compiled by g++), so that a size that a change of the rule sends elsewhere is noticed.

Tolerances as in test_linear.py: K + 12 roundings of the terms' magnitudes, 7 * 2^-13 of the largest of each eight terms for 8-bit operands of a
bf16 result, and the epilogue's operations."""
import os
import subprocess

import numpy as np
import pytest

from paper_2508_13716_amd import binding as B
from tests.row_ops import CODE, EPS, HALF, ttype

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2508_13716_amd", "csrc")
BYTES = {"f32": 4, "bf16": 2, "e4m3": 1}

PROGRAM = r"""
#include "linear_plan.h"
#include <cstdio>
#include <cstdlib>
using namespace capgnn;
int main(int argc, char **argv) {
    for (int i = 1; i + 4 < argc; i += 5) {
        const int64_t M = atoll(argv[i]), N = atoll(argv[i + 1]), K = atoll(argv[i + 2]);
        const int es = atoi(argv[i + 3]);
        const LinearPlan p = linear_plan(M, N, K, es);
        const LinearWay w = linear_way(p, M, N, K, es, atoi(argv[i + 4]) != 0);
        std::printf("%d %d %d %d %d %lld\n", w.tile, int(w.direct), int(w.cut), p.parts, w.waves, static_cast<long long>(p.part_k));
    }
}
"""


@pytest.fixture(scope="module")
def ways(tmp_path_factory):
    """(M, N, K, type, rows start on 4 bytes) of each -> (tile, straight to LDS, in three pieces, parts, waves, k of a part)"""
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-I", CSRC, "-o", str(d / "plan"), str(d / "plan.cpp")], check=True)

    def ask(sizes):
        done = subprocess.run([str(d / "plan"), *[str(x) for M, N, K, t, a in sizes for x in (M, N, K, BYTES[t], int(a))]], check=True, capture_output=True, text=True)
        return [tuple(int(x) for x in line.split()) for line in done.stdout.splitlines()]
    return ask


# size, type, and the tile that it is here for.  Reductions of whole steps and with a rest; rows and columns that end inside a tile, and one that does not
LARGE = [(3700, 3690, 1000, "bf16", 256), (3700, 3690, 1024, "bf16", 256), (3584, 3840, 1030, "bf16", 256), (3600, 3700, 521, "f32", 256), (3600, 3700, 544, "f32", 256),
         (3650, 3600, 4000, "e4m3", 256), (3650, 3603, 4096, "e4m3", 256), (2100, 2090, 516, "e4m3", 128), (2100, 2090, 768, "e4m3", 128), (2100, 2090, 300, "bf16", 128),
         (2100, 2090, 256, "bf16", 128), (2100, 2090, 200, "f32", 128), (1300, 1300, 320, "bf16", 64), (1300, 1300, 516, "e4m3", 64)]


def test_sizes_take_the_tiles_they_are_here_for(ways):
    got = ways([(M, N, K, t, True) for M, N, K, t, _ in LARGE])
    for (M, N, K, t, tile), w in zip(LARGE, got):
        assert w[0] == tile and w[1] == 1 and w[2] == (t == "f32") and w[3] == 1, (M, N, K, t, w)
    # a pitch that is no multiple of 4 bytes: tiles of 64 through registers
    assert all(w[:3] == (64, 0, 0) for w in ways([(M, N, K, t, False) for M, N, K, t, _ in LARGE]))


def test_a_few_rows_by_many_results_are_fewer_threads_than_a_launch_has(ways):
    sizes = [(M, N, K, t, True) for M in (1, 16) for N in (1, (1 << 25) + 1, (1 << 26) - 16, (1 << 26) - 15, 1 << 26) for K in (1, 1000, 4096) for t in BYTES]
    for (M, N, K, t, _), w in zip(sizes, ways(sizes)):
        assert w[0] == 0 and 1 <= w[4] <= 16 and -(-N // 16) * w[4] * 64 < 1 << 32, (M, N, K, t, w)


def act(kind, u):
    import torch
    if kind == "gelu":
        return 0.5 * u * (1 + torch.erf(u / 2 ** 0.5))
    if kind == "silu":
        return u / (1 + torch.exp(-u))
    return torch.where(u <= 0, 0.0, u) if kind == "relu" else u


def matrix(rows, cols, ld, offset, t, g, scale=1.0):
    """[rows x cols] at pitch ld, `offset` elements into its allocation, NaN in the padding"""
    import torch
    flat = torch.full((rows * ld + offset,), float("nan"), device="cuda").to(ttype(t))
    view = flat[offset:].view(rows, ld)
    view[:, :cols] = (torch.randn(rows, cols, generator=g, device="cuda") * scale).to(ttype(t))
    return flat, view[:, :cols]


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K,t,tile", LARGE)
@pytest.mark.parametrize("to", ["f32", "bf16"])
@pytest.mark.parametrize("kind,residual,save,pad", [("none", False, False, 0), ("gelu", True, True, 8), ("silu", True, False, 4), ("relu", False, True, 0)])
def test_large_tiles(M, N, K, t, tile, to, kind, residual, save, pad):
    import torch
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    ldk, ldn, code = K + pad, N + pad, {"none": B.ACT_NONE, "relu": B.ACT_RELU, "gelu": B.ACT_GELU, "silu": B.ACT_SILU}[kind]
    if t == "e4m3":
        ldk = -(-ldk // 4) * 4
    if t == "bf16":
        ldk = -(-ldk // 2) * 2
    aflat, a = matrix(M, K, ldk, 4 if pad else 0, t, g)
    wflat, w = matrix(N, K, ldk, 8 if pad else 0, t, g, 1.0 if t == "e4m3" else K ** -0.5)
    a64, w64 = a.double(), w.double().t().contiguous()
    sums, mass = a64 @ w64, a64.abs() @ w64.abs()
    dropped = torch.zeros((), dtype=torch.float64, device="cuda")
    if t == "e4m3" and to == "bf16":                 # (the largest of eight products is at most the product of the largest)
        most = lambda x: torch.nn.functional.pad(x.abs(), (0, -K % 8)).reshape(x.shape[0], -1, 8).amax(2)
        dropped = 7 * 2.0 ** -13 * (most(a64) @ most(w64.t()).t().contiguous())
    sa = sw = None
    if t == "e4m3":
        sa, sw = torch.exp(torch.randn(M, generator=g, device="cuda")), torch.exp(torch.randn(N, generator=g, device="cuda")) * K ** -0.5
        both = sa.double()[:, None] * sw.double()
        sums, mass, dropped = sums * both, mass * both, dropped * both
    bias = torch.randn(N, generator=g, device="cuda")
    rflat, r = matrix(M, N, ldn, 1, to, g) if residual else (None, None)
    yflat, y = matrix(M, N, ldn, 3 if pad else 0, to, g)
    uflat, u = matrix(M, N, ldn, 1 if pad else 0, to, g) if save else (None, None)
    at = lambda flat, view: None if view is None else view.data_ptr()
    size = B.linear_workspace_bytes(M, N, K, CODE[t])
    ws = torch.empty(max(size, 256), dtype=torch.uint8, device="cuda")

    def run():
        B.linear(M, N, K, at(aflat, a), ldk, sa, at(wflat, w), ldk, sw, CODE[t], bias, code, at(rflat, r), ldn, at(uflat, u), ldn, at(yflat, y), ldn, CODE[to], ws, size)
    run()
    torch.cuda.synchronize()
    want_u = sums + bias.double()
    u_err = (mass * (K + 12) * EPS + dropped + 2 * EPS * want_u.abs() + 1e-36) * 1.001
    want = act(kind, want_u)
    if residual:
        want = want + r.double()
    err = 1.13 * u_err + 8 * EPS * want_u.abs() + (2 * EPS + HALF[to]) * 1.001 * want.abs()
    for got, value, tol, what in ((y, want, err, "Y"),) + (((u, want_u, u_err + HALF[to] * 1.001 * want_u.abs(), "U"),) if save else ()):
        off = (got.double() - value).abs() - tol
        assert bool(torch.isfinite(got.double()).all()) and float(off.max()) <= 0, f"{what}: {float(off.max()):.3g} beyond the tolerance, {int((off > 0).sum())} of {off.numel()}"
    if pad:
        pads = yflat[3:].view(M, ldn)[:, N:].double()
        assert bool(torch.isnan(pads).all()) and bool(torch.isnan(yflat[:3].double()).all())
    first = yflat.view(torch.uint8).clone()
    for _ in range(3):                               # the same bits every time
        y.zero_()
        run()
    torch.cuda.synchronize()
    assert torch.equal(first, yflat.view(torch.uint8))
