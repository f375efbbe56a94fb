"""What the tests of the row-wise operators and products share: device matrices at any pitch, roundings, captured graphs.

EPS = 2^-24 is one float rounding, HALF[t] half a step of a type relative to the value (nearest rounding's error)."""
from collections import deque

import numpy as np
import pytest

from paper_2508_13716_amd import binding as B

EPS = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "e4m3": 2.0 ** -4}
CODE = {"f32": B.F32, "bf16": B.BF16, "e4m3": B.E4M3}
FAKE = 1 << 20          # an address that nothing reads


def ttype(t):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}[t]


def refuse(code, f, *a, **k):
    with pytest.raises(B.CapgnnError) as e:
        f(*a, **k)
    assert e.value.code == code, e.value


def held(x, t):
    """float64 values of x as the type holds them"""
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).to(ttype(t)).double().numpy()


_alive = deque(maxlen=32)       # a call takes addresses: what a test makes for one inside its argument list stays until it has run


class Mat:
    """[n x cols] on the GPU at pitch ld, `offset` elements into its allocation; the padding holds a pattern that must stay."""

    def __init__(self, x, t, ld=None, offset=0, shape=None):
        import torch
        n, cols = shape if x is None else x.shape
        self.t, self.n, self.cols, self.ld = t, n, cols, cols if ld is None else ld
        raw = {"f32": torch.int32, "bf16": torch.int16, "e4m3": torch.uint8}[t]
        mark = {"f32": 0x7FC12345, "bf16": 0x7FC1, "e4m3": 0x7F}[t]     # NaN in every type
        self.bits = torch.full((n * self.ld + offset + 3,), mark, dtype=raw, device="cuda")
        self.mark, self.offset = mark, offset
        _alive.append(self.bits)
        self.flat = self.bits.view(ttype(t))
        self.view = self.flat[offset: offset + n * self.ld].view(n, self.ld)
        if x is not None and x.size:
            self.view[:, :cols] = torch.from_numpy(np.ascontiguousarray(x)).to(ttype(t)).cuda()

    @property
    def p(self):
        return self.bits.data_ptr() + self.offset * self.bits.element_size()

    def get(self):
        """float64 values; what is no part of the matrix has to be as it was"""
        a = self.bits.cpu()
        assert (a[: self.offset] == self.mark).all() and (a[self.offset + self.n * self.ld:] == self.mark).all(), "written outside the matrix"
        inner = a[self.offset: self.offset + self.n * self.ld].view(self.n, self.ld)
        assert (inner[:, self.cols:] == self.mark).all(), "padding written"
        return inner.view(ttype(self.t))[:, : self.cols].double().numpy()

    def raw(self):
        return self.bits.cpu().clone()


def vec(x, t="f32"):
    return None if x is None else Mat(np.asarray(x).reshape(1, -1), t)


def new(n, cols, t, ld=None, offset=0):
    return Mat(None, t, ld, offset, (n, cols))


def p(m):
    return None if m is None else m.p


def ws_of(size):
    import torch
    ws = torch.empty(max(size, 256), dtype=torch.uint8, device="cuda")
    _alive.append(ws)
    return ws, size


def close(got, want, tol, what=""):
    got, want, tol = np.asarray(got, np.float64), np.asarray(want, np.float64), np.broadcast_to(np.asarray(tol, np.float64), np.shape(want))
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaN elsewhere"
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), f"{what}: infinities differ"
    off = np.abs(got - want)[fine] - tol[fine]
    assert not off.size or off.max() <= 0, f"{what}: {off.max():.3g} beyond the tolerance, {int((off > 0).sum())} of {off.size}"


def replayed(run, read, times=3):
    """run() recorded once and replayed with work of the program's own between: every replay gives what the eager call gave (bits)."""
    import torch
    run(torch.cuda.current_stream())
    torch.cuda.synchronize()
    want = read()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(torch.cuda.current_stream())
    for _ in range(times):
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(read(), want):
            assert torch.equal(a, b)
        torch.ones(1000, device="cuda").sum().item()
        run(torch.cuda.current_stream())
        torch.cuda.synchronize()
        for a, b in zip(read(), want):
            assert torch.equal(a, b)
