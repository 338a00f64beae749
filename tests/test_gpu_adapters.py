"""gptq2d_adapters and its gradients against the formulas in 64 bits.

Tolerances. u = 2^-24. A result is (or is a rounding of) a sum in 32 bits of exact
products: n terms in any order are off by at most n u times the sum of magnitudes, and
typically by far less. What bounds a test is n u sum |terms|, with n = the length of the
sum (a matrix instruction adds several terms at once, which only shortens it), plus 2^-23
for numbers held as two or three 16-bit ones, plus half a step of the output type."""
import math

import pytest
import torch

import serving
from paper_2607_27042_amd import binding as g

pytestmark = pytest.mark.gpu

HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
# of h and p where the instruction takes them as the sum of two 16-bit numbers: bf16 twice 8 bits, of which the
# first is cut off, f16 twice 11 bits relative to the row's largest
HELD = {"f32": 0.0, "f16": 2.0 ** -21, "bf16": 2.0 ** -16}


def gen(seed):
    r = torch.Generator(device="cuda")
    r.manual_seed(seed)
    return r


class Problem:
    def __init__(self, M, N, K, R, count, dtype, seed=0, pad=0, index=None, scales=True):
        r = gen(seed)
        dt = serving.DTYPE[dtype]

        def mat(rows, cols, size=1.0):
            t = torch.full((rows, cols + pad), math.nan, device="cuda", dtype=dt)
            t[:, pad // 2:pad // 2 + cols] = (size * torch.randn(rows, cols, generator=r, device="cuda")).to(dt)
            return t[:, pad // 2:pad // 2 + cols]

        self.shape, self.dtype, self.dt = (M, N, K, R, count), dtype, dt
        self.X, self.Y, self.G, self.D = mat(M, K), mat(M, N), mat(M, N, 0.1), mat(M, K, 0.1)
        a, b = mat(count * R, K, K ** -0.5), mat(count * N, R, R ** -0.5)
        three = lambda t, n: t.as_strided((count, n, t.shape[1]), (n * t.stride(0), t.stride(0), 1))
        self.A, self.B = three(a, R), three(b, N)
        self.scales = torch.rand(count, generator=r, device="cuda") + 0.5 if scales else None
        if index is None:
            index = torch.randint(-1, count + 1, (M,), generator=r, device="cuda")
        self.index = index.to(torch.int32)
        self.groups = torch.full((g.gptq2d_adapter_groups_size(M, count),), -99, dtype=torch.int32, device="cuda")
        g.gptq2d_adapter_groups(self.index, count, self.groups)

    def space(self, size):
        return torch.full((max(size, 256),), 0xff, dtype=torch.uint8, device="cuda")  # NaN everywhere

    def forward(self, out=None, want_h=True, Y=True):
        M, N, K, R, count = self.shape
        O = torch.full((M, N), math.nan, device="cuda", dtype=self.dt) if out is None else out
        H = torch.full((M, R), math.nan, device="cuda") if want_h else None
        g.gptq2d_adapters(self.X, self.A, self.B, self.scales, self.groups, self.Y if Y else None, O, H,
                          self.space(g.gptq2d_adapters_workspace_size(*self.shape)))
        return O, H

    def backward(self, H, D=True, wants=(True, True, True), out=None):
        M, N, K, R, count = self.shape
        dX = (torch.full((M, K), math.nan, device="cuda", dtype=self.dt) if out is None else out) if wants[0] else None
        dA = torch.full((count, R, K), math.nan, device="cuda") if wants[1] else None
        dB = torch.full((count, N, R), math.nan, device="cuda") if wants[2] else None
        g.gptq2d_adapters_backward(self.G, self.X, self.A, self.B, self.scales, self.groups, H, self.D if D else None, dX, dA,
                                   dB, self.space(g.gptq2d_adapters_backward_workspace_size(*self.shape)))
        return dX, dA, dB

    def rows(self):
        """Of each adapter: its number, rows, weights and scale in 64 bits."""
        for a in range(self.shape[4]):
            at = (self.index == a).nonzero()[:, 0]
            yield a, at, self.A[a].double(), self.B[a].double(), 1.0 if self.scales is None else float(self.scales[a])

    def check_forward(self, O, H, Y=True):
        M, N, K, R, count = self.shape
        o = self.Y.double().clone() if Y else torch.zeros(M, N, dtype=torch.float64, device="cuda")
        h = torch.zeros(M, R, dtype=torch.float64, device="cuda")
        h_off, off = torch.zeros_like(h), torch.zeros_like(o)
        for a, at, A, B, s in self.rows():
            x = self.X[at].double()
            h[at] = torch.matmul(x, A.T)
            h_off[at] = 2.0 ** -24 * (K + 20) * torch.matmul(x.abs(), A.T.abs())
            o[at] += s * torch.matmul(h[at], B.T)
            far = h_off[at] + (HELD[self.dtype] + 2.0 ** -24 * (2 * R + 4)) * h[at].abs().amax(1, keepdim=True)
            off[at] += s * torch.matmul(far, B.T.abs())
        if H is not None:
            assert bool(((H.double() - h).abs() <= h_off).all())
        none = (self.index < 0) | (self.index >= count)
        assert torch.equal(O[none], self.Y[none] if Y else torch.zeros_like(O[none]))
        off += (off + o.abs()) * (HALF[self.dtype] + 2.0 ** -23) + 1e-30
        if self.dtype == "f16":
            off += 2.0 ** -25
        bad = (O.double() - o).abs() > off
        assert not bool(bad.any()), ((O.double() - o).abs() / off).max()

    def check_backward(self, H, dX, dA, dB, D=True):
        M, N, K, R, count = self.shape
        dx = self.D.double().clone() if D else torch.zeros(M, K, dtype=torch.float64, device="cuda")
        off = torch.zeros_like(dx)
        u = 2.0 ** -24
        for a, at, A, B, s in self.rows():
            x, gr = self.X[at].double(), self.G[at].double()
            p = s * torch.matmul(gr, B)
            p_off = u * (N + 24) * s * torch.matmul(gr.abs(), B.abs())
            dx[at] += torch.matmul(p, A)
            far = p_off + (HELD[self.dtype] + u * (2 * R + 4)) * p.abs().amax(1, keepdim=True) if len(at) else p_off
            off[at] += torch.matmul(far, A.abs())
            n = len(at) + 24
            if dA is not None:
                top = p.abs().amax(0, keepdim=True).expand_as(p) if len(at) else p
                bound = torch.matmul((p_off + u * n * p.abs() + 2.0 ** -21 * (self.dtype == "f16") * top).T, x.abs()) + 1e-30
                assert bool(((dA[a].double() - torch.matmul(p.T, x)).abs() <= bound).all())
            if dB is not None:
                h = H[at].double()
                top = h.abs().amax(0, keepdim=True).expand_as(h) if len(at) else h
                bound = s * torch.matmul(gr.abs().T, u * n * h.abs() + 2.0 ** -21 * (self.dtype == "f16") * top) + 1e-30
                assert bool(((dB[a].double() - s * torch.matmul(gr.T, h)).abs() <= bound).all())
        if dX is not None:
            none = (self.index < 0) | (self.index >= count)
            assert torch.equal(dX[none], self.D[none] if D else torch.zeros_like(dX[none]))
            off += (off + dx.abs()) * (HALF[self.dtype] + 2.0 ** -23) + 1e-30
            if self.dtype == "f16":
                off += 2.0 ** -25
            assert bool(((dX.double() - dx).abs() <= off).all()), ((dX.double() - dx).abs() / off).max()

    def check(self, **k):
        O, H = self.forward()
        self.check_forward(O, H)
        self.check_backward(H, *self.backward(H))


@pytest.mark.parametrize("M,count", [(0, 3), (1, 1), (7, 4096), (255, 2), (4096, 1), (4097, 33), (20000, 5)])
def test_groups(M, count):
    index = torch.randint(-2, count + 2, (M,), generator=gen(M), device="cuda", dtype=torch.int32)
    out = torch.full((g.gptq2d_adapter_groups_size(M, count) + 1,), -9, dtype=torch.int32, device="cuda")
    g.gptq2d_adapter_groups(index, count, out[:-1])
    key = torch.where((index < 0) | (index >= count), count, index)
    order = torch.argsort(key, stable=True)
    start = torch.searchsorted(key[order], torch.arange(count + 1, device="cuda", dtype=torch.int32))
    assert torch.equal(out[:M], order.int()) and torch.equal(out[M:2 * M], key[order].int())
    assert torch.equal(out[2 * M:2 * M + count + 1], start.int()) and out[2 * M + count + 1:].tolist() == [M, -9]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,N,K,R,count", [(1, 1, 1, 1, 1), (1, 64, 128, 16, 3), (5, 300, 200, 8, 7), (16, 257, 33, 20, 2),
                                           (64, 512, 1024, 16, 48), (100, 1000, 700, 33, 3), (130, 128, 4096, 64, 2),
                                           (333, 96, 520, 128, 5), (70, 1031, 264, 100, 9)])
def test_few_rows(M, N, K, R, count, dtype):
    Problem(M, N, K, R, count, dtype, seed=M + R).check()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,N,K,R,count", [(2100, 264, 512, 16, 3), (2049, 520, 136, 32, 20), (3001, 128, 264, 64, 4),
                                           (2500, 200, 328, 128, 2), (2100, 301, 123, 12, 40)])
def test_many_rows(M, N, K, R, count, dtype):
    # requests behind one another, some of a few rows
    n = M // 60
    index = torch.randint(-1, count, (n,), generator=gen(M), device="cuda").repeat_interleave(61)[:M]
    index = torch.cat([index, torch.zeros(M - len(index), dtype=index.dtype, device="cuda")])
    Problem(M, N, K, R, count, dtype, seed=M + R, index=index).check()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,N,K,R,count", [(2, 2688, 384, 4, 1), (70, 1408, 632, 1, 12), (20, 300, 200, 2, 3), (33, 130, 70, 7, 2),
                                           (40, 5, 300, 16, 2), (40, 300, 3, 16, 2), (9, 7, 6, 5, 2), (50, 260, 9, 9, 3),
                                           (2100, 136, 200, 3, 4), (2100, 300, 5, 16, 2), (2100, 6, 256, 40, 2),
                                           (2100, 264, 260, 65, 2)])
def test_short_sides(M, N, K, R, count, dtype):
    """Sides shorter than the pieces that rows are read in, and ends inside them."""
    Problem(M, N, K, R, count, dtype, seed=N + R).check()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,N,K,R,count", [(30, 40, 24, 8, 64), (30, 40, 24, 8, 65), (512, 136, 260, 20, 64), (513, 136, 260, 20, 64),
                                           (512, 300, 70, 33, 2), (300, 64, 1100, 16, 300), (1500, 1030, 64, 5, 9)])
def test_adapters_of_a_window(M, N, K, R, count, dtype):
    """Many adapters in a window, one window or several, adapters without rows."""
    Problem(M, N, K, R, count, dtype, seed=M + count).check()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,N,K,R,count", [(1100, 40, 6200, 64, 3), (1030, 6200, 48, 20, 5), (300, 7100, 72, 100, 4), (1025, 6161, 6157, 65, 2),
                                           (2500, 100, 8200, 16, 2)])
def test_long_sides(M, N, K, R, count, dtype):
    """Long sides of few rows, which are taken as of many, in both directions."""
    Problem(M, N, K, R, count, dtype, seed=M + R).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M", [1000, 2100])
def test_crowded_window(M, dtype):
    """Most rows have one adapter, a few windows many more than their share."""
    index = torch.zeros(M, dtype=torch.int64, device="cuda")
    index[-40:] = torch.arange(40, device="cuda") - 1
    Problem(M, 300, 200, 16, 39, dtype, seed=M, index=index).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [1, 8, 10])
def test_views(dtype, pad):
    """Rows with a stride, on and off the 16-byte boundaries, with NaN between them."""
    Problem(75, 136, 72, 24, 3, dtype, seed=pad, pad=pad).check()
    Problem(2100, 72, 64, 16, 2, dtype, seed=pad, pad=pad).check()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_what_is_left_out(dtype):
    """No Y, D, scales; O in the place of Y and dX in that of D; each gradient by itself."""
    p = Problem(90, 200, 96, 16, 4, dtype, seed=2, scales=False)
    O, H = p.forward(Y=False)
    p.check_forward(O, H, Y=False)
    full = p.forward()[0]
    assert torch.equal(p.forward(want_h=False)[0], full)
    y = p.Y.clone()
    p.Y = y.clone()
    p.forward(out=p.Y)
    assert torch.equal(p.Y, full)
    p.Y = y
    whole = p.backward(H)
    p.check_backward(H, *p.backward(H, D=False), D=False)
    for i in range(3):
        one = p.backward(H if i == 2 else None, wants=[i == j for j in range(3)])
        assert torch.equal(one[i], whole[i])
    p.D = p.D.clone()
    assert torch.equal(p.backward(H, out=p.D)[0], whole[0])


@pytest.mark.parametrize("index", [[-1] * 40, [2] * 40, [5] + [-1] * 39, list(range(6)) * 6 + [-7, 6, 99, 2 ** 30]])
def test_adapters_without_rows(index):
    """No rows at all, of one adapter or of all but some; their gradients are zeros."""
    index = torch.tensor(index, device="cuda")
    p = Problem(40, 64, 48, 8, 6, "bf16", index=index)
    p.check()
    dA, dB = p.backward(p.forward()[1])[1:]
    for a in range(6):
        if not bool((index == a).any()):
            assert int(torch.count_nonzero(dA[a])) == 0 and int(torch.count_nonzero(dB[a])) == 0


def test_no_rows():
    p = Problem(0, 64, 48, 8, 6, "bf16")
    O, H = p.forward()
    dX, dA, dB = p.backward(H)
    assert O.shape == (0, 64) and dX.shape == (0, 48)
    assert int(torch.count_nonzero(dA)) == 0 and int(torch.count_nonzero(dB)) == 0


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_not_finite(dtype):
    """NaN and infinities reach the rows that hold them, and the gradients of their adapter."""
    M = 200
    index = torch.arange(M, device="cuda") // 50
    p = Problem(M, 72, 64, 16, 4, dtype, seed=4, index=index)
    O, H = p.forward()
    back = p.backward(H)
    p.X[10, 3], p.X[60, 5], p.Y[150, 7] = math.nan, math.inf, math.nan
    p.G[10, 1], p.G[70, 2] = math.nan, math.inf
    O2, H2 = p.forward()
    dX2, dA2, dB2 = p.backward(H)
    keep = torch.ones(M, dtype=torch.bool, device="cuda")
    keep[[10, 60, 150]] = False
    assert torch.equal(O[keep], O2[keep]) and bool(torch.isnan(O2[10]).all()) and not bool(torch.isfinite(O2[60]).any())
    assert int(torch.isnan(O2[150]).sum()) == 1
    keep = torch.ones(M, dtype=torch.bool, device="cuda")
    keep[[10, 70]] = False
    assert torch.equal(back[0][keep], dX2[keep]) and bool(torch.isnan(dX2[10]).all())
    for a in (2, 3):
        assert torch.equal(back[1][a], dA2[a]) and torch.equal(back[2][a], dB2[a])
    assert bool(torch.isnan(dA2[0]).all()) and bool(torch.isnan(dB2[0][1]).all()) and bool(torch.isfinite(dB2[0][0]).all())


def test_large_and_small_values():
    """f16 values whose h and p lie outside f16's range."""
    for size in (300.0, 1e-4):
        p = Problem(70, 136, 256, 16, 2, "f16", seed=6)
        p.X *= size
        p.A.mul_(16.0 if size > 1 else 1e-2)
        p.B.mul_(1e-3 if size > 1 else 1.0)
        p.check()


def test_a_difference():
    """The gradients are those of the forward pass: differences of a linear function in 64
    bits, of sum(g o): o changes by delta B (X A)^T and so on, whose sums are the gradients'."""
    p = Problem(60, 40, 32, 8, 3, "f32", seed=8)
    O, H = p.forward()
    dX, dA, dB = p.backward(H, D=False)
    loss = lambda: float((p.forward(want_h=False)[0].double() * p.G.double()).sum())
    base = loss()
    r = gen(9)
    for t, grad in ((p.X, dX), (p.A, dA), (p.B, dB)):
        d = torch.randn(t.shape, generator=r, device="cuda") * 2.0 ** -6
        old = t.clone()
        t.copy_(old + d)
        moved = loss()
        want = float((grad.double() * (t - old).double()).sum())
        t.copy_(old)
        # linear in each of the three; two losses of 2400 terms, each off by 2^-24 of its size times some tens
        assert abs(moved - base - want) <= 2.0 ** -24 * 100 * float((O.abs() * p.G.abs()).sum())


def test_far_offsets():
    """Rows past 2^31 bytes."""
    M, N, K = 140000, 8192, 64
    index = (torch.arange(M, device="cuda") % 2).int()
    p = Problem(M, 8, K, 8, 2, "bf16", seed=1, index=index)
    big = torch.zeros(M, N, dtype=torch.bfloat16, device="cuda")
    B = torch.zeros(2, N, 8, dtype=torch.bfloat16, device="cuda")
    B[:, :8], B[:, -8:] = p.B, p.B
    big[:, :8], big[:, -8:] = p.Y, p.Y
    O, H = p.forward()
    out = torch.empty_like(big)
    g.gptq2d_adapters(p.X, p.A, B, p.scales, p.groups, big, out, None, p.space(g.gptq2d_adapters_workspace_size(M, N, K, 8, 2)))
    assert torch.equal(out[:, :8], O) and torch.equal(out[:, -8:], O) and int(torch.count_nonzero(out[:, 8:-8])) == 0
    big.zero_()
    big[:, -8:] = p.G
    dX, dA = torch.empty_like(p.X), torch.empty(2, 8, K, device="cuda")
    dB = torch.empty(2, N, 8, device="cuda")
    ws = p.space(g.gptq2d_adapters_backward_workspace_size(M, N, K, 8, 2))
    g.gptq2d_adapters_backward(big, p.X, p.A, B, p.scales, p.groups, H, p.D, dX, dA, dB, ws)
    # the same sums with zeros between them
    p.check_backward(H, dX, dA, dB[:, -8:].contiguous())
    assert int(torch.count_nonzero(dB[:, :-8])) == 0


def test_graph_and_streams():
    """Forward and backward captured with their workspaces and replayed on other rows, beside
    calls on another stream; the same bits each time."""
    p = Problem(150, 264, 136, 16, 5, "bf16", seed=3)
    M, N, K, R, count = p.shape
    O, H = torch.empty_like(p.Y), torch.empty(M, R, device="cuda")
    dX, dA, dB = torch.empty_like(p.X), torch.empty(count, R, K, device="cuda"), torch.empty(count, N, R, device="cuda")
    f, b = p.space(g.gptq2d_adapters_workspace_size(*p.shape)), p.space(g.gptq2d_adapters_backward_workspace_size(*p.shape))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        g.gptq2d_adapter_groups(p.index, count, p.groups)
        g.gptq2d_adapters(p.X, p.A, p.B, p.scales, p.groups, p.Y, O, H, f)
        g.gptq2d_adapters_backward(p.G, p.X, p.A, p.B, p.scales, p.groups, H, p.D, dX, dA, dB, b)
    other = torch.cuda.Stream()
    for i in range(3):
        p.index.copy_(torch.randint(-1, count, (M,), generator=gen(i), device="cuda"))
        p.X.copy_(torch.randn(M, K, generator=gen(i + 9), device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        p.check_forward(O, H)
        p.check_backward(H, dX, dA, dB)
        with torch.cuda.stream(other):
            again, h = p.forward()
            back = p.backward(h)
        torch.cuda.synchronize()
        assert torch.equal(again, O) and all(torch.equal(x, y) for x, y in zip(back, (dX, dA, dB)))
