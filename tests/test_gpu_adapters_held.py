"""What gptq2d_adapters and its gradients hold of h and p between their two products.

h and p are made exact in 32 bits: two terms each, x0 a0 + x1 a1 with whole numbers below
2^8, the second 2^-8 as large, so a whole number of 2^-8 below 2^16 (24 bits). What a test
allows then is the second product's own: of n exact products in 32 bits n 2^-24 of the sum
of magnitudes, and half a step of the output type. A row of weights has three ranks other
than zero, each of whose products is made of at most three (f16: six) of numbers: n = 9 (18),
and 4 for scale, addition and conversions. Y (and D) take nearly all of the result away, so that
the last rounding hides nothing.

Loud ranks and rows, whose other factor is zero, may take nothing from the others: what is
allowed goes by the sum of the magnitudes of a result's own terms."""
import math

import pytest
import torch

from test_gpu_adapters import HALF, Problem, gen

pytestmark = pytest.mark.gpu

SIZES = [(1, 300, 200, 8, 1), (5, 300, 200, 3, 2), (70, 136, 64, 20, 3), (40, 264, 72, 64, 2), (33, 300, 130, 128, 2),
         (300, 2000, 500, 16, 5), (2100, 264, 260, 16, 3), (2100, 300, 136, 100, 2)]
USED = 3
NUMBERS = {"f32": 1, "f16": 6, "bf16": 3}  # products that one of a 32-bit and a given number is made of
TOP = {"f32": 256, "f16": 2048, "bf16": 256}


def whole(r, low, high, *shape):
    return torch.randint(low, high, shape, generator=r, device="cuda").float()


def sides(r, rows, weights):
    """rows [m, n] and weights [count, rank, n] whose products have 24 bits."""
    n = rows.shape[1]
    for t, second in ((rows, 1.0), (weights, 2.0 ** -8)):
        t.zero_()
        t[..., 0] = whole(r, 128, 256, *t.shape[:-1]).to(t.dtype)
        t[..., n // 2] = (whole(r, 1, 256, *t.shape[:-1]) * second).to(t.dtype)


def few(r, weights, top):
    """weights [count, n, rank] with USED ranks other than zero, whole numbers up to top of 2^-14."""
    rank = weights.shape[2]
    weights.zero_()
    at = torch.rand(weights.shape, generator=r, device="cuda").topk(min(USED, rank), dim=2).indices
    sign = torch.where(torch.rand(at.shape, generator=r, device="cuda") < 0.5, -1.0, 1.0)
    weights.scatter_(2, at, (sign * whole(r, 1, top, *at.shape) * 2.0 ** -14).to(weights.dtype))


def products(p, left, right):
    """Of each row, left [rows, n] times right[a]^T, and the sums of magnitudes, in 64 bits."""
    out = torch.zeros(left.shape[0], right.shape[1], dtype=torch.float64, device="cuda")
    size = torch.zeros_like(out)
    for a in range(right.shape[0]):
        at = (p.index == a).nonzero()[:, 0]
        x, w = left[at].double(), right[a].double()
        out[at], size[at] = torch.matmul(x, w.T), torch.matmul(x.abs(), w.abs().T)
    return out, size


def expect(got, low, size, rest, dtype):
    """got = low + rest, rounded, with low of n products."""
    far = 2.0 ** -24 * (max(3, NUMBERS[dtype]) * USED + 4) * size
    want = low + rest.double()
    off = far + (far + want.abs()) * (HALF[dtype] + 2.0 ** -23) + (2.0 ** -25 if dtype == "f16" else 0.0)
    bad = (got.double() - want).abs() > off
    assert not bool(bad.any()), ((got.double() - want).abs() / off).max()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,N,K,R,count", SIZES)
def test_h(M, N, K, R, count, dtype):
    p, r = Problem(M, N, K, R, count, dtype, seed=M + R, scales=False), gen(M)
    sides(r, p.X, p.A)
    few(r, p.B, TOP[dtype])
    h, _ = products(p, p.X, p.A)
    o, size = products(p, h, p.B)
    p.Y.copy_(-o)
    O, H = p.forward()
    assert torch.equal(H.double(), h)
    expect(O, o, size, p.Y, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,N,K,R,count", SIZES)
def test_p(M, N, K, R, count, dtype):
    p, r = Problem(M, N, K, R, count, dtype, seed=M + R, scales=False), gen(M)
    turned = p.B.transpose(1, 2)
    sides(r, p.G, turned)
    a = torch.empty(count, K, R, device="cuda")
    few(r, a, TOP[dtype])
    p.A.copy_(a.transpose(1, 2))
    pr, _ = products(p, p.G, turned)
    dx, size = products(p, pr, p.A.transpose(1, 2))
    p.D.copy_(-dx)
    dX = p.backward(None, wants=(True, False, False))[0]
    expect(dX, dx, size, p.D, dtype)


def componentwise(p, dtype, O, H, dX, dA, dB):
    """The results without Y and D, each bounded by its own terms; H as given for dB."""
    M, N, K, R, count = p.shape
    u, each = 2.0 ** -24, NUMBERS[dtype]
    last = lambda x, far: far + (far + x.abs()) * (HALF[dtype] + 2.0 ** -23) + (2.0 ** -25 if dtype == "f16" else 0.0)
    worst = lambda got, x, off: (float(((got.double() - x).abs() / (off + 1e-300)).max()) if x.numel() else 0.0)
    for a, at, A, B, s in p.rows():
        x, gr, n = p.X[at].double(), p.G[at].double(), each * len(at) + 24
        h, h_off = torch.matmul(x, A.T), u * (K + 20) * torch.matmul(x.abs(), A.T.abs())
        o, far = s * torch.matmul(h, B.T), s * torch.matmul(h_off + u * (each * R + 4) * h.abs(), B.T.abs())
        assert worst(O[at], o, last(o, far)) <= 1.0, ("o", worst(O[at], o, last(o, far)))
        q, q_off = s * torch.matmul(gr, B), u * (N + 24) * s * torch.matmul(gr.abs(), B.abs())
        dx, far = torch.matmul(q, A), torch.matmul(q_off + u * (each * R + 4) * q.abs(), A.abs())
        assert worst(dX[at], dx, last(dx, far)) <= 1.0, ("dx", worst(dX[at], dx, last(dx, far)))
        off = torch.matmul((q_off + u * n * q.abs()).T, x.abs())
        assert worst(dA[a], torch.matmul(q.T, x), off) <= 1.0, ("dA", worst(dA[a], torch.matmul(q.T, x), off))
        h = H[at].double()
        off = s * torch.matmul(gr.abs().T, u * n * h.abs())
        assert worst(dB[a], s * torch.matmul(gr.T, h), off) <= 1.0, ("dB", worst(dB[a], s * torch.matmul(gr.T, h), off))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,N,K,R,count", [(70, 136, 64, 8, 2), (70, 136, 264, 20, 2), (40, 264, 72, 64, 2), (600, 130, 70, 128, 3),
                                           (2100, 264, 512, 16, 3)])
def test_loud_ranks(M, N, K, R, count, dtype):
    """One rank's h (or p) is 2^26 times the others', and the weights after it are zero."""
    p = Problem(M, N, K, R, count, dtype, seed=M + R)
    p.A[:, 0] *= 2.0 ** 12
    p.A[:, 1:] *= 2.0 ** -10
    p.B[:, :, 0] = 0.0
    p.B[:, :, 1:] *= 2.0 ** 4
    p.X *= 2.0 ** -2
    O, H = p.forward(Y=False)
    # backward with the parts of A and B changed: rank 1's p is loud
    none = p.backward(H, D=False)
    p.A[:, 1] = 0.0
    p.B[:, :, 1] *= 2.0 ** 10
    O2, H2 = p.forward(Y=False)
    back = p.backward(H2, D=False)
    componentwise(p, dtype, O2, H2, *back)
    for t in (O, *none):
        assert bool(torch.isfinite(t).all())
    p = Problem(M, N, K, R, count, dtype, seed=M + R)
    p.A[:, 0] *= 2.0 ** 12
    p.A[:, 1:] *= 2.0 ** -10
    p.B[:, :, 0] = 0.0
    O, H = p.forward(Y=False)
    componentwise(p, dtype, O, H, *p.backward(H, D=False))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,N,K,R,count", [(70, 136, 64, 8, 2), (70, 133, 77, 40, 2), (900, 264, 72, 16, 2), (2100, 136, 264, 33, 3)])
def test_loud_rows(M, N, K, R, count, dtype):
    """Rows whose h is 2^30 times the others' and whose gradient is zero (masked tokens of a prompt), and
    rows whose gradient is as much larger and whose input is zero."""
    p = Problem(M, N, K, R, count, dtype, seed=M + R)
    at = torch.arange(M, device="cuda") % 7
    H = torch.randn(M, R, generator=gen(M), device="cuda")
    H[at == 0] *= 2.0 ** 30
    p.G[at == 0] = 0.0
    p.G[at == 1] *= 2.0 ** 14
    p.G[at > 1] *= 2.0 ** -10
    p.X[at == 1] = 0.0
    O, _ = p.forward(Y=False)
    componentwise(p, dtype, O, H, *p.backward(H, D=False))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_infinities_stay(dtype):
    """An infinite h or gradient beside numbers that fewer bits hold gives infinities, not NaN."""
    M, N, K, R = 40, 72, 64, 4
    p = Problem(M, N, K, R, 1, dtype, seed=3, index=torch.zeros(M, dtype=torch.int32, device="cuda"), scales=False)
    p.A.fill_(1.0)
    p.B.fill_(0.5)
    p.X.fill_(1.0)
    p.G.fill_(1.0)
    p.X[3, 5], p.X[4, 6] = math.inf, -math.inf
    O, H = p.forward(Y=False)
    assert bool((O[3] == math.inf).all()) and bool((O[4] == -math.inf).all()) and bool((O[5:] == 128.0).all())
    p.X.fill_(1.0)
    p.G[7, 2] = math.inf
    dX, dA, dB = p.backward(torch.ones(M, R, device="cuda"), D=False)
    assert bool((dX[7] == math.inf).all()) and bool((dX[8:] == 144.0).all()) and bool((dA == math.inf).all())
    assert bool((dB[0, 2] == math.inf).all()) and bool((dB[0, 3:] == 40.0).all())
