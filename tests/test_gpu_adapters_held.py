"""What gptq2d_adapters and its gradients hold of h and p between their two products.

h and p are made exact in 32 bits: two terms each, x0 a0 + x1 a1 with whole numbers below
2^8, the second 2^-8 as large, so a whole number of 2^-8 below 2^16 (24 bits). What a test
allows then is the second product's own: of n exact products in 32 bits n 2^-24 of the sum
of magnitudes, and half a step of the output type. A row of weights has three ranks other
than zero, each of whose products is made of at most three numbers: n = 9, and 4 for scale,
addition and conversions. Y (and D) take nearly all of the result away, so that the last
rounding hides nothing."""
import pytest
import torch

from test_gpu_adapters import HALF, Problem, gen

pytestmark = pytest.mark.gpu

SIZES = [(1, 300, 200, 8, 1), (5, 300, 200, 3, 2), (70, 136, 64, 20, 3), (40, 264, 72, 64, 2), (33, 300, 130, 128, 2),
         (300, 2000, 500, 16, 5), (2100, 264, 260, 16, 3), (2100, 300, 136, 100, 2)]
USED = 3


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


def judge(got, low, size, rest, dtype):
    """got = low + rest, rounded, with low of n products."""
    far = 2.0 ** -24 * (3 * USED + 4) * size
    want = low + rest.double()
    off = far + (far + want.abs()) * (HALF[dtype] + 2.0 ** -23) + (2.0 ** -25 if dtype == "f16" else 0.0)
    bad = (got.double() - want).abs() > off
    assert not bool(bad.any()), ((got.double() - want).abs() / off).max()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K,R,count", SIZES)
def test_h(M, N, K, R, count, dtype):
    p, r = Problem(M, N, K, R, count, dtype, seed=M + R, scales=False), gen(M)
    sides(r, p.X, p.A)
    few(r, p.B, 256)
    h, _ = products(p, p.X, p.A)
    o, size = products(p, h, p.B)
    p.Y.copy_(-o)
    O, H = p.forward()
    assert torch.equal(H.double(), h)
    judge(O, o, size, p.Y, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K,R,count", SIZES)
def test_p(M, N, K, R, count, dtype):
    p, r = Problem(M, N, K, R, count, dtype, seed=M + R, scales=False), gen(M)
    turned = p.B.transpose(1, 2)
    sides(r, p.G, turned)
    a = torch.empty(count, K, R, device="cuda")
    few(r, a, 256)
    p.A.copy_(a.transpose(1, 2))
    pr, _ = products(p, p.G, turned)
    dx, size = products(p, pr, p.A.transpose(1, 2))
    p.D.copy_(-dx)
    dX = p.backward(None, wants=(True, False, False))[0]
    judge(dX, dx, size, p.D, dtype)
