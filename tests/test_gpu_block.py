"""Eight-bit blocks through the C ABI against the plain 64-bit forms: the
quantiser bit for bit, products and gradients within bounds derived from the
types (below), at odd sizes, strides and blocks that are not finite.

Bounds. A result is off by at most
  half a unit of its type's last place (relative 2^-8 / 2^-11 / 2^-24), and
  of the sum of magnitudes sum |a b| of its products:
    32-bit results: each addition of 32-bit sums rounds by 2^-24; a chain has at
      most 128 terms in a block, the blocks, eight waves or sixteen splits
      (152 + blocks) additions and two scalings a block;
    16-bit results: the eight-bit instruction keeps at least 11 bits below the
      largest product of a block, 2^-11 of the sum of magnitudes.
"""
import pytest
import torch

from paper_2607_27042_amd import binding

import eightbit as eb

pytestmark = pytest.mark.gpu


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(seed, *shape):
    return torch.randn(*shape, generator=_gen(seed), device="cuda", dtype=torch.float64)


def _data(seed, rows, cols, dtype, pad=0, offset=0):
    """Values over ten powers of two by row, in a buffer whose rows are `pad`
    wider and start `offset` elements late."""
    x = _randn(seed, rows, cols) * torch.exp2(torch.randint(-5, 6, (rows, 1), generator=_gen(seed + 1),
                                                            device="cuda").double())
    buf = torch.full((rows, cols + pad + offset), 777.0, dtype=eb.DTYPE[dtype], device="cuda")
    view = buf[:, offset:offset + cols]
    view.copy_(x)
    return view


def _check_codes(Q, S, x, block_rows, pow2, rows_first):
    q, s = eb.blocks(x, block_rows, pow2)
    assert torch.equal(torch.nan_to_num(S.double(), nan=-1.0), torch.nan_to_num(s if rows_first else s.T, nan=-1.0))
    assert torch.equal(Q.float().double(), q)


QUANT = [(1, 1), (1, 128), (3, 5), (2, 129), (130, 257), (128, 128), (257, 640), (64, 4096)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols", QUANT)
def test_quantiser_is_the_definition(rows, cols, dtype):
    for pow2 in (False, True):
        for pad, offset in ((0, 0), (3, 0), (8, 1)):
            x = _data(rows * 7 + cols, rows, cols, dtype, pad, offset)
            for br in (1, 128):
                Q, QT = eb.empty_codes(rows, cols, 16), eb.empty_codes(cols, rows)
                shape = (-(-cols // 128), rows) if br == 1 else (-(-rows // 128), -(-cols // 128))
                shape_t = (-(-rows // 128), cols) if br == 1 else (-(-cols // 128), -(-rows // 128))
                S = torch.full(shape, -5.0, device="cuda")
                ST = torch.full(shape_t, -5.0, device="cuda")
                binding.gptq2d_block_quantize(x, Q, S, QT, ST, block_rows=br, pow2=pow2)
                _check_codes(Q, S, x, br, pow2, br != 1)
                _check_codes(QT, ST, x.T, br, pow2, br != 1)
                # each output by itself
                Q2, S2 = eb.empty_codes(rows, cols), torch.zeros_like(S)
                binding.gptq2d_block_quantize(x, Q2, S2, block_rows=br, pow2=pow2)
                assert torch.equal(Q2.view(torch.uint8), Q.view(torch.uint8)) and torch.equal(S, S2)
                QT2, ST2 = eb.empty_codes(cols, rows), torch.zeros_like(ST)
                binding.gptq2d_block_quantize(x, None, None, QT2, ST2, block_rows=br, pow2=pow2)
                assert torch.equal(QT2.view(torch.uint8), QT.view(torch.uint8)) and torch.equal(ST, ST2)


def test_quantiser_writes_its_rows_and_nothing_else():
    x = _data(3, 5, 37, "bf16")
    buf = torch.full((7, 64), 0x55, dtype=torch.uint8, device="cuda")
    Q = buf[1:6].view(torch.float8_e4m3fn)[:, :37]
    binding.gptq2d_block_quantize(x, Q, torch.empty(1, 5, device="cuda"))
    assert (buf[0] == 0x55).all() and (buf[6] == 0x55).all() and (buf[:, 48:] == 0x55).all()
    assert (buf[1:6, 37:48] == 0).all()


def test_quantiser_extremes():
    """Zeros, subnormal blocks, the largest numbers, ties, NaN and infinity."""
    x = torch.zeros(8, 256, device="cuda")
    x[1, :128] = 1e-42
    x[2, 3] = 3.4e38
    x[3, :8] = torch.tensor([448.0, 17.0, 19.0, -17.0, 2 ** -10, 3 * 2 ** -10, -2 ** -10, 1.0])
    x[4, 5] = float("nan")
    x[5, 200] = float("inf")
    x[6, 1] = -float("inf")
    x[7] = torch.arange(256) - 128
    for br in (1, 128):
        for pow2 in (False, True):
            Q, QT = eb.empty_codes(8, 256), eb.empty_codes(256, 8)
            S = torch.empty(2, 8, device="cuda") if br == 1 else torch.empty(1, 2, device="cuda")
            ST = torch.empty(1, 256, device="cuda") if br == 1 else torch.empty(2, 1, device="cuda")
            binding.gptq2d_block_quantize(x, Q, S, QT, ST, block_rows=br, pow2=pow2)
            _check_codes(Q, S, x, br, pow2, br != 1)
            _check_codes(QT, ST, x.T, br, pow2, br != 1)


def test_small_integers_are_exact_with_powers_of_two():
    z = torch.randint(-16, 17, (300, 500), generator=_gen(5), device="cuda")
    Q, S = eb.empty_codes(300, 500), torch.empty(3, 4, device="cuda")
    binding.gptq2d_block_quantize(z.float(), Q, S, block_rows=128, pow2=True)
    assert torch.equal((Q.float() * eb.spread(S, 300, 500, 128)).long(), z)


def _bound(exact, mags, dtype, K):
    blocks = -(-K // 128)
    rel = (152 + 4 * blocks) * 2.0 ** -24 if dtype == "f32" else 2.0 ** -11
    return exact.abs() * eb.HALF_ULP[dtype] * 1.01 + mags * rel + 1e-30


def _assert_close(got, exact, mags, dtype, K, what):
    # past the type's range a result is infinite; within the bound of its end it may be
    largest, bound = torch.finfo(eb.DTYPE[dtype]).max, _bound(exact, mags, dtype, K)
    inf = torch.isinf(got)
    assert (inf | (exact.abs() - bound <= largest * (1 + eb.HALF_ULP[dtype]))).all()
    assert (exact.abs() + bound >= largest)[inf].all() and (got[inf].double().sign() == exact[inf].sign()).all()
    got, exact = got.double().masked_fill(inf, 0.0), exact.masked_fill(inf, 0.0)
    err = (got - exact).abs()
    bad = ~(err <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {err[bad].max()}"
    # a sum over random signs is far nearer than its bound
    rms = float(err.pow(2).mean().sqrt() / exact.pow(2).mean().sqrt())
    assert rms <= {"f32": 1e-5, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}[dtype], f"{what}: rms {rms}"


SIZES = [(1, 1, 1), (1, 128, 128), (2, 17, 31), (16, 16, 2048), (17, 100, 129), (33, 130, 1000), (64, 257, 384),
         (65, 64, 100), (130, 131, 700), (300, 1000, 513), (513, 384, 128), (128, 128, 4096), (700, 640, 1400)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_product(M, N, K, dtype):
    print(f"[block] {M}x{N}x{K} {dtype}", flush=True)
    for br in (128, 1):
        qa, sa = eb.blocks(_data(M + K, M, K, "f32"))
        qb, sb = eb.blocks(_data(N + 2 * K, N, K, "f32"), br)
        A, SA = eb.to_codes(qa, sa, True)
        B, SB = eb.to_codes(qb, sb, br == 1)
        ws = torch.empty(max(256, binding.gptq2d_block_matmul_workspace_size(M, N, K)), dtype=torch.uint8, device="cuda")
        buf = torch.full((M, N + 5), -9.0, dtype=eb.DTYPE[dtype], device="cuda")
        for C in (buf[:, :N], buf[:, 1:N + 1], torch.empty(M, N, dtype=eb.DTYPE[dtype], device="cuda")):
            binding.gptq2d_block_matmul(A, SA, B, SB, C, ws, block_rows=br)
            a, b = qa * eb.spread(sa, M, K, 1), qb * eb.spread(sb, N, K, br)
            _assert_close(C, a @ b.T, a.abs() @ b.abs().T, dtype, K, f"rows of {br}")
            first = C.clone()
            binding.gptq2d_block_matmul(A, SA, B, SB, C, ws, block_rows=br)
            assert torch.equal(first, C), "the same call gave other bits"
        assert (buf[:, N + 1:] == -9.0).all()


# few rows of large weights, tiles of 128 with K in parts and whole, tiles of 256, each with a short last block
LARGE = [(20, 8300, 300), (32, 500, 4200), (1100, 1030, 4300), (2000, 2300, 385), (3900, 2901, 200), (3900, 2816, 512)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,N,K", LARGE)
def test_large_products(M, N, K, dtype):
    test_product(M, N, K, dtype)


@pytest.mark.parametrize("M,N,K", [(2000, 2300, 385), (3900, 2901, 200)])
@pytest.mark.parametrize("br", [1, 128])
def test_large_products_pass_on_what_is_not_finite(M, N, K, br):
    test_product_passes_on_what_is_not_finite(M, N, K, br)


@pytest.mark.parametrize("M,N,K", [(1, 40, 300), (70, 200, 200)])
@pytest.mark.parametrize("br", [1, 128])
def test_product_passes_on_what_is_not_finite(M, N, K, br):
    x, w = _data(1, M, K, "f32"), _data(2, N, K, "f32")
    x[0, 130] = float("inf")
    w[7, 5] = float("nan")
    qa, sa = eb.blocks(x)
    qb, sb = eb.blocks(w, br)
    A, SA = eb.to_codes(qa, sa, True)
    B, SB = eb.to_codes(qb, sb, br == 1)
    ws = torch.empty(max(256, binding.gptq2d_block_matmul_workspace_size(M, N, K)), dtype=torch.uint8, device="cuda")
    C = torch.empty(M, N, device="cuda")
    binding.gptq2d_block_matmul(A, SA, B, SB, C, ws, block_rows=br)
    want = torch.isnan((qa * eb.spread(sa, M, K, 1)).sum(1))[:, None] | torch.isnan(
        (qb * eb.spread(sb, N, K, br)).sum(1))[None]
    assert torch.equal(torch.isnan(C), want) and want.any() and (M == 1 or not want.all())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 512, 384), (3, 100, 200), (40, 300, 500), (200, 130, 700)])
def test_linear(M, N, K, dtype):
    print(f"[linear] {M}x{N}x{K} {dtype}", flush=True)
    w = _randn(9, N, K) / K ** 0.5
    for pow2, pad, offset in ((False, 0, 0), (True, 5, 1)):
        x = _data(M + N, M, K, dtype, pad, offset)
        qw, sw = eb.blocks(w, 128, pow2)
        W, SW = eb.to_codes(qw, sw, False)
        Y = torch.empty(M, N, dtype=x.dtype, device="cuda")
        ws = torch.empty(binding.gptq2d_block_linear_workspace_size(M, N, K), dtype=torch.uint8, device="cuda")
        binding.gptq2d_block_linear(x, W, SW, Y, ws, pow2=pow2)
        a, b = eb.values(x, 1, pow2), qw * eb.spread(sw, N, K, 128)
        _assert_close(Y, a @ b.T, a.abs() @ b.abs().T, dtype, K, "linear")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (5, 130, 200), (130, 300, 129), (513, 200, 256)])
def test_gradients(M, N, K, dtype):
    print(f"[gradients] {M}x{N}x{K} {dtype}", flush=True)
    w = _randn(9, N, K) / K ** 0.5
    for pow2, pad, offset in ((False, 0, 0), (True, 5, 1)):
        x, dy = _data(M + N, M, K, dtype, pad, offset), _data(M + K, M, N, dtype, pad, offset)
        qw, sw = eb.blocks(w.T.contiguous(), 128, pow2)
        WT, SWT = eb.to_codes(qw, sw, False)
        ws = torch.empty(binding.gptq2d_block_linear_backward_workspace_size(M, N, K), dtype=torch.uint8, device="cuda")
        dX, dW = torch.empty(M, K, dtype=x.dtype, device="cuda"), torch.empty(N, K, device="cuda")
        binding.gptq2d_block_linear_backward(dy, x, WT, SWT, dX, dW, ws, pow2=pow2)
        a, b = eb.values(dy, 1, pow2), qw * eb.spread(sw, K, N, 128)
        _assert_close(dX, a @ b.T, a.abs() @ b.abs().T, dtype, N, "dX")
        a, b = eb.values(dy.T, 1, pow2), eb.values(x.T, 1, pow2)
        _assert_close(dW, a @ b.T, a.abs() @ b.abs().T, "f32", M, "dW")
        only = torch.empty_like(dX)
        binding.gptq2d_block_linear_backward(dy, None, WT, SWT, only, None, ws, pow2=pow2)
        assert torch.equal(only, dX)
        only = torch.empty_like(dW)
        binding.gptq2d_block_linear_backward(dy, x, None, None, None, only, ws, pow2=pow2)
        assert torch.equal(only, dW)


def test_gradients_against_differences():
    """Where the layer is linear (inputs that are exact in eight bits), the
    gradients are those of differences of sum(G Y)."""
    M, N, K = 6, 20, 150
    ints = lambda seed, *s: torch.randint(-8, 9, s, generator=_gen(seed), device="cuda").float()
    x, w, G = ints(1, M, K), ints(2, N, K), ints(3, M, N)
    # a seven in each block of weights and tokens keeps every scale a power of two that holds integers
    WT, SWT = eb.to_codes(*eb.blocks(w.T.contiguous(), 128, True), False)
    W, SW = eb.to_codes(*eb.blocks(w, 128, True), False)
    dX, dW = torch.empty(M, K, device="cuda"), torch.empty(N, K, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    binding.gptq2d_block_linear_backward(G, x, WT, SWT, dX, dW, ws, pow2=True)

    def loss(xx, ww):
        Wc, Sc = eb.to_codes(*eb.blocks(ww, 128, True), False)
        Y = torch.empty(M, N, device="cuda")
        binding.gptq2d_block_linear(xx, Wc, Sc, Y, ws, pow2=True)
        return float((G.double() * Y.double()).sum())
    base = loss(x, w)
    for i, j in ((0, 0), (5, 149), (3, 128)):
        d = x.clone(); d[i, j] += 1
        assert loss(d, w) - base == float(dX[i, j])
        d = w.clone(); d[i, j] -= 1
        assert base - loss(x, d) == float(dW[i, j])


def test_stream_and_graph():
    """A call on a side stream, and captured in a graph and replayed on new inputs."""
    M, N, K = 70, 300, 260
    W, SW = eb.to_codes(*eb.blocks(_randn(1, N, K), 128), False)
    x, Y = _data(2, M, K, "bf16").contiguous(), torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(binding.gptq2d_block_linear_workspace_size(M, N, K), dtype=torch.uint8, device="cuda")
    binding.gptq2d_block_linear(x, W, SW, Y, ws)
    want = Y.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        Y2 = torch.empty_like(Y)
        binding.gptq2d_block_linear(x, W, SW, Y2, ws)
    side.synchronize()
    assert torch.equal(want, Y2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.gptq2d_block_linear(x, W, SW, Y, ws)
    for seed in (3, 4, 5):
        x.copy_(_data(seed, M, K, "bf16"))
        graph.replay()
        torch.cuda.synchronize()
        got = Y.clone()
        binding.gptq2d_block_linear(x, W, SW, Y2, ws)
        assert torch.equal(got, Y2)


def test_refusals():
    W, SW = eb.to_codes(*eb.blocks(_randn(1, 40, 200), 128), False)
    x, Y = torch.zeros(3, 200, device="cuda"), torch.zeros(3, 40, device="cuda")
    ws = torch.empty(binding.gptq2d_block_linear_workspace_size(3, 40, 200), dtype=torch.uint8, device="cuda")
    with pytest.raises(TypeError, match="float32, float16"):
        binding.gptq2d_block_linear(x.double(), W, SW, Y.double(), ws)
    with pytest.raises(TypeError, match="one dtype"):
        binding.gptq2d_block_linear(x, W, SW, Y.half(), ws)
    with pytest.raises(TypeError, match="float8"):
        binding.gptq2d_block_linear(x, W.view(torch.uint8), SW, Y, ws)
    with pytest.raises(ValueError, match="W must be 40 x 200"):
        binding.gptq2d_block_linear(x, W[:, :100], SW, Y, ws)
    with pytest.raises(ValueError, match="16-byte"):
        binding._codes(torch.zeros(4, 200, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn), 4, 200, "W")
    with pytest.raises(ValueError, match="SW must be"):
        binding.gptq2d_block_linear(x, W, SW[:, :1], Y, ws)
    with pytest.raises(binding.Gptq2dError, match="ERR_WORKSPACE"):
        binding.gptq2d_block_linear(x, W, SW, Y, ws[:100])
    with pytest.raises(binding.Gptq2dError, match="256-byte"):
        binding.gptq2d_block_linear(x, W, SW, Y, torch.empty(ws.numel() + 256, dtype=torch.uint8, device="cuda")[1:])
    with pytest.raises(ValueError, match="neither"):
        binding.gptq2d_block_linear_backward(Y, x, None, None, None, None, ws)
