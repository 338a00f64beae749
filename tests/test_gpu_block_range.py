"""Products whose two scales multiply to less or more than 32 bits hold, while
the results are in their range: every route gives them, within the bounds of
ordinary ones (tests/test_gpu_block.py)."""
import pytest
import torch

from paper_2607_27042_amd import binding

import eightbit as eb
from test_gpu_block import _gen

pytestmark = pytest.mark.gpu

# few rows; tiles of 64; of 128, whole and in parts; of 256
SIZES = [(1, 40, 300), (16, 100, 300), (17, 100, 300), (40, 70, 260), (130, 200, 300), (300, 130, 1500), (1100, 1030, 4300),
         (2000, 2300, 385), (3900, 2901, 200), (3900, 2816, 512)]


def _codes(seed, rows, cols, low=0):
    """Codes of 2^low times odd integers up to 7, a tenth of the rows zero."""
    q = (2 * torch.randint(-4, 4, (rows, cols), generator=_gen(seed), device="cuda") + 1).double() * 2.0 ** low
    q[::10] = 0
    return q


def _third(e):
    """4/3 2^e as 32 bits hold it: a factor with all of its bits in use."""
    return float(torch.tensor(4 / 3)) * 2.0 ** e


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("br", [1, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scales_far_from_one(M, N, K, br, dtype):
    nb = -(-K // 128)
    # exponents of the two scales in every block, of the codes. Products of the scales: below the
    # smallest normal number (and below all), above the largest; then one factor that takes the sum
    # of a block out of the range before the other brings it back
    for ea, eb_, low in ((-66, -68, 6), (-70, -72, 6), (63, 65, -9), (120, -118, 4), (-118, 120, 4), (-124, 118, -9),
                         (118, -124, -9)):
        qa, qb = _codes(M, M, K, low), _codes(N + 1, N, K, low)
        sa = torch.full((M, nb), _third(ea), dtype=torch.float64, device="cuda")
        sb = torch.full((-(-N // br), nb), _third(eb_), dtype=torch.float64, device="cuda")
        # one row of each in ordinary scales, in its last block
        sa[min(1, M - 1), -1] = sb[-1, -1] = 1.0
        A, SA = eb.to_codes(qa, sa, True)
        B, SB = eb.to_codes(qb, sb, br == 1)
        C = torch.empty(M, N, dtype=eb.DTYPE[dtype], device="cuda")
        ws = torch.empty(max(256, binding.gptq2d_block_matmul_workspace_size(M, N, K)), dtype=torch.uint8, device="cuda")
        binding.gptq2d_block_matmul(A, SA, B, SB, C, ws, block_rows=br)
        a, b = qa * eb.spread(sa, M, K, 1), qb * eb.spread(sb, N, K, br)
        want, mags = a @ b.T, a.abs() @ b.abs().T
        inside = (want.abs() < torch.finfo(C.dtype).max / 2) & (mags < 2.0 ** 126)
        rel = (152 + 4 * nb) * 2.0 ** -24 if dtype == "f32" else 2.0 ** -11
        bound = want.abs() * eb.HALF_ULP[dtype] * 1.01 + mags * rel + 2.0 ** -126  # (results below normal ones may be 0)
        err = (C.double() - want).abs()
        assert inside.any()
        bad = inside & ~(err <= bound)
        assert not bad.any(), f"scales 2^{ea}, 2^{eb_}: {int(bad.sum())} of {int(inside.sum())} off, {C[bad][:3]} {want[bad][:3]}"


@pytest.mark.parametrize("M", [1, 2, 3, 17, 150])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layer_far_from_one(M, dtype):
    N, K = 200, 700
    for ex, ew in ((-62, -64), (-60, -62), (110, -118), (-110, 118)):
        x = (torch.randn(M, K, generator=_gen(1), device="cuda").double() * 2.0 ** ex).to(eb.DTYPE[dtype])
        x[:, :128] = 0
        qw, sw = eb.blocks(torch.randn(N, K, generator=_gen(2), device="cuda").double() * 2.0 ** ew, 128)
        W, SW = eb.to_codes(qw, sw, False)
        Y = torch.empty(M, N, dtype=x.dtype, device="cuda")
        ws = torch.empty(binding.gptq2d_block_linear_workspace_size(M, N, K), dtype=torch.uint8, device="cuda")
        binding.gptq2d_block_linear(x, W, SW, Y, ws)
        a, b = eb.values(x), qw * eb.spread(sw, N, K, 128)
        want, mags = a @ b.T, a.abs() @ b.abs().T
        rel = (152 + 24) * 2.0 ** -24 if dtype == "f32" else 2.0 ** -11
        bound = want.abs() * eb.HALF_ULP[dtype] * 1.01 + mags * rel + 2.0 ** -126
        bad = ~((Y.double() - want).abs() <= bound) & (mags < 2.0 ** 126)
        assert not bad.any(), f"2^{ex}, 2^{ew}: {int(bad.sum())} off, {Y[bad][:3]} {want[bad][:3]}"
