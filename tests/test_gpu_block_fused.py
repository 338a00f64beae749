"""Layers of one and two rows, which quantise X in the product's own launch: both
kinds of scales, a short last block and tile, more blocks than a wave holds at
once, blocks that are not finite. Bounds as in tests/test_gpu_block.py."""
import pytest
import torch

from paper_2607_27042_amd import binding

import eightbit as eb
from test_gpu_block import _assert_close, _bound, _data, _gen

pytestmark = pytest.mark.gpu

SIZES = [(2, 17, 200), (1, 130, 4226), (2, 300, 4226), (2, 64, 130), (1, 16, 2), (2, 33, 9000)]


def _layer(x, W, SW, pow2):
    M, N = x.shape[0], W.shape[0]
    Y = torch.full((M, N + 3), 5.0, dtype=x.dtype, device="cuda")
    ws = torch.empty(binding.gptq2d_block_linear_workspace_size(M, N, x.shape[1]), dtype=torch.uint8, device="cuda")
    binding.gptq2d_block_linear(x, W, SW, Y[:, :N], ws, pow2=pow2)
    assert (Y[:, N:] == 5.0).all()
    return Y[:, :N]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_few_rows(M, N, K, dtype):
    w = torch.randn(N, K, generator=_gen(9), device="cuda").double() / K ** 0.5
    for pow2 in (False, True):
        qw, sw = eb.blocks(w, 128, pow2)
        W, SW = eb.to_codes(qw, sw, False)
        for pad, offset in ((0, 0), (6, 2)):  # even strides and starts: rows that are read in pairs
            x = _data(M + N, M, K, dtype, pad, offset)
            Y = _layer(x, W, SW, pow2)
            a, b = eb.values(x, 1, pow2), qw * eb.spread(sw, N, K, 128)
            want, mags = a @ b.T, a.abs() @ b.abs().T
            _assert_close(Y, want, mags, dtype, K, f"pow2 {pow2}")
            apart = binding.block_matmul(binding.block_quantize(x, 1, pow2), binding.Blocks(W, SW, 128), x.dtype)
            assert ((Y.double() - apart.double()).abs() <= 2 * _bound(want, mags, dtype, K)).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("K", [300, 4226])
def test_few_rows_that_are_not_finite(K, dtype):
    N = 40
    qw, sw = eb.blocks(torch.randn(N, K, generator=_gen(3), device="cuda").double(), 128)
    W, SW = eb.to_codes(qw, sw, False)
    x = _data(5, 2, K, dtype)
    whole = _layer(x, W, SW, False).clone()
    assert torch.isfinite(whole.float()).all()
    for row in (0, 1):
        for value, at in ((float("nan"), 3), (float("inf"), 130), (-float("inf"), K - 1)):
            y = x.clone()
            y[row, at] = value
            got = _layer(y, W, SW, False)
            assert torch.isnan(got[row]).all() and torch.equal(got[1 - row], whole[1 - row])
        y = x.clone()
        y[row, 3], y[row, 200] = float("nan"), float("inf")
        assert torch.isnan(_layer(y, W, SW, False)[row]).all()
        one = _layer(y[row:row + 1], W, SW, False)
        assert torch.isnan(one).all()
