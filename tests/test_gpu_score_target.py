"""A target matters to the gradient of its log probability only."""
import pytest
import torch

from paper_2607_27042_amd import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_entropy_alone_does_not_read_the_target(dtype):
    x = torch.randn(4, 50, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(dtype)
    target = torch.tensor([50, -1, 2 ** 40, 7], device="cuda")
    got = binding.token_logprobs(x, target)
    one = torch.ones(4, device="cuda")
    want = binding.token_logprobs_backward(x, None, got, g_entropy=one)
    assert torch.isfinite(want.float()).all() and (want != 0).any(1).all()
    assert torch.equal(binding.token_logprobs_backward(x, target, got, g_entropy=one), want)
    both = binding.token_logprobs_backward(x, target, got, one, one)
    assert torch.isnan(both).all(1).tolist() == [True, False, True, False] and torch.equal(both[1], want[1])
