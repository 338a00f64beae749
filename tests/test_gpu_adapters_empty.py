"""Adapters in autograd over batches without rows (the last requests of a shard have ended, say)."""
import itertools

import pytest
import torch

from paper_2607_27042_amd import binding as g

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("wants", [w for w in itertools.product([True, False], repeat=4) if any(w)])
def test_no_rows(wants, dtype):
    """Every choice of gradients, among them X's alone: of the adapters zeros, of the rest nothing."""
    shapes = (0, 64), (3, 8, 64), (3, 96, 8), (0, 96)
    X, A, B, Y = (torch.randn(s, device="cuda").to(dtype).requires_grad_(w) for s, w in zip(shapes, wants))
    groups = g.adapter_groups(torch.empty(0, dtype=torch.int32, device="cuda"), 3)
    O = g.adapters(X, A, B, groups, Y, torch.ones(3, device="cuda"))
    O.backward(torch.zeros_like(O))
    for t, w in zip((X, A, B, Y), wants):
        assert (t.grad is not None) == w
        if w:
            assert t.grad.shape == t.shape and int(torch.count_nonzero(t.grad)) == 0


def test_expanded_gradient_of_no_rows():
    """The gradient of a sum over no rows has no strides."""
    X, A, B = (torch.randn(s, device="cuda").requires_grad_() for s in ((0, 64), (3, 8, 64), (3, 96, 8)))
    groups = g.adapter_groups(torch.empty(0, dtype=torch.int32, device="cuda"), 3)
    g.adapters(X, A, B, groups).sum().backward()
    assert X.grad.shape == (0, 64) and int(torch.count_nonzero(A.grad)) == 0 and int(torch.count_nonzero(B.grad)) == 0
