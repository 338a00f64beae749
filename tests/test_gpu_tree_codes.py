"""A NaN code among a token's values makes NaN of its own element, in the rows
that see the token and no others, in the context as among the drafted tokens."""
import pytest
import torch

import eightbit as eb
from test_gpu_tree import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("group,dim,width", [(2, 64, 6), (10, 48, 6), (1, 128, 6), (6, 128, 6), (1, 192, 6), (3, 256, 6),
                                             (1, 64, 40)])
def test_nan_codes(group, dim, width, dtype):
    c = Case([50, 20, 0], width, 2, group, dim, 16, "e4m3", dtype, seed=dim + group)
    o, l, bo, bl = c.reference()
    nan = torch.zeros(3, width, 2, group, dim, dtype=torch.bool, device="cuda")
    # (sequence, position, head, element): two drafted tokens, two elements of one of them, and one of the context
    for b, x, head, d in ((0, 53, 1, dim - 1), (0, 52, 1, 5), (0, 53, 1, 16), (0, 51, 0, 0), (1, 3, 0, 7), (2, 2, 1, 9)):
        page = int(c.table[b, x // 16])
        c.C[1].view(torch.uint8)[page, head, x % 16, d] = 0xFF if d % 2 else 0x7F
        sees = torch.ones(width, dtype=torch.bool, device="cuda") if x < c.contexts[b] else c.sees(b)[:, x - c.contexts[b]]
        assert sees.any()
        nan[b, :, head, :, d] |= sees[:, None]
    O, lse = c.run()
    nan = nan.view(3 * width, -1)
    assert nan.any() and torch.equal(torch.isnan(O), nan)
    assert ((O.double() - o).abs() <= bo)[~nan].all()
    assert torch.equal(torch.isinf(lse), torch.isinf(l)) and ((lse.double() - l).abs() <= bl)[~torch.isinf(l)].all()
