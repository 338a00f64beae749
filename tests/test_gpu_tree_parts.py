"""What is not finite in a token that a query sees shows in its result, wherever
the token lies and into however many parts the sequence is split."""
import math

import pytest
import torch

from test_gpu_tree import Case

pytestmark = pytest.mark.gpu


# one sequence is split into many parts, 600 of them are not split
@pytest.mark.parametrize("seqs,context", [(1, 4096), (1, 1500), (5, 3000), (600, 300)])
@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_value_far_below_the_best(seqs, context, value, dtype):
    c = Case([context] * seqs, 1, 1, 1, 64, 16, "e4m3", dtype, seed=1)
    b, late, early = seqs - 1, context - 10, 5
    # a late key along the query: a score that no other token comes within 126 binary orders of
    page = int(c.table[b, late // 16])
    c.C[0].view(torch.uint8)[page, 0, late % 16] = torch.where(c.Q[b].float() < 0, 0xB8, 0x38).to(torch.uint8)
    c.S[0][page, 0, late % 16] = 256.0
    plain, lse = c.run()
    assert torch.isfinite(plain.float()).all() and float(lse[b, 0]) > 400
    c.S[1][int(c.table[b, early // 16]), 0, early % 16] = value
    O, lse2 = c.run()
    assert not torch.isfinite(O[b].float()).any() if math.isnan(value) else not torch.isfinite(O[b].float()).all()
    assert torch.equal(O[:b], plain[:b]) and torch.allclose(lse, lse2, rtol=2.0 ** -20)
