"""The end of the example: the verified tree, its cache and pages, and the adapters'
gradients."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

import serving  # noqa: E402
from paper_2607_27042_amd import binding as g  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ran():
    import serve_rounded
    return serve_rounded.run(width=128, heads=4, kv_heads=2, vocab=200, prompt=70, page_size=16)


def test_kept_tokens(ran):
    r, n = ran, ran["prompt"]
    kept, pages = r["kept"], r["pages"]
    count = int(kept.count)
    assert 1 <= count <= 8 and int(kept.path[0, 0]) == 0 and int(r["length"]) == n + count
    assert 0 <= int(kept.next) < 200
    # every kept token follows the one before it
    path = kept.path[0, :count].tolist()
    assert [int(r["parents"][0, p]) for p in path[1:]] == path[:-1]
    # both continuations hold the prompt and the kept tokens
    old, new = r["cache"], r["later"]
    at = torch.tensor(list(range(n)) + [n + p for p in path], dtype=torch.int32, device="cuda")
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    whole = [x[at.long()] for x in old.read(old.slots(r["table"], zero, n + 8))]
    for b in range(2):
        got = new.read(new.slots(pages.table[b:b + 1], zero, n + count))
        assert all(torch.equal(a, e) for a, e in zip(got, whole))
    assert int(pages.left) >= 0
    last = (n + count) // 16
    assert pages.table[0, :last].tolist() == pages.table[1, :last].tolist()
    if (n + count) % 16:
        assert int(pages.table[0, last]) != int(pages.table[1, last])


def test_gradients_of_the_adapters(ran):
    """Those of the last step, at the adapters it began from, against the formulas in 64 bits: of a
    loss whose logits are rounded to 16 bits (2^-8 of up to some twenty), so p is off by a tenth at most."""
    A, B, groups, index, grads = ran["adapters"]
    before = [(t.double() + 0.5 * d.double()) for t, d in zip((A, B), grads)]  # (the step's own rounding: 2^-8)
    a, b = (t.requires_grad_() for t in before)
    h, target = ran["head_in"].double(), ran["target"].flatten()
    y = ran["rounded"]["head"](ran["head_in"]).double()
    logits = []
    for i in range(2):
        rows = index == i
        logits.append(y[rows] + torch.matmul(torch.matmul(h[rows], a[i].T), b[i].T))
    logits = torch.cat(logits)  # (the index ascends)
    loss = -torch.log_softmax(logits, 1).gather(1, target[:, None]).mean()
    for got, want in zip(grads, torch.autograd.grad(loss, (a, b))):
        assert got.shape == want.shape and bool(torch.isfinite(got).all())
        cosine = float((got.double() * want).sum() / (got.double().norm() * want.norm()))
        assert cosine >= 0.99, cosine
    assert torch.equal(g.adapters(ran["head_in"], A, B, groups, ran["rounded"]["head"](ran["head_in"])), ran["tuned"])
