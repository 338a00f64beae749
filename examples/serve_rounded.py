"""From calibration to serving: one attention layer and its output head, rounded
by the library and served in eight bits.

  1. Calibrate. Sequences of tokens run through the layer and are scored
     (gptq2d_token_logprobs). What every matrix takes in gives the input side of its
     two-sided metric, the scores' gradient at what it gives out the other: through
     the scores (gptq2d_token_logprobs_backward), the head, whose product is in eight
     bits already (gptq2d_block_linear_backward), and the attention.
  2. Round. W / step is rounded to integers Z under ||A (Z - X) B|| with A and B
     the Cholesky factors of the two Grams (gptq2d_factor, gptq2d_round).
  3. Hold Z in e4m3 tiles with scales that are powers of two, which keep integers
     up to 16 as they are (gptq2d_block_quantize).
  4. Serve. A prompt's keys and values go into an eight-bit paged cache
     (gptq2d_cache_append); a tree of drafted tokens attends to it
     (gptq2d_tree_attention), and every product with a rounded matrix is
     gptq2d_block_linear.
  5. Score the drafted tokens, beside the same layer unrounded.
  6. Verify the tree (gptq2d_tree_verify), move the kept tokens' keys and values up
     (gptq2d_cache_commit), and go on with two continuations, which share the pages that are
     full and have a copy each of the last one (gptq2d_pages_update, gptq2d_cache_copy).
  7. Give back some of what rounding took: low-rank adapters of two requests beside the
     rounded head (gptq2d_adapters), fitted to its calibration targets through
     gptq2d_adapters_backward.

    python examples/serve_rounded.py [--width 256] [--vocab 1000] [--prompt 300]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2607_27042_amd import binding as g  # noqa: E402


def gram_factor(rows: torch.Tensor) -> torch.Tensor:
    """Upper R with R^T R = the rows' damped mean Gram, in 64 bits."""
    gram = rows.double().T @ rows.double() / rows.shape[0]
    gram.diagonal().add_(0.01 * gram.diagonal().mean() + 1e-12)
    return torch.linalg.cholesky(gram).T.contiguous()


class Rounded:
    """W (out x in) as step * Z with integers |Z| <= 7, rounded under the Grams of
    the output gradients (rows of out) and inputs (rows of in)."""

    def __init__(self, W, inputs, gradients):
        self.step = float(W.abs().amax()) / 6.0
        factors = g.Factors.from_bases(gram_factor(gradients), gram_factor(inputs).T.contiguous())
        Z, _, objective = g.round_matrix(factors, W.double() / self.step)
        factors.close()
        self.Z = Z.clamp(-16, 16)
        self.objective = float(objective[0])
        self.blocks = g.block_quantize(self.Z.float(), 128, pow2=True)
        self.blocks.scales.mul_(self.step)

    def __call__(self, x):
        return g.block_linear(x, self.blocks)


def calibrate(weights, embed, tokens, target, kv_heads):
    """Of every matrix: the rows that it takes in, and the gradient of the targets'
    log probabilities at those that it gives out. tokens, target: sequences x length."""
    x = embed[tokens.flatten()]
    q, k, v = ((x @ weights[n].T).requires_grad_() for n in "qkv")
    seqs, t, dim = *tokens.shape, k.shape[1] // kv_heads
    split = lambda y: y.view(seqs, t, -1, dim).transpose(1, 2)
    kk, vv = (split(y).repeat_interleave(q.shape[1] // k.shape[1], 1) for y in (k, v))
    z = (split(q) @ kk.transpose(2, 3)) * dim ** -0.5
    ahead = torch.ones(t, t, dtype=torch.bool, device=x.device).triu(1)
    p = torch.softmax(z.masked_fill(ahead, float("-inf")), -1)
    attended = (p @ vv).transpose(1, 2).reshape(seqs * t, -1)
    o = attended @ weights["o"].T
    h = x + o
    logits = g.block_linear(h, g.block_quantize(weights["head"]))
    o.retain_grad()
    logits.retain_grad()
    g.token_logprobs(logits, target.flatten()).logprob.sum().backward()
    return {"q": (x, q.grad), "k": (x, k.grad), "v": (x, v.grad), "o": (attended.detach(), o.grad),
            "head": (h.detach(), logits.grad)}


def plain_attention(q, k, v, kv_heads, context, sees):
    """One sequence, 64 bits: rows of q over `context` tokens and the tree's."""
    t, dim = q.shape[0], k.shape[1] // kv_heads
    q = q.double().view(t, -1, dim)
    k, v = (x.double().view(-1, kv_heads, dim).repeat_interleave(q.shape[1] // kv_heads, 1) for x in (k, v))
    z = torch.einsum("thd,xhd->htx", q, k) * dim ** -0.5
    keep = torch.cat([torch.ones(t, context, dtype=torch.bool, device=q.device), sees], 1)
    p = torch.softmax(z.masked_fill(~keep, float("-inf")), -1)
    return torch.einsum("htx,xhd->thd", p, v).reshape(t, -1)


def decide(cache, table, prompt, words, parents, logits, gen, spare=4):
    """The tree's kept tokens, committed in a copy of the cache (with pages to spare), and the
    tables of two continuations of them."""
    width, before = parents.shape[1], cache
    cache = g.Cache(before.KC.shape[0] + spare, cache.heads, cache.page_size, cache.dim, cache.KC.dtype)
    for new, old in zip(cache.tensors, before.tensors):
        new.view(torch.uint8)[:old.shape[0]] = old.view(torch.uint8)
    context = torch.tensor([prompt], dtype=torch.int32, device="cuda")
    uniform = torch.rand(1, width, generator=gen, device="cuda")
    kept = g.tree_verify(logits, words[prompt:].view(1, -1).long(), parents, uniform=uniform)
    g.cache_commit([cache], table, context, kept.path)
    length = context + kept.count
    twice = torch.zeros(2, dtype=torch.int32, device="cuda")
    pages = g.pages_update(table, length, (length + width).repeat(2), cache.KC.shape[0], cache.page_size, source=twice)
    g.cache_copy([cache], pages.copies)
    return kept, pages, length, cache


def tune(head, h, target, index, count=2, rank=8, steps=4, rate=0.5):
    """Adapters beside a rounded head, by gradient steps on the targets' log probabilities;
    index: the adapter (the request's) of every row. Their gradients of the last step come back too."""
    N, K = head.blocks.codes.shape
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    A = (torch.randn(count, rank, K, generator=gen, device="cuda") / K ** 0.5).to(h.dtype).requires_grad_()
    B = torch.zeros(count, N, rank, dtype=h.dtype, device="cuda", requires_grad=True)
    groups = g.adapter_groups(index, count)
    with torch.no_grad():
        Y = head(h)
    for _ in range(steps):
        loss = -g.token_logprobs(g.adapters(h, A, B, groups, Y), target).logprob.mean()
        grads = torch.autograd.grad(loss, (A, B))
        with torch.no_grad():
            for t, d in zip((A, B), grads):
                t -= rate * d
    return A.detach(), B.detach(), groups, grads


def run(width=256, heads=8, kv_heads=2, vocab=1000, prompt=300, page_size=64, seed=0, dtype=torch.bfloat16):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    dim, kv_width = width // heads, width // heads * kv_heads
    weights = {"q": randn(width, width), "k": randn(kv_width, width), "v": randn(kv_width, width),
               "o": randn(width, width), "head": 4 * randn(vocab, width)}
    weights = {n: w / width ** 0.5 for n, w in weights.items()}
    embed = randn(vocab, width)

    # 1. calibration: sequences of tokens, each of which is to say a given one
    tokens, target = (torch.randint(vocab, (8, 128), generator=gen, device="cuda") for _ in range(2))
    seen = calibrate(weights, embed, tokens, target, kv_heads)

    # 2. and 3.: rounded and held in eight bits
    rounded = {n: Rounded(w, *seen[n]) for n, w in weights.items()}

    # 4. a prompt into the cache, then a tree of drafted tokens
    cache = g.Cache(-(-(prompt + 8) // page_size) + 1, kv_heads, page_size, dim)
    table = torch.arange(cache.KC.shape[0] - 1, -1, -1, dtype=torch.int32, device="cuda").view(1, -1)
    parents = torch.tensor([[-1, 0, 0, 1, 1, 2, 3, 5]], dtype=torch.int32, device="cuda")
    masks = g.tree_masks(parents)
    context = torch.tensor([prompt], dtype=torch.int32, device="cuda")
    words = torch.randint(vocab, (prompt + 8,), generator=gen, device="cuda")
    h = embed[words].to(dtype)
    k, v = rounded["k"](h), rounded["v"](h)
    cache.append(k, v, cache.slots(table, torch.zeros_like(context), prompt + 8))
    draft = h[prompt:].contiguous()
    attended, _ = cache.attend(rounded["q"](draft), table, context, masks)
    out = rounded["head"]((draft + rounded["o"](attended)).contiguous())

    # 5. every drafted token scores the next one of its branch; the tree's last ones any
    child = words[prompt:].roll(-1)
    served = g.token_logprobs(out, child, top=3)

    w = {n: m.double() for n, m in weights.items()}
    sees = torch.stack([((masks[0] >> u) & 1).bool() for u in range(8)], 1)
    he = embed[words].double()
    a = plain_attention(he[prompt:] @ w["q"].T, he @ w["k"].T, he @ w["v"].T, kv_heads, prompt, sees)
    ref = (he[prompt:] + a @ w["o"].T) @ w["head"].T
    exact = torch.log_softmax(ref, 1).gather(1, child.unsqueeze(1))[:, 0]
    kept, pages, length, later = decide(cache, table, prompt, words, parents, out, gen)
    head_in = seen["head"][0].to(dtype)
    index = (torch.arange(head_in.shape[0], device="cuda") * 2 // head_in.shape[0]).to(torch.int32)
    A, B, groups, grads = tune(rounded["head"], head_in, target.flatten(), index)
    tuned = g.adapters(head_in, A, B, groups, rounded["head"](head_in))
    return {"kept": kept, "pages": pages, "length": length, "later": later, "adapters": (A, B, groups, index, grads), "tuned": tuned,
            "head_in": head_in, "words": words, "parents": parents, "target": target,
            "served": served, "unrounded": exact, "logits": out, "reference": ref, "rounded": rounded,
            "weights": weights, "cache": cache, "k": k, "v": v, "table": table, "prompt": prompt}


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--vocab", type=int, default=1000)
    ap.add_argument("--prompt", type=int, default=300)
    args = ap.parse_args()
    r = run(width=args.width, vocab=args.vocab, prompt=args.prompt)
    for n, m in r["rounded"].items():
        print(f"{n}: {m.Z.shape[0]} x {m.Z.shape[1]}, integers in [{int(m.Z.min())}, {int(m.Z.max())}], "
              f"objective {m.objective:.4g}")
    print("drafted tokens, log probability rounded and served in eight bits / unrounded:")
    for a, b, e, t in zip(r["served"].logprob.tolist(), r["unrounded"].tolist(), r["served"].entropy.tolist(),
                          r["served"].ids.tolist()):
        print(f"  {a:9.4f} / {b:9.4f}   entropy {e:.3f}   most likely {t}")
    kept = r["kept"]
    print(f"kept {int(kept.count)} of the tree's tokens (places {kept.path[0, :int(kept.count)].tolist()}), then token "
          f"{int(kept.next)}; pages of two continuations {r['pages'].table.tolist()}, {int(r['pages'].left)} left")
    target = r["target"].flatten()
    plain = g.token_logprobs(r["rounded"]["head"](r["head_in"]), target).logprob.mean()
    print(f"calibration targets: mean log probability {float(plain):.4f} of the rounded head, "
          f"{float(g.token_logprobs(r['tuned'], target).logprob.mean()):.4f} with its adapters")


if __name__ == "__main__":
    main()
