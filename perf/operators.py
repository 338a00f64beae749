"""The eight-bit serving and scoring operators as cases to be timed.

A case is a dict of plain values. Its "op" names the operator:

  linear      Y = X W^T with X quantised to e4m3 in blocks of 1 x 128 on the way
              and W held in e4m3 with a scale for each 128 x 128 tile
  gradients   of that layer: dX from dY and the weights' transposed codes, dW
              from dY and X, both quantised along the tokens
  cache       keys and values written to a paged eight-bit cache, a scale for
              each token and head, then read back
  attention   a tree of drafted tokens over such a cache (one token: decoding)
  logprobs    of given tokens, with the entropy and the top alternatives;
              "train": with the gradient of the logits

`own` selects the library's kernels; otherwise the same is computed with
elementary torch operations in 32 bits.
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_ES = {"f32": 4, "f16": 2, "bf16": 2}
_TOP = {"e4m3": 448.0, "int8": 127.0}


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def _linear(op, tokens, n, k, dtype, pow2):
    return {"op": op, "tokens": tokens, "n": n, "k": k, "dtype": dtype, "pow2": pow2}


def _cache(tokens, heads, dim, page, code, dtype):
    return {"op": "cache", "tokens": tokens, "heads": heads, "dim": dim, "page": page, "code": code, "dtype": dtype}


def _attention(seqs, width, kv_heads, group, dim, context, page, code, dtype):
    return {"op": "attention", "seqs": seqs, "width": width, "kv_heads": kv_heads, "group": group, "dim": dim,
            "context": context, "page": page, "code": code, "dtype": dtype}


def _logprobs(rows, vocab, top, dtype, train):
    return {"op": "logprobs", "rows": rows, "vocab": vocab, "top": top, "dtype": dtype, "train": train}


def listed():
    cases = {
        # one token through a projection: a step of decoding, latency and the weights' bytes
        "linear 1x4096x4096 bf16": _linear("linear", 1, 4096, 4096, "bf16", False),
        # a ragged handful of tokens through a small odd layer
        "linear 333x1000x700 f16": _linear("linear", 333, 1000, 700, "f16", True),
        # a long prompt through an MLP's first matrix
        "linear 8192x11008x4096 bf16": _linear("linear", 8192, 11008, 4096, "bf16", False),
        # the backward pass of that matrix for a ragged batch of a tuning run
        "gradients 2047x11008x4096 bf16": _linear("gradients", 2047, 11008, 4096, "bf16", False),
        # one new token for each of 64 sequences
        "cache 64x8x128 e4m3 bf16": _cache(64, 8, 128, 64, "e4m3", "bf16"),
        # a batch of prompts
        "cache 32768x8x128 int8 f16": _cache(32768, 8, 128, 64, "int8", "f16"),
        # one sequence, one token: the latency of decoding
        "attention 1x1 over 4096 e4m3 bf16": _attention(1, 1, 8, 4, 128, 4096, 64, "e4m3", "bf16"),
        # drafted trees for a batch of mixed lengths, short pages, odd tree width
        "attention 16x13 over 8192 int8 f16": _attention(16, 13, 8, 4, 64, 8192, 16, "int8", "f16"),
        # a loaded server with long contexts and small trees
        "attention 32x8 over 32768 e4m3 bf16": _attention(32, 8, 8, 4, 128, 32768, 64, "e4m3", "bf16"),
        # the last logits of one sequence, as a server returns them
        "logprobs 1x32000 top 20 f32": _logprobs(1, 32000, 20, "f32", False),
        # a step of tuning: value and gradient, odd vocabulary
        "logprobs 2047x50257 train bf16": _logprobs(2047, 50257, 0, "bf16", True),
        # every token of a long evaluation text
        "logprobs 4096x128000 top 8 bf16": _logprobs(4096, 128000, 8, "bf16", False),
    }
    return [dict(c, name=name) for name, c in cases.items()]


def draw(rng):
    def size(lo, hi, step=1):
        d = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return max(lo, d // step * step)

    def layer():  # half as layers have them, half as they come
        return size(128, 11008, 128) if rng.random() < 0.5 else size(64, 11008)

    op = rng.choice(["linear", "linear", "gradients", "cache", "attention", "attention", "logprobs", "logprobs"])
    dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
    while True:
        if op in ("linear", "gradients"):
            c = _linear(op, size(1, 8192), layer(), layer(), dtype, rng.random() < 0.5)
            fits = c["tokens"] * c["n"] * c["k"] * (2 if op == "gradients" else 1) <= 3.6e11
        elif op == "cache":
            c = _cache(size(1, 32768), rng.randint(1, 16), 16 * rng.randint(2, 16), rng.choice([16, 32, 48, 64, 128]),
                       rng.choice(["e4m3", "int8"]), dtype)
            fits = c["tokens"] * c["heads"] * c["dim"] <= 33_000_000
        elif op == "attention":
            c = _attention(size(1, 64), size(1, 64), rng.randint(1, 16), rng.choice([1, 2, 3, 4, 5, 8, 16]),
                           rng.choice([32, 64, 64, 80, 96, 128, 128, 128, 192, 256]), size(16, 65536),
                           rng.choice([16, 32, 48, 64, 128]), rng.choice(["e4m3", "int8"]), dtype)
            cells = c["seqs"] * c["context"] * c["kv_heads"] * c["dim"]
            fits = cells <= 1_000_000_000 and cells * c["width"] * c["group"] <= 3.3e10
        else:
            c = _logprobs(size(1, 8192), size(128, 262144), rng.choice([0, 1, 5, 8, 20, 50]), dtype,
                          rng.random() < 0.4)
            fits = c["rows"] * c["vocab"] * (2 if c["train"] else 1) <= 500_000_000
        if fits and 3072 not in c.values():
            return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 29)
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _activations(g, rows, cols, dtype):
    """Gaussian with a few loud channels, as activations have them."""
    x = _normal(g, rows, cols)
    x *= torch.where(torch.rand(cols, generator=g, device="cuda") < 0.01, 20.0, 1.0)
    return x.to(dtype)


def _up(v, m):
    return -(-v // m) * m


def _lengths(case, g):
    """Tokens before the tree, for each sequence: the largest first, the others down to a quarter of it."""
    f = 0.25 + 0.75 * torch.rand(case["seqs"], generator=g, device="cuda", dtype=torch.float64)
    f[0] = 1.0
    return (f * case["context"]).long()


def _inputs(case, seed):
    g = _generator(seed)
    dt = _DT[case["dtype"]]
    s = {"case": case}
    if case["op"] in ("linear", "gradients"):
        m, n, k = case["tokens"], case["n"], case["k"]
        s["X"] = _activations(g, m, k, dt)
        W = _normal(g, n, k) / math.sqrt(k)
        # the weights as a checkpoint holds them: codes and a scale for each 128 x 128 tile
        if case["op"] == "linear":
            s["W"], s["WS"] = _weights(W, case["pow2"])
        else:
            s["dY"] = (1e-3 * _normal(g, m, n)).to(dt)
            s["W"], s["WS"] = _weights(W.T.contiguous(), case["pow2"])
    elif case["op"] == "cache":
        t, h, d, page = case["tokens"], case["heads"], case["dim"], case["page"]
        pages = -(-t // page) + 3
        s["K"] = _activations(g, t, h * d, dt)
        s["V"] = _normal(g, t, h * d).to(dt)
        s["slots"] = torch.randperm(pages, generator=g, device="cuda")[: -(-t // page)].repeat_interleave(page)[:t]
        s["slots"] = s["slots"] * page + torch.arange(t, device="cuda") % page
        for c in ("KC", "VC"):
            s[c] = torch.zeros(pages, h, page, d, dtype=_CODE[case["code"]], device="cuda")
        for c in ("KS", "VS"):
            s[c] = torch.ones(pages, h, page, device="cuda")
    elif case["op"] == "attention":
        b, t, h, d, page = case["seqs"], case["width"], case["kv_heads"], case["dim"], case["page"]
        s["context"] = _lengths(case, g).to(torch.int32)
        s["lengths"] = s["context"].tolist()
        need = [-(-(c + t) // page) for c in s["lengths"]]
        pages = sum(need) + 1
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        s["table"] = torch.zeros(b, max(need), dtype=torch.int32, device="cuda")
        at = 0
        for i, c in enumerate(need):
            s["table"][i, :c] = order[at:at + c]
            at += c
        s["Q"] = _normal(g, b * t, h * case["group"] * d).to(dt)
        for c in "KV":
            codes = torch.empty(pages, h, page, d, dtype=_CODE[case["code"]], device="cuda")
            scales = torch.empty(pages, h, page, device="cuda")
            step = max(1, 2 ** 26 // (h * page * d))
            for p in range(0, pages, step):
                v = _normal(g, min(step, pages - p), h, page, d)
                scales[p:p + step] = _scale(v.abs().amax(-1), _TOP[case["code"]], False)
                codes[p:p + step] = _code(v, scales[p:p + step].unsqueeze(-1), case["code"])
            s[c + "C"], s[c + "S"] = codes, scales
        # a tree: every token's parent is an earlier one, mostly a recent one, or the context (-1)
        back = (torch.rand(b, t, generator=g, device="cuda") ** 2 * 4).long() + 1
        parent = (torch.arange(t, device="cuda") - back).clamp(min=-1)
        mask = torch.zeros(b, t + 1, dtype=torch.int64, device="cuda")  # the last column stands for parent -1
        for u in range(t):
            bit = -(1 << 63) if u == 63 else 1 << u
            mask[:, u] = mask.gather(1, parent[:, u:u + 1] % (t + 1))[:, 0] | bit
        s["mask"] = mask[:, :t].contiguous()
        s["scale"] = 1.0 / math.sqrt(d)
    else:
        r, v = case["rows"], case["vocab"]
        s["X"] = torch.empty(r, v, dtype=dt, device="cuda")
        step = max(1, 2 ** 27 // v)
        for i in range(0, r, step):  # a language model's logits: wide, with a long right tail
            x = _normal(g, min(step, r - i), v)
            s["X"][i:i + step] = (2.0 * x + 0.4 * x * x * x.sign()).to(dt)
        s["target"] = torch.randint(v, (r,), generator=g, device="cuda")
        s["scale"] = 1.25
        s["g_logprob"] = _normal(g, r) / r
        s["g_entropy"] = 0.1 * _normal(g, r) / r
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        _plan(s)
    return s


# ---------------------------------------------------------------------------
# the library's calls
# ---------------------------------------------------------------------------

def _plan(s):
    """Outputs, workspaces and the prepared call, which a program keeps."""
    from paper_2607_27042_amd import binding

    c = s["case"]
    dt = _DT[c["dtype"]]

    def empty(*shape, dtype=dt):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    def space(size):
        return empty(max(size, 256), dtype=torch.uint8)

    if c["op"] == "linear":
        m, n, k = c["tokens"], c["n"], c["k"]
        s["out"] = (empty(m, n),)
        ws = space(binding.gptq2d_block_linear_workspace_size(m, n, k))
        s["call"] = binding.gptq2d_block_linear(s["X"], s["W"], s["WS"], s["out"][0], ws, pow2=c["pow2"], prepare=True)
    elif c["op"] == "gradients":
        m, n, k = c["tokens"], c["n"], c["k"]
        s["out"] = (empty(m, k), empty(n, k, dtype=torch.float32))
        ws = space(binding.gptq2d_block_linear_backward_workspace_size(m, n, k))
        s["call"] = binding.gptq2d_block_linear_backward(s["dY"], s["X"], s["W"], s["WS"], *s["out"], ws,
                                                         pow2=c["pow2"], prepare=True)
    elif c["op"] == "cache":
        cache = (s["KC"], s["VC"], s["KS"], s["VS"])
        back = empty(c["tokens"], c["heads"] * c["dim"]), empty(c["tokens"], c["heads"] * c["dim"])
        append = binding.gptq2d_cache_append(s["K"], s["V"], s["slots"], *cache, prepare=True)
        read = binding.gptq2d_cache_read(s["slots"], *cache, *back, prepare=True)
        s["out"] = back + (s["KS"], s["VS"])
        s["call"] = lambda: (append(), read())
    elif c["op"] == "attention":
        heads = c["kv_heads"] * c["group"]
        s["out"] = empty(*s["Q"].shape), empty(c["seqs"] * c["width"], heads, dtype=torch.float32)
        ws = space(binding.gptq2d_tree_attention_workspace_size(c["seqs"], c["width"], heads, c["kv_heads"], c["dim"]))
        s["call"] = binding.gptq2d_tree_attention(s["Q"], s["KC"], s["VC"], s["KS"], s["VS"], s["table"], s["context"],
                                                  None, s["mask"], s["scale"], *s["out"], ws, prepare=True)
    else:
        r, v, top = c["rows"], c["vocab"], c["top"]
        value = [empty(r, dtype=torch.float32) for _ in range(3)]
        best = [empty(r, top, dtype=torch.int32), empty(r, top, dtype=torch.float32)] if top else [None, None]
        ws = space(binding.gptq2d_token_logprobs_workspace_size(r, v, top))
        forward = binding.gptq2d_token_logprobs(s["X"], s["target"], s["scale"], *value, *best, ws, prepare=True)
        s["out"] = tuple(value) + (tuple(best) if top else ())
        s["call"] = forward
        if c["train"]:
            dX = empty(r, v)
            backward = binding.gptq2d_token_logprobs_backward(s["X"], s["target"], s["scale"], value[2], value[1],
                                                              s["g_logprob"], s["g_entropy"], dX, prepare=True)
            s["out"] += (dX,)
            s["call"] = lambda: (forward(), backward())


def run(s):
    if own:
        s["call"]()
        return s["out"]
    return _PLAIN[s["case"]["op"]](s)


# ---------------------------------------------------------------------------
# the same in elementary torch operations, 32 bits
# ---------------------------------------------------------------------------

_CODE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def _scale(amax, top, pow2):
    s = (amax * (1.0 / top)).clamp(min=2.0 ** -126)
    if pow2:
        mantissa, exponent = torch.frexp(s)
        s = torch.ldexp(torch.ones_like(s), exponent - (mantissa == 0.5).int())
    s = torch.where(amax == 0, torch.ones_like(s), s)
    return torch.where(torch.isfinite(amax), s, torch.full_like(s, float("nan")))


def _code(x, s, code):
    y = (x * torch.reciprocal(s)).clamp(-_TOP[code], _TOP[code])
    return y.to(torch.float8_e4m3fn) if code == "e4m3" else torch.round(y).to(torch.int8)


def _pad(x, rows, cols):
    return torch.nn.functional.pad(x, (0, cols - x.shape[1], 0, rows - x.shape[0]))


def _rows(x, pow2):
    """What the codes of 1 x 128 blocks stand for, in 32 bits."""
    r, c = x.shape
    b = _pad(x.float(), r, _up(c, 128)).view(r, -1, 128)
    s = _scale(b.abs().amax(-1, keepdim=True), 448.0, pow2)
    return (_code(b, s, "e4m3").float() * s).view(r, -1)[:, :c]


def _weights(w, pow2):
    """Codes (rows of a whole number of 16 bytes) and scales of 128 x 128 tiles."""
    r, c = w.shape
    t = _pad(w, _up(r, 128), _up(c, 128)).view(_up(r, 128) // 128, 128, -1, 128)
    s = _scale(t.abs().amax(3, keepdim=True).amax(1, keepdim=True), 448.0, pow2)
    q = _code(t, s, "e4m3").view(_up(r, 128), -1)[:r, :_up(c, 16)].contiguous()
    return q[:, :c], s[:, 0, :, 0].contiguous()


def _values(q, s):
    r, c = q.shape
    return q.float() * s.repeat_interleave(128, 0)[:r].repeat_interleave(128, 1)[:, :c]


def _plain_linear(s):
    c = s["case"]
    y = _rows(s["X"], c["pow2"]) @ _values(s["W"], s["WS"]).T
    return (y.to(_DT[c["dtype"]]),)


def _plain_gradients(s):
    c = s["case"]
    dx = _rows(s["dY"], c["pow2"]) @ _values(s["W"], s["WS"]).T
    dw = _rows(s["dY"].T, c["pow2"]) @ _rows(s["X"].T, c["pow2"]).T
    return dx.to(_DT[c["dtype"]]), dw


def _plain_cache(s):
    c = s["case"]
    t, h, d, page = c["tokens"], c["heads"], c["dim"], c["page"]
    at, off = s["slots"] // page, s["slots"] % page
    out = []
    for x, codes, scales in ((s["K"], s["KC"], s["KS"]), (s["V"], s["VC"], s["VS"])):
        x = x.float().view(t, h, d)
        a = _scale(x.abs().amax(-1), _TOP[c["code"]], False)
        codes.view(torch.uint8)[at, :, off] = _code(x, a.unsqueeze(-1), c["code"]).view(torch.uint8)
        scales[at, :, off] = a
        q = codes.view(torch.uint8)[at, :, off].view(codes.dtype)
        out.append((q.float() * scales[at, :, off].unsqueeze(-1)).view(t, h * d).to(_DT[c["dtype"]]))
    return out[0], out[1], s["KS"], s["VS"]


def _sequence(s, i, codes, scales):
    """Head by head, what sequence i's pages stand for: kv_heads x tokens x dim."""
    c = s["case"]
    n = s["lengths"][i] + c["width"]
    p = s["table"][i, : -(-n // c["page"])].long()
    v = codes.view(torch.uint8)[p].view(codes.dtype).float() * scales[p].unsqueeze(-1)
    return v.transpose(0, 1).reshape(c["kv_heads"], -1, c["dim"])[:, :n].contiguous()


def _visible(s, i):
    """width x tokens: which tokens a drafted one sees."""
    c = s["case"]
    tree = (s["mask"][i].unsqueeze(-1) >> torch.arange(c["width"], device="cuda")) & 1
    before = torch.ones(c["width"], s["lengths"][i], dtype=torch.bool, device="cuda")
    return torch.cat([before, tree.bool()], 1)


def _plain_attention(s):
    c = s["case"]
    t, h, g, d = c["width"], c["kv_heads"], c["group"], c["dim"]
    q = s["Q"].float().view(-1, t, h, g, d).permute(0, 2, 3, 1, 4).reshape(-1, h, g * t, d).contiguous()
    o = torch.empty(c["seqs"], t, h, g, d, device="cuda")
    lse = torch.empty(c["seqs"], t, h, g, device="cuda")
    for i in range(c["seqs"]):
        k, v = _sequence(s, i, s["KC"], s["KS"]), _sequence(s, i, s["VC"], s["VS"])
        z = (q[i] @ k.transpose(1, 2).contiguous()) * s["scale"]
        z = z.view(h, g, t, -1).masked_fill(~_visible(s, i), float("-inf"))
        m = z.amax(-1, keepdim=True)
        m = torch.where(m == float("-inf"), torch.zeros_like(m), m)
        e = torch.exp(z - m)
        l = e.sum(-1, keepdim=True)
        p = e / torch.where(l == 0, torch.ones_like(l), l)
        o[i] = (p.view(h, g * t, -1) @ v).view(h, g, t, d).permute(2, 0, 1, 3)
        lse[i] = (m + torch.log(l))[..., 0].permute(2, 0, 1)
    return o.view(-1, h * g * d).to(_DT[c["dtype"]]), lse.view(-1, h * g)


def _best(x, top):
    """The largest of each row, the lowest index first where they are equal."""
    bits = (x + 0.0).view(torch.int32).long()
    order = torch.where(bits < 0, -(bits & 0x7fffffff), bits)
    key = order * 2 ** 32 + (2 ** 30 - torch.arange(x.shape[1], device="cuda"))
    key = torch.topk(key, top, dim=1).values
    return (2 ** 30 - key % 2 ** 32).to(torch.int32)


def _plain_logprobs(s):
    c = s["case"]
    logprob, entropy, whole, ids, tops, grads = [], [], [], [], [], []
    step = max(1, 2 ** 28 // c["vocab"])
    for i in range(0, c["rows"], step):
        x = s["X"][i:i + step].float()
        z = x * s["scale"]
        m = z.amax(1, keepdim=True)
        lse = m + torch.log(torch.exp(z - m).sum(1, keepdim=True))
        lp = z - lse
        p = torch.exp(lp)
        h = -(p * torch.where(p == 0, torch.zeros_like(lp), lp)).sum(1, keepdim=True)
        y = s["target"][i:i + step].unsqueeze(1)
        logprob.append(lp.gather(1, y)[:, 0])
        entropy.append(h[:, 0])
        whole.append(lse[:, 0])
        if c["top"]:
            ids.append(_best(x, c["top"]))
            tops.append(lp.gather(1, ids[-1].long()))
        if c["train"]:
            ga, gh = s["g_logprob"][i:i + step].unsqueeze(1), s["g_entropy"][i:i + step].unsqueeze(1)
            d = -p * (ga + gh * (torch.where(p == 0, torch.zeros_like(lp), lp) + h))
            d.scatter_add_(1, y, ga)
            grads.append((d * s["scale"]).to(_DT[c["dtype"]]))
    out = [torch.cat(v) for v in (logprob, entropy, whole)]
    return tuple(out + ([torch.cat(ids), torch.cat(tops)] if c["top"] else [])
                 + ([torch.cat(grads)] if c["train"] else []))


_PLAIN = {"linear": _plain_linear, "gradients": _plain_gradients, "cache": _plain_cache,
          "attention": _plain_attention, "logprobs": _plain_logprobs}


# ---------------------------------------------------------------------------
# the same from the definitions, 64 bits
# ---------------------------------------------------------------------------
# A block's scale s is the 32-bit value nearest to amax times the 32-bit 1 / top,
# its codes those of the 32-bit product of x and the 32-bit 1 / s. Quotients and
# products of two 32-bit numbers round to 32 bits alike from 64.

def _exact_codes(x, dims, top, pow2):
    """(codes, scales) of x in 64 bits; the block runs over `dims`."""
    x = x.double()
    amax = x.abs().amax(dims, keepdim=True)
    s = (amax * torch.tensor(1.0 / top).float().double().item()).float().double().clamp(min=2.0 ** -126)
    if pow2:
        s = torch.exp2(torch.ceil(torch.log2(s)))
    s[amax == 0] = 1.0
    y = (x * (1.0 / s).float().double()).float().double().clamp(-top, top)
    if top == 127.0:
        return torch.round(y), s
    ulp = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / ulp) * ulp, s


def _exact_rows(x, pow2):
    r, c = x.shape
    full = torch.zeros(r, _up(c, 128), dtype=torch.float64, device=x.device)
    full[:, :c] = x
    q, s = _exact_codes(full.view(r, -1, 128), 2, 448.0, pow2)
    return (q * s).view(r, -1)[:, :c].contiguous()


def _exact_weights(q, s):
    w = q.double()
    for i in range(s.shape[0]):
        for j in range(s.shape[1]):
            w[128 * i:128 * i + 128, 128 * j:128 * j + 128] *= s[i, j].double()
    return w


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "linear":
        w = _exact_weights(s["W"], s["WS"])
        return (_exact_rows(s["X"], case["pow2"]) @ w.T,)
    if op == "gradients":
        w = _exact_weights(s["W"], s["WS"])
        dx = _exact_rows(s["dY"], case["pow2"]) @ w.T
        a, b = _exact_rows(s["dY"].T, case["pow2"]), _exact_rows(s["X"].T, case["pow2"])
        return dx, a @ b.T
    if op == "cache":
        t, h, d, page = case["tokens"], case["heads"], case["dim"], case["page"]
        back, scales = [], []
        for x, old in ((s["K"], s["KS"]), (s["V"], s["VS"])):
            q, a = _exact_codes(x.view(t, h, d), 2, _TOP[case["code"]], False)
            back.append((q * a).view(t, h * d))
            new = old.double()
            new[s["slots"] // page, :, s["slots"] % page] = a[:, :, 0]
            scales.append(new)
        return back[0], back[1], scales[0], scales[1]
    if op == "attention":
        t, h, g, d, page = case["width"], case["kv_heads"], case["group"], case["dim"], case["page"]
        o = torch.zeros(case["seqs"], t, h * g, d, dtype=torch.float64, device="cuda")
        lse = torch.zeros(case["seqs"], t, h * g, dtype=torch.float64, device="cuda")
        q = s["Q"].double().view(case["seqs"], t, h, g, d)
        for i in range(case["seqs"]):
            n = s["lengths"][i]
            pages = s["table"][i, :-(-(n + t) // page)].long()
            keep = torch.ones(t, n + t, dtype=torch.bool, device="cuda")
            for u in range(t):
                keep[:, n + u] = (s["mask"][i] & (-(1 << 63) if u == 63 else 1 << u)) != 0
            for j in range(h):
                k, v = ((s[c + "C"].view(torch.uint8)[pages, j].view(s[c + "C"].dtype).double()
                         * s[c + "S"][pages, j].double().unsqueeze(-1)).reshape(-1, d)[:n + t] for c in "KV")
                z = torch.matmul(q[i, :, j].reshape(t * g, d), k.T).view(t, g, -1) * s["scale"]
                z = torch.where(keep.unsqueeze(1), z, -float("inf"))
                lse[i, :, j * g:(j + 1) * g] = torch.logsumexp(z, -1)
                o[i, :, j * g:(j + 1) * g] = torch.matmul(torch.softmax(z, -1).view(t * g, -1), v).view(t, g, d)
        return o.view(-1, h * g * d), lse.view(-1, h * g)
    out = [[] for _ in range(6)]
    for i in range(0, case["rows"], 256):
        x = s["X"][i:i + 256].double()
        lp = torch.log_softmax(x * s["scale"], 1)
        y = s["target"][i:i + 256]
        n = torch.arange(len(y), device="cuda")
        p = lp.exp()
        h = -(p * lp).sum(1)
        out[0].append(lp[n, y])
        out[1].append(h)
        out[2].append(torch.logsumexp(x * s["scale"], 1))
        if case["top"]:
            ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :case["top"]]
            out[3].append(ids.to(torch.int32))
            out[4].append(lp.gather(1, ids))
        if case["train"]:
            ga, gh = s["g_logprob"][i:i + 256].double(), s["g_entropy"][i:i + 256].double()
            d = -p * (ga[:, None] + gh[:, None] * (lp + h[:, None]))
            d[n, y] += ga
            out[5].append(d * s["scale"])
    return tuple(torch.cat(v) for v in out if v)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    es = _ES[case["dtype"]]
    if case["op"] in ("linear", "gradients"):
        m, n, k = float(case["tokens"]), float(case["n"]), float(case["k"])
        w = n * k + 4 * math.ceil(n / 128) * math.ceil(k / 128)
        if case["op"] == "linear":
            return {"bytes": es * m * (k + n) + w, "flops": 2 * m * n * k}
        return {"bytes": es * m * (n + k + k) + w + 4 * n * k, "flops": 4 * m * n * k}
    if case["op"] == "cache":
        vectors = 2.0 * case["tokens"] * case["heads"]
        return {"bytes": vectors * (case["dim"] * (2 * es + 2) + 8) + 16 * case["tokens"],
                "flops": 4 * vectors * case["dim"]}
    if case["op"] == "attention":
        # the lengths spread evenly from a quarter of the largest to all of it
        tokens = case["context"] * (1 + 0.625 * (case["seqs"] - 1)) + case["seqs"] * case["width"]
        rows = float(case["seqs"] * case["width"] * case["kv_heads"] * case["group"])
        return {"bytes": 2 * tokens * case["kv_heads"] * (case["dim"] + 4) + rows * (2 * es * case["dim"] + 4),
                "flops": 4 * tokens * case["width"] * case["kv_heads"] * case["group"] * case["dim"]}
    cells = float(case["rows"]) * case["vocab"]
    out = case["rows"] * (20 + 8 * case["top"])
    if case["train"]:
        return {"bytes": 2 * es * cells + out + 8 * case["rows"], "flops": 9 * cells}
    return {"bytes": es * cells + out, "flops": 5 * cells}
