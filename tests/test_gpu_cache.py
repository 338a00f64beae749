"""The eight-bit cache through the C ABI: codes, scales and values read back are
those of the definition (tests/eightbit.py), bit for bit; what is not written
stays as it was."""
import pytest
import torch

from paper_2607_27042_amd import binding

import eightbit as eb

pytestmark = pytest.mark.gpu

CODE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def make_cache(pages, heads, page, dim, code):
    """Codes and scales that are NaN (or -128) where nothing was written."""
    fill = 0x7F if code == "e4m3" else 0x80
    codes = [torch.full((pages, heads, page, dim), fill, dtype=torch.uint8, device="cuda").view(CODE[code])
             for _ in range(2)]
    return codes + [torch.full((pages, heads, page), float("nan"), device="cuda") for _ in range(2)]


def _vectors(seed, tokens, heads, dim, dtype, pad, offset):
    g = _gen(seed)
    x = torch.randn(tokens, heads * dim, generator=g, device="cuda")
    x *= torch.exp2(torch.randint(-8, 9, (tokens, 1), generator=g, device="cuda").float())
    buf = torch.full((tokens, heads * dim + pad + offset), 99.0, dtype=eb.DTYPE[dtype], device="cuda")
    view = buf[:, offset:offset + heads * dim]
    view.copy_(x.clamp(-6e4, 6e4))
    return view, buf


def _as(q, s, dtype):
    return (q * s).float().to(eb.DTYPE[dtype])


@pytest.mark.parametrize("code", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("tokens,heads,dim,page", [(1, 1, 16, 16), (3, 2, 48, 48), (65, 5, 64, 16), (100, 8, 128, 64),
                                                   (33, 3, 144, 32), (257, 1, 256, 4096), (31, 2, 80, 112)])
def test_cache(tokens, heads, dim, page, dtype, code):
    print(f"[cache] {tokens}x{heads}x{dim} page {page} {dtype} {code}", flush=True)
    pages = -(-tokens // page) + 2
    for pad, offset in ((0, 0), (8, 8), (3, 1)):
        k, _ = _vectors(1, tokens, heads, dim, dtype, pad, offset)
        v, _ = _vectors(2, tokens, heads, dim, dtype, offset, pad)
        KC, VC, KS, VS = make_cache(pages, heads, page, dim, code)
        before = [t.view(torch.uint8).clone() for t in (KC, VC, KS, VS)]
        slots = torch.randperm(pages * page, generator=_gen(3), device="cuda")[:tokens]
        slots[::5] = torch.where(torch.arange(len(slots[::5]), device="cuda") % 2 == 0, -1, pages * page)
        if tokens > 4:
            slots[4] = 2 ** 40
        binding.gptq2d_cache_append(k, v, slots, KC, VC, KS, VS)
        live = (slots >= 0) & (slots < pages * page)
        at, off = slots[live] // page, slots[live] % page
        for x, C, S, was in ((k, KC, KS, before[0]), (v, VC, VS, before[1])):
            t = x.double().reshape(tokens, heads, dim)[live]
            s = eb.scale_of(t.abs().amax(-1), code)
            q = eb.codes_of(t, s[..., None], code)
            assert torch.equal(S[at, :, off].double(), s)
            got = C.view(torch.uint8)[at, :, off].view(CODE[code])
            assert torch.equal(got.double() if code == "int8" else got.float().double(), q)
            keep = torch.ones(pages, page, dtype=torch.bool, device="cuda")
            keep[at, off] = False
            assert torch.equal(C.view(torch.uint8).transpose(1, 2)[keep], was.transpose(1, 2)[keep])
            assert torch.isnan(S.transpose(1, 2)[keep]).all() and not torch.isnan(S[at, :, off]).any()
        k2, kb = _vectors(5, tokens, heads, dim, dtype, pad, offset)
        v2, vb = _vectors(6, tokens, heads, dim, dtype, offset, pad)
        kb0 = kb.clone()
        binding.gptq2d_cache_read(slots, KC, VC, KS, VS, k2, v2)
        for x, got in ((k, k2), (v, v2)):
            t = x.double().reshape(tokens, heads, dim)
            s = eb.scale_of(t.abs().amax(-1), code)
            want = _as(eb.codes_of(t, s[..., None], code), s[..., None], dtype).reshape(tokens, -1)
            want[~live] = 0
            assert torch.equal(got, want)
        hd = heads * dim
        assert torch.equal(kb[:, :offset], kb0[:, :offset]) and torch.equal(kb[:, offset + hd:], kb0[:, offset + hd:])


@pytest.mark.parametrize("code", ["e4m3", "int8"])
def test_vectors_that_are_not_finite(code):
    KC, VC, KS, VS = make_cache(2, 2, 16, 32, code)
    k = torch.randn(4, 64, device="cuda")
    v = torch.zeros(4, 64, device="cuda")
    k[0, 3] = float("nan")
    k[1, 40] = float("-inf")
    v[3, 0] = 1e-44
    slots = torch.tensor([0, 5, 17, 31], device="cuda")
    binding.gptq2d_cache_append(k, v, slots, KC, VC, KS, VS)
    bad = torch.zeros(4, 2, dtype=torch.bool, device="cuda")
    bad[0, 0] = bad[1, 1] = True
    assert torch.equal(torch.isnan(KS[slots // 16, :, slots % 16]), bad)
    codes = KC.view(torch.uint8)[slots // 16, :, slots % 16]
    assert (codes[bad] == 0).all() and (codes[~bad] != 0).any()
    assert torch.equal(VS[slots // 16, :, slots % 16][:3], torch.ones(3, 2, device="cuda"))
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    binding.gptq2d_cache_read(slots, KC, VC, KS, VS, k2, v2)
    assert torch.equal(torch.isnan(k2.view(4, 2, 32)).all(-1), bad) and not torch.isnan(v2).any()
    assert (v2[:3] == 0).all()


def test_offsets_past_32_bits():
    """Pages whose codes start past 2^32 bytes."""
    pages, heads, page, dim = 70000, 4, 64, 256  # 4.6 GB of codes each
    KC, VC = (torch.zeros(pages, heads, page, dim, dtype=torch.int8, device="cuda") for _ in range(2))
    KS, VS = (torch.zeros(pages, heads, page, device="cuda") for _ in range(2))
    k, v = (torch.randn(5, heads * dim, device="cuda") for _ in range(2))
    slots = torch.tensor([0, 65536 * 64, 69999 * 64 + 63, 33000 * 64 + 1, 68000 * 64 + 7], device="cuda")
    binding.gptq2d_cache_append(k, v, slots, KC, VC, KS, VS)
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    binding.gptq2d_cache_read(slots, KC, VC, KS, VS, k2, v2)
    for x, got in ((k, k2), (v, v2)):
        t = x.double().view(5, heads, dim)
        s = eb.scale_of(t.abs().amax(-1), "int8")
        assert torch.equal(got, _as(eb.codes_of(t, s[..., None], "int8"), s[..., None], "f32").view(5, -1))
    assert int((KC != 0).any(-1).sum()) == 5 * heads


def test_refusals():
    KC, VC, KS, VS = make_cache(2, 2, 16, 32, "int8")
    k, slots = torch.zeros(3, 64, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    with pytest.raises(TypeError, match="slots must be"):
        binding.gptq2d_cache_append(k, k, slots.int(), KC, VC, KS, VS)
    with pytest.raises(ValueError, match="slots must be"):
        binding.gptq2d_cache_append(k, k, slots[:2], KC, VC, KS, VS)
    with pytest.raises(TypeError, match="one dtype"):
        binding.gptq2d_cache_append(k, k.half(), slots, KC, VC, KS, VS)
    with pytest.raises(TypeError, match="float8_e4m3fn or both int8"):
        binding.gptq2d_cache_append(k, k, slots, KC.float(), VC, KS, VS)
    with pytest.raises(ValueError, match="K must be 3 x 64"):
        binding.gptq2d_cache_append(k[:, :32], k, slots, KC, VC, KS, VS)
    with pytest.raises(ValueError, match="KS and VS"):
        binding.gptq2d_cache_read(slots, KC, VC, KS[:1], VS, k, k)
    odd = make_cache(2, 2, 24, 32, "int8")
    with pytest.raises(binding.Gptq2dError, match="page_size"):
        binding.gptq2d_cache_append(k, k, slots, *odd)
    odd = make_cache(2, 2, 16, 24, "int8")
    with pytest.raises(binding.Gptq2dError, match="dim must be"):
        binding.gptq2d_cache_append(k[:, :48], k[:, :48], slots, *odd)
    # no tokens is no work
    binding.gptq2d_cache_append(k[:0], k[:0], slots[:0], KC, VC, KS, VS)
