"""Plain 64-bit counterparts of the eight-bit operators (oracle of their tests).

Scales and codes are defined through 32-bit products; a product (quotient) of
two 32-bit numbers rounds to 32 bits the same from its 64-bit value."""
import torch

TOP = {"e4m3": 448.0, "int8": 127.0}
DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# half the distance between neighbouring results, relative
HALF_ULP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def fl(x):
    return x.float().double()


def scale_of(amax, code="e4m3", pow2=False):
    inv = fl(torch.tensor(1.0 / TOP[code], dtype=torch.float64, device=amax.device))
    s = fl(amax.double() * inv).clamp(min=2.0 ** -126)
    if pow2:
        s = torch.exp2(torch.ceil(torch.log2(s)))
    s = torch.where(amax == 0, torch.ones_like(s), s)
    return torch.where(torch.isfinite(amax), s, torch.full_like(s, float("nan")))


def codes_of(x, s, code="e4m3"):
    """The values of the codes (64 bits) of x with scales s that broadcast."""
    y = fl(x.double() * fl(1.0 / s)).clamp(-TOP[code], TOP[code])
    if code == "int8":
        q = torch.round(y)
    else:
        ulp = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
        q = torch.round(y / ulp) * ulp
    return torch.where(torch.isnan(s.expand_as(q)), torch.zeros_like(q), q)


def blocks(x, block_rows=1, pow2=False):
    """(code values, scales [row blocks, column blocks]) of e4m3 blocks."""
    r, c = x.shape
    R, C = -(-r // block_rows), -(-c // 128)
    full = torch.zeros(R * block_rows, C * 128, dtype=torch.float64, device=x.device)
    full[:r, :c] = x.double()
    t = full.view(R, block_rows, C, 128)
    amax = t.abs().amax((1, 3))
    bad = torch.isnan(t).any(3).any(1)
    s = scale_of(torch.where(bad, torch.full_like(amax, float("nan")), amax), pow2=pow2)
    q = codes_of(torch.nan_to_num(t, posinf=0, neginf=0), s[:, None, :, None])
    return q.view(R * block_rows, C * 128)[:r, :c].contiguous(), s


def spread(s, rows, cols, block_rows):
    return s.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)[:, :cols]


def values(x, block_rows=1, pow2=False):
    q, s = blocks(x, block_rows, pow2)
    return q * spread(s, *x.shape, block_rows)


def up(v, m):
    return -(-v // m) * m


def empty_codes(rows, cols, extra=0):
    """e4m3 codes with rows on 16-byte boundaries, filled with NaN codes."""
    buf = torch.full((rows, up(cols, 16) + extra), 0x7F, dtype=torch.uint8, device="cuda")
    return buf.view(torch.float8_e4m3fn)[:, :cols]


def to_codes(q, s, cols_scales_first):
    """Device tensors (codes, scales) as the library takes them."""
    out = empty_codes(*q.shape)
    out.copy_(q.float().to(torch.float8_e4m3fn))
    return out, (s.T if cols_scales_first else s).float().contiguous().to(q.device)
