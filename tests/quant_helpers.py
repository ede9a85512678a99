"""Plain 64-bit forms of the 8-bit operators, for their tests: blocks, scales and
values as the header defines them, on whatever device the tensors are."""
import torch

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


def exponent(amax):
    """The least e >= -126 with amax <= 448 * 2^e (float64 amax, finite)."""
    m, e = torch.frexp(amax.double())
    e = e + (m > 0.875) - 9
    return torch.where(amax > 0, e, torch.full_like(e, -126)).clamp(min=-126)


def finite_amax(y, dim):
    return torch.where(torch.isfinite(y), y.abs(), torch.zeros_like(y)).amax(dim)


def row_blocks(y):
    y = torch.nn.functional.pad(y, (0, -y.shape[1] % 128))
    return y.reshape(y.shape[0], -1, 128)


def power(e):
    """2^e in float64, exactly (torch.ldexp goes through a float32 power)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def quantize_rows(y):
    """(q in float64, e) of float64 rows whose products with powers of two are exact:
    values rounded to e4m3 to nearest even, infinities and NaN as NaN."""
    b = row_blocks(y)
    e = exponent(finite_amax(b, -1))
    q = round_e4m3(b * power(-e)[..., None])
    return q.reshape(y.shape[0], -1)[:, :y.shape[1]], e


def step(v):
    """Distance of neighbouring e4m3 values around |v| <= 448: 2^-9 at the least."""
    _, e = torch.frexp(v.abs().clamp(min=2.0 ** -6))
    return power(e - 4)


def round_e4m3(v):
    s = step(v)
    return torch.where(torch.isfinite(v), torch.round(v / s) * s, torch.full_like(v, float("nan")))


def scales(S):
    """Exponents of a tensor of scales."""
    return S.view(torch.uint8).to(torch.int32) - 127


def values(Q, S):
    s = torch.where(S.view(torch.uint8) == 255, torch.nan, power(scales(S)))
    return Q.double() * s.repeat_interleave(128, -1)[..., :Q.shape[-1]]


def weight_values(Q, S):
    s = torch.where(S.view(torch.uint8) == 255, torch.nan, power(scales(S)))
    s = s.repeat_interleave(128, -2)[..., :Q.shape[-2], :]
    return Q.double() * s.repeat_interleave(128, -1)[..., :Q.shape[-1]]
