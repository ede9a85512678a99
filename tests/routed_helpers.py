"""Shared by the tests of the routed layer's operators: inputs, and the operators' plain forms
in 64 bits, on whatever device the tensors are."""
import torch

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
U = 2.0 ** -24


def half_step(dtype):
    """A rounding to `dtype` is off by this at most, relative to the value."""
    return torch.finfo(dtype).eps / 2


def tiniest(dtype):
    """Half of the least subnormal: what a rounding near 0 is off by at most."""
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def gen(*seed, device="cuda:0"):
    s = 0
    for x in seed:
        s = s * 1000003 + int(x)
    return torch.Generator(device=device).manual_seed(s % (1 << 40))


def randn(shape, dtype, *seed, device="cuda:0"):
    return torch.randn(shape, generator=gen(*shape, *seed, device=device), device=device).to(dtype)


def padded(t, pad, offset=0):
    """A copy of t with `pad` more columns a row, starting `offset` elements into its storage,
    with values around it that spoil any result they get into."""
    n, f = t.shape
    fill = float("nan") if t.is_floating_point() else 77
    raw = torch.full((offset + n * (f + pad),), fill, device=t.device).to(t.dtype)
    v = raw[offset:].view(n, f + pad)[:, :f]
    v.copy_(t)
    return v


def sort(ids, groups):
    """(offsets, place) slot by slot, as the header defines them."""
    flat = [e if 0 <= e < groups else groups for e in ids.reshape(-1).tolist()]
    count = [0] * (groups + 2)
    for e in flat:
        count[e + 1] += 1
    for e in range(groups + 1):
        count[e + 1] += count[e]
    offsets, place = count[:groups + 1], []
    for e in flat:
        place.append(count[e] if e < groups else -1 - count[e])
        count[e] += 1
    return (torch.tensor(offsets, dtype=torch.int32, device=ids.device),
            torch.tensor(place, dtype=torch.int32, device=ids.device).view(ids.shape))


def rows_of(place):
    return torch.where(place < 0, -1 - place, place).long(), place >= 0


def dispatch(X, place):
    row, kept = rows_of(place)
    Y = torch.zeros((place.numel(), X.shape[1]), dtype=X.dtype, device=X.device)
    for c in range(place.shape[1]):
        Y[row[kept[:, c], c]] = X[kept[:, c]]
    return Y


def combine(R, place, w):
    """The sum in 64 bits, and the sum of its terms' sizes."""
    row, kept = rows_of(place)
    out = torch.zeros((place.shape[0], R.shape[1]), dtype=torch.float64, device=R.device)
    size = torch.zeros_like(out)
    for c in range(place.shape[1]):
        t = kept[:, c]
        part = R[row[t, c]].double() * w[t, c].double()[:, None]
        out[t] += part
        size[t] += part.abs()
    return out, size


def norm(h, g, b, eps):
    """(y, xh, mean, 1 / sqrt(var + eps)) of float64 rows h."""
    mean = h.mean(1, keepdim=True)
    rs = 1 / torch.sqrt(((h - mean) ** 2).mean(1, keepdim=True) + eps)
    xh = (h - mean) * rs
    return xh * g + b, xh, mean, rs


def norm_grad(dy, h, stats, g):
    """dx, dg, db in 64 bits with the given statistics."""
    xh = (h.double() - stats[:, :1].double()) * stats[:, 1:].double()
    d = dy.double() * g.double()
    dx = stats[:, 1:].double() * (d - d.mean(1, keepdim=True) - xh * (d * xh).mean(1, keepdim=True))
    return dx, (dy.double() * xh).sum(0), dy.double().sum(0)
