"""Workloads of the 8-bit operators: norm, product and grouped product.

A graph network of many layers, or one whose nodes are of several types, keeps
a residual stream H and runs per layer ``H += layer(norm(H))``. Its dense half
at inference is three operators:

* ``norm``     h = x + r, y = h / sqrt(mean(h^2) + eps) * g, y cut into blocks
               of 128 along a row; a block is held as 8-bit floats (e4m3) and
               one scale, the power of two that brings its largest value to
               448 or less
* ``linear``   Y = act(A W^T) of two matrices held that way: A (M, K) with a
               scale for each row and 128 columns, W (N, K) with one for each
               128 x 128 block
* ``grouped``  the same with a weight for each group of rows (expert, node or
               relation type): rows offsets[e] .. offsets[e + 1] take W[e], rows
               past the last offset are 0

Plain torch operations compute them where ``own`` is false, the package's
entry points where it is true.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
EPS = 1e-6
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


def listed():
    return [
        # One token's residual stream at a step of generation: latency counts.
        dict(name="norm_token", op="norm", M=1, K=4096, dtype="bfloat16", residual=True),
        # A hidden layer of the benchmark's graph: many short rows.
        dict(name="norm_nodes", op="norm", M=230000, K=128, dtype="float32", residual=True),
        # Raw features of odd width, the first norm of a model: no residual yet.
        dict(name="norm_odd", op="norm", M=60000, K=601, dtype="float16", residual=False),
        # Prefill of a wide model: the residual stream far larger than any cache.
        dict(name="norm_large", op="norm", M=32768, K=8192, dtype="bfloat16", residual=True),
        # One token through a square projection: the weights are all the traffic.
        dict(name="linear_token", op="linear", M=1, K=4096, N=4096, dtype="bfloat16", act="none"),
        # A batch of single tokens, or of queried nodes, through a wide layer.
        dict(name="linear_batch", op="linear", M=48, K=8192, N=2048, dtype="bfloat16", act="relu"),
        # First layer of the benchmark's graph: wide raw features, many rows.
        dict(name="linear_nodes", op="linear", M=230000, K=602, N=256, dtype="float32", act="none"),
        # Prefill through a large layer: bound by the matrix cores.
        dict(name="linear_large", op="linear", M=16384, K=8192, N=8192, dtype="bfloat16",
             act="none"),
        # A batch of single tokens routed to many experts; the last rows of the
        # fixed batch are unused.
        dict(name="grouped_tokens", op="grouped", M=64, K=2048, N=1024, E=32, empty=4, spare=5,
             dtype="bfloat16", act="none"),
        # Node types of a typed graph, each with its weights, rows in type order.
        dict(name="grouped_types", op="grouped", M=230000, K=128, N=128, E=4, empty=0, spare=0,
             dtype="float32", act="relu"),
        # Class scores per relation: odd widths, packed rows, an empty type.
        dict(name="grouped_odd", op="grouped", M=5000, K=602, N=41, E=7, empty=1, spare=0,
             dtype="float16", act="none", packed=True),
        # Prefill through the experts: ragged shares of a long batch.
        dict(name="grouped_large", op="grouped", M=32768, K=4096, N=2048, E=64, empty=2, spare=0,
             dtype="bfloat16", act="none"),
    ]


#: No drawn case multiplies more, or holds more values, than the largest listed ones.
MOST_MNK = 16384 * 8192 * 8192
MOST_MK = 32768 * 8192
MOST_MN = 16384 * 8192
MOST_W = 64 * 4096 * 2048


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Widths: whole blocks of 128 (no third of them), odd multiples of 16, odd ones."""
    w, kind = _log(rng, lo, hi), rng.random()
    if kind < 0.5:
        blocks = max(1, w // 128)
        return 128 * (blocks + (blocks % 3 == 0))
    return w // 32 * 32 + 16 if kind < 0.75 else w | 1


def draw(rng):
    op = rng.choice(["norm", "linear", "grouped"])
    c = dict(op=op, M=_log(rng, 1, 250000), K=_width(rng, 16, 16384),
             dtype=rng.choice(["float32", "bfloat16", "float16"]))
    while c["M"] * c["K"] > MOST_MK // (2 if c["dtype"] == "float32" else 1):
        c["M"] = max(1, c["M"] // 2)
    if op == "norm":
        c["residual"] = rng.random() < 0.7
        return c
    c["N"], c["act"] = _width(rng, 8, 16384), rng.choice(["none", "none", "relu"])
    if op == "grouped":
        c["E"] = _log(rng, 1, 128)
        while c["E"] * c["K"] * c["N"] > MOST_W:
            c["E"], c["N"] = max(1, c["E"] // 2), max(8, c["N"] // 2)
        c["empty"] = rng.randint(0, c["E"] // 4)
        c["spare"] = rng.choice([0, 0, c["M"] // 10])
    while c["M"] * c["K"] * c["N"] > MOST_MNK // 2 or c["M"] * c["N"] > MOST_MN:
        c["M"] = max(1, c["M"] // 2)
        if "spare" in c:
            c["spare"] = min(c["spare"], c["M"] // 10)
    if rng.random() < 0.2:
        c["packed"] = True
    return c


# --- inputs ---------------------------------------------------------------------


def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(int(seed))


def _power(e):
    """2^e in float32, exactly, for whole e of -126 to 127."""
    return ((e + 127) << 23).view(torch.float32)


def _blocks(y):
    """Rows of y in blocks of 128, the last one filled up with zeros."""
    k = y.shape[-1]
    y = torch.nn.functional.pad(y, (0, -k % 128))
    return y.reshape(*y.shape[:-1], -1, 128)


def _exponent(amax):
    """The least e with amax <= 448 * 2^e, not below -126: 448 is 0.875 * 2^9."""
    m, e = torch.frexp(amax)
    e = e - 9 + (m > 0.875).to(e.dtype)
    return torch.where(amax > 0, e, torch.full_like(e, -126)).clamp(min=-126)


def _scales(e):
    return (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _quantize(y):
    """(q, s) of the float32 rows y: e4m3 values, and a power of two for each 128."""
    b = _blocks(y)
    e = _exponent(b.abs().amax(-1))
    q = (b * _power(-e)[..., None]).to(torch.float8_e4m3fn)
    return q.reshape(*y.shape[:-1], -1)[..., :y.shape[-1]], _scales(e)


def _quantize_weight(w):
    """(q, s) of float32 (..., N, K): a power of two for each 128 x 128 block."""
    n = w.shape[-2]
    b = _blocks(torch.nn.functional.pad(w, (0, 0, 0, -n % 128)))
    b = b.reshape(*b.shape[:-3], -1, 128, *b.shape[-2:])  # (..., NB, 128, KB, 128)
    e = _exponent(b.abs().amax((-3, -1)))
    q = (b * _power(-e)[..., None, :, None]).to(torch.float8_e4m3fn)
    q = q.reshape(*w.shape[:-2], -1, q.shape[-2] * 128)[..., :n, :w.shape[-1]]
    return q, _scales(e)


def _rows(q, packed):
    """q with rows that start on 16 bytes, as the quantiser lays them out, or packed."""
    if packed:
        return q.contiguous()
    k = q.shape[-1]
    to = torch.zeros((*q.shape[:-1], -(-k // 16) * 16), dtype=torch.uint8, device=DEVICE)
    to[..., :k] = q.view(torch.uint8) if q.is_contiguous() else q.contiguous().view(torch.uint8)
    return to.view(torch.float8_e4m3fn)[..., :k]


def _features(m, k, gen):
    """Rows of a residual stream: a few heavy features, row norms that differ."""
    x = torch.randn((m, k), generator=gen, device=DEVICE)
    heavy = torch.rand(k, generator=gen, device=DEVICE) < 0.01
    x *= torch.where(heavy, 12.0, 1.0)
    return x * torch.exp(torch.randn((m, 1), generator=gen, device=DEVICE))


def _sizes(case, seed):
    """Rows of each group, ragged, as a host list: the routing's shares."""
    gen = torch.Generator().manual_seed(int(seed))
    e, rows = case["E"], case["M"] - case["spare"]
    share = torch.rand(e, generator=gen, dtype=torch.float64) ** 2 + 0.1
    share[torch.randperm(e, generator=gen)[:case["empty"]]] = 0
    pick = torch.multinomial(share, rows, replacement=True, generator=gen) if rows else \
        torch.zeros(0, dtype=torch.int64)
    return torch.bincount(pick, minlength=e).tolist()


def prepare(case, seed):
    gen = _generator(seed)
    m, k, dtype = case["M"], case["K"], TYPES[case["dtype"]]
    s = {"case": case}
    if case["op"] == "norm":
        s["x"] = _features(m, k, gen).to(dtype)
        if m > 8:
            s["x"][m // 3] = 0  # a node without features
        if case["residual"]:
            s["r"] = _features(m, k, gen).mul_(0.3).to(dtype)
            if m > 8:
                s["r"][m // 3] = 0
        s["g"] = 1 + 0.2 * torch.randn(k, generator=gen, device=DEVICE)
        return s
    packed = case.get("packed", False)
    q, s["a_s"] = _quantize(_features(m, k, gen))
    s["a_q"] = _rows(q, packed)
    del q
    n = case["N"]
    shape = (case["E"], n, k) if case["op"] == "grouped" else (n, k)
    w = (torch.rand(shape, generator=gen, device=DEVICE) * 2 - 1) * math.sqrt(6.0 / (k + n))
    q, s["w_s"] = _quantize_weight(w)
    s["w_q"] = _rows(q, packed)
    if case["op"] == "grouped":
        sizes = _sizes(case, seed)
        s["offsets"] = torch.tensor([0] + sizes, device=DEVICE).cumsum(0).int()
        s["most"] = max(sizes)  # the plain form pads the groups to this many rows
    return s


# --- one pass ---------------------------------------------------------------------


def _values(q, s):
    """The float32 values that 8-bit rows and their scales stand for."""
    return q.float() * s.float().repeat_interleave(128, -1)[..., :q.shape[-1]]


def _weight_values(q, s):
    return _values(q, s.float().repeat_interleave(128, -2)[..., :q.shape[-2], :])


def _finish(y, case):
    if case["act"] == "relu":
        y = y.clamp(min=0)
    return y.to(TYPES[case["dtype"]])


def _plain(s):
    case = s["case"]
    if case["op"] == "norm":
        h = s["x"].float()
        if case["residual"]:
            h = h + s["r"].float()
        y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * s["g"]
        q, scale = _quantize(y)
        if not case["residual"]:
            return {"q": q, "s": scale}
        return {"q": q, "s": scale, "h": h.to(TYPES[case["dtype"]])}
    a, w = _values(s["a_q"], s["a_s"]), _weight_values(s["w_q"], s["w_s"])
    if case["op"] == "linear":
        return _finish(a @ w.t(), case)
    # Each group's rows, padded to the largest group, in one batched product.
    offsets, rows = s["offsets"].long(), torch.arange(case["M"], device=DEVICE)
    group = torch.searchsorted(offsets[1:], rows, right=True)
    used = group < case["E"]
    group = group.clamp(max=case["E"] - 1)
    place = torch.where(used, rows - offsets[group], torch.full_like(rows, s["most"]))
    padded = torch.zeros((case["E"], s["most"] + 1, case["K"]), device=DEVICE)
    padded[group, place] = a
    y = torch.bmm(padded, w.transpose(1, 2).contiguous())[group, place]
    return _finish(torch.where(used[:, None], y, torch.zeros_like(y)), case)


def run(s):
    if not own:
        return _plain(s)
    import paper_2308_11825_amd as agcn
    case = s["case"]
    if case["op"] == "norm":
        if not case["residual"]:
            q, scale = agcn.rms_norm(s["x"], s["g"], eps=EPS)
            return {"q": q, "s": scale}
        q, scale, h = agcn.rms_norm(s["x"], s["g"], residual=s["r"], eps=EPS)
        return {"q": q, "s": scale, "h": h}
    dtype = TYPES[case["dtype"]]
    if case["op"] == "linear":
        return agcn.quantized_linear(s["a_q"], s["a_s"], s["w_q"], s["w_s"], dtype=dtype,
                                     act=case["act"])
    return agcn.grouped_linear(s["a_q"], s["a_s"], s["w_q"], s["w_s"], s["offsets"], dtype=dtype,
                               act=case["act"])


# --- the work a pass cannot do without, and its results in 64 bits -----------------


def work(case):
    m, k = case["M"], case["K"]
    size, kb = 4 if case["dtype"] == "float32" else 2, -(-k // 128)
    if case["op"] == "norm":
        moved = 3 if case["residual"] else 1
        return {"bytes": m * k * (size * moved + 1) + m * kb + 4 * k, "flops": 6 * m * k}
    n, groups, rows = case["N"], case.get("E", 1) - case.get("empty", 0), m - case.get("spare", 0)
    groups = min(groups, max(rows, 1))  # weights that no row takes are not read
    weights = groups * (n * k + -(-n // 128) * kb)
    return {"bytes": rows * (k + kb) + weights + m * n * size, "flops": 2 * rows * n * k}


def _exact_product(a_q, a_s, w_q, w_s):
    """Sum over the blocks of 128 of (q_a q_w) s_a s_w, in float64."""
    m, k = a_q.shape
    n = w_q.shape[0]
    y = torch.zeros((m, n), dtype=torch.float64, device=DEVICE)
    block = torch.arange(n, device=DEVICE) // 128
    for b in range(-(-k // 128)):
        at = slice(128 * b, min(k, 128 * (b + 1)))
        part = a_q[:, at].double() @ w_q[:, at].double().t()
        part *= a_s[:, b].double()[:, None]
        part *= w_s[:, b].double()[block]
        y += part
    return y


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        h = s["x"].double()
        if case["residual"]:
            h = h + s["r"].double()
        y = h / torch.sqrt(torch.mean(h ** 2, dim=1, keepdim=True) + EPS) * s["g"].double()
        del s
        out = torch.empty_like(y)
        for at in range(0, case["K"], 128):
            part = y[:, at:at + 128]
            top = part.abs().amax(1, keepdim=True)
            e = torch.ceil(torch.log2(top / 448)).clamp(min=-126)
            out[:, at:at + 128] = part * torch.exp2(-torch.where(top > 0, e, torch.zeros_like(e)))
        # q: the real numbers that the 8 bits are the nearest of. The scale of a
        # block whose largest value is a rounding away from 448 * 2^e may be either.
        return {"q": out, "s": None, "h": h if case["residual"] else None}
    if case["op"] == "linear":
        y = _exact_product(s["a_q"], s["a_s"], s["w_q"], s["w_s"])
    else:
        y = torch.zeros((case["M"], case["N"]), dtype=torch.float64, device=DEVICE)
        at = 0
        for e, size in enumerate(_sizes(case, seed)):
            if size:
                y[at:at + size] = _exact_product(s["a_q"][at:at + size], s["a_s"][at:at + size],
                                                 s["w_q"][e], s["w_s"][e])
            at += size
    return y.clamp(min=0) if case["act"] == "relu" else y
