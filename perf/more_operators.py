"""Workloads of the routed layer's operators: layer norm, groups, integer products.

A layer that sends each row (token, node) to a few of many weights (experts,
types) normalises the rows, sorts them by group, multiplies each group by its
weight, and adds the results up per row. In training its first and last parts
have gradients. Its operators here:

* ``norm``       h = x + r, y = (h - mean) / sqrt(var + eps) * g + b per row, and the
                 rows' mean and 1 / sqrt(var + eps)
* ``norm_grad``  its gradients: of h (with the residual stream's own added), g and b
* ``route``      k group ids a row -> where each of the n k slots goes in group order
                 (stable), the groups' offsets, and the rows laid out that way. An id
                 outside [0, groups) drops its slot: it goes past the last offset,
                 its place is written as -1 - place, and its row is 0
* ``combine``    out[t] = sum over c of weight[t][c] rows[place[t][c]], dropped slots
                 left out; with ``grad`` its gradients, of the rows and the weights
* ``linear``     Y = act(A W^T) with A's rows in 8-bit integers with a scale each
                 (made in the call) and W's rows too (made once)
* ``grouped``    the same with a weight for each group of rows

Plain torch operations compute them where ``own`` is false, the package's
entry points where it is true.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
EPS = 1e-5
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


def listed():
    return [
        # One token's residual stream at a step of generation: latency counts.
        dict(name="norm_token", op="norm", n=1, f=4096, dtype="bfloat16", params="bfloat16",
             bias=True, residual=True),
        # Prefill or training of a wide model: rows far larger than any cache.
        dict(name="norm_large", op="norm", n=32768, f=8192, dtype="bfloat16", params="float32",
             bias=True, residual=True),
        # A hidden layer of the benchmark's graph in training: many short rows.
        dict(name="norm_grad_nodes", op="norm_grad", n=230000, f=128, dtype="float32",
             params="float32", bias=True, residual=True),
        # Raw features of odd width, the first norm of a model: no residual stream yet.
        dict(name="norm_grad_odd", op="norm_grad", n=60000, f=601, dtype="float16",
             params="float32", bias=True, residual=False),
        # A batch of single tokens sent to a few of many experts.
        dict(name="route_batch", op="route", n=48, f=2048, k=4, groups=64, dropped=0.0,
             dtype="bfloat16"),
        # A long prefill's tokens; some slots fell to experts that are elsewhere.
        dict(name="route_large", op="route", n=32768, f=4096, k=8, groups=128, dropped=0.03,
             dtype="bfloat16"),
        # Nodes of a graph with two relations each, odd width, back in their order.
        dict(name="combine_nodes", op="combine", n=60000, f=601, k=2, groups=7, dropped=0.1,
             dtype="float16", weights=True, grad=False),
        # A training batch's way back through the experts' sum.
        dict(name="combine_grad", op="combine", n=16384, f=4096, k=8, groups=64, dropped=0.0,
             dtype="bfloat16", weights=True, grad=True),
        # One token through a square projection: the weights are all the traffic.
        dict(name="linear_token", op="linear", n=1, fin=4096, fout=4096, dtype="bfloat16",
             act="none"),
        # Prefill through a large layer: bound by the matrix cores.
        dict(name="linear_large", op="linear", n=16384, fin=8192, fout=8192, dtype="bfloat16",
             act="none"),
        # Class scores per relation: odd widths, packed weights, an empty type, unused rows.
        dict(name="grouped_odd", op="grouped", n=5000, fin=602, fout=41, groups=7, empty=1,
             spare=100, dtype="float32", act="relu", packed=True),
        # Prefill through the experts: ragged shares of a long batch.
        dict(name="grouped_large", op="grouped", n=32768, fin=4096, fout=2048, groups=64, empty=2,
             spare=0, dtype="bfloat16", act="none"),
    ]


#: No drawn case holds more values, or multiplies more, than the largest listed ones.
MOST_NF = 32768 * 8192
MOST_SLOTS = 32768 * 8 * 4096
MOST_SLOTS_GRAD = 16384 * 8 * 4096
MOST_MNK = 16384 * 8192 * 8192
MOST_MN = 16384 * 8192
MOST_W = 64 * 4096 * 2048


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Widths: multiples of 128 (no third of them), odd multiples of 16, odd ones."""
    w, kind = _log(rng, lo, hi), rng.random()
    if kind < 0.5:
        blocks = max(1, w // 128)
        return 128 * (blocks + (blocks % 3 == 0))
    return w // 32 * 32 + 16 if kind < 0.75 else w | 1


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "route", "combine", "linear", "grouped"])
    c = dict(op=op, n=_log(rng, 1, 250000), dtype=rng.choice(["float32", "bfloat16", "float16"]))
    size = 2 if c["dtype"] == "float32" else 1
    if op in ("norm", "norm_grad"):
        c.update(f=_width(rng, 16, 16384), params=rng.choice(["float32", c["dtype"]]),
                 bias=rng.random() < 0.8, residual=rng.random() < 0.6)
        while c["n"] * c["f"] > MOST_NF // size // (2 if op == "norm_grad" else 1):
            c["n"] = max(1, c["n"] // 2)
        return c
    if op in ("route", "combine"):
        c.update(f=_width(rng, 16, 8192), k=rng.choice([1, 2, 4, 6, 8, 10]),
                 groups=_log(rng, 1, 1024), dropped=rng.choice([0.0, 0.0, 0.05, 0.5]))
        if op == "combine":
            c.update(weights=True, grad=rng.random() < 0.5)
            if not c["grad"]:  # without weights: the gradient of laying the rows out
                c["weights"] = rng.random() < 0.7
        while c["n"] * c["k"] * c["f"] > (MOST_SLOTS_GRAD if c.get("grad") else MOST_SLOTS) // size:
            c["n"] = max(1, c["n"] // 2)
        return c
    c.update(fin=_width(rng, 16, 16384), fout=_width(rng, 8, 16384),
             act=rng.choice(["none", "none", "relu"]))
    if op == "grouped":
        c["groups"] = _log(rng, 1, 128)
        while c["groups"] * c["fin"] * c["fout"] > MOST_W:
            c["groups"], c["fout"] = max(1, c["groups"] // 2), max(8, c["fout"] // 2)
        c["empty"] = rng.randint(0, c["groups"] // 4)
        c["spare"] = rng.choice([0, 0, c["n"] // 10])
    while (c["n"] * c["fin"] * c["fout"] > MOST_MNK // 2 or c["n"] * c["fout"] > MOST_MN
           or c["n"] * c["fin"] > MOST_NF // 2 // size):
        c["n"] = max(1, c["n"] // 2)
        if "spare" in c:
            c["spare"] = min(c["spare"], c["n"] // 10)
    if rng.random() < 0.2:
        c["packed"] = True
    return c


# --- inputs ---------------------------------------------------------------------


def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(int(seed))


def _features(n, f, gen):
    """Rows of a residual stream: a few heavy features, row norms and means that differ."""
    x = torch.randn((n, f), generator=gen, device=DEVICE)
    heavy = torch.rand(f, generator=gen, device=DEVICE) < 0.01
    x *= torch.where(heavy, 12.0, 1.0)
    x += 0.5 * torch.randn((n, 1), generator=gen, device=DEVICE)
    return x.mul_(torch.exp(torch.randn((n, 1), generator=gen, device=DEVICE)))


def _ids(case, gen):
    """k group ids for each row: popular groups and rare ones, distinct in a row where the
    groups are enough; a share of them dropped (-1)."""
    n, k, groups = case["n"], case["k"], case["groups"]
    score = torch.rand((n, groups), generator=gen, device=DEVICE)
    score *= 0.2 + torch.rand(groups, generator=gen, device=DEVICE)
    ids = score.topk(min(k, groups), dim=1).indices
    ids = ids.repeat(1, -(-k // groups))[:, :k] if k > groups else ids
    if case["dropped"]:
        out = torch.rand((n, k), generator=gen, device=DEVICE) < case["dropped"]
        ids = torch.where(out, torch.full_like(ids, -1), ids)
    return ids.int().contiguous()


def _sizes(case, seed):
    """Rows of each group, ragged, as a host list: the routing's shares."""
    gen = torch.Generator().manual_seed(int(seed))
    e, rows = case["groups"], case["n"] - case["spare"]
    share = torch.rand(e, generator=gen, dtype=torch.float64) ** 2 + 0.1
    share[torch.randperm(e, generator=gen)[:case["empty"]]] = 0
    pick = torch.multinomial(share, rows, replacement=True, generator=gen) if rows else \
        torch.zeros(0, dtype=torch.int64)
    return torch.bincount(pick, minlength=e).tolist()


def _quantize(x):
    """8-bit integers and a scale for each row of the float32 x. (Quotients of tensors: a
    number's quotient with a tensor is a product with a rounded reciprocal.)"""
    top = x.abs().amax(-1)
    most = torch.full_like(top, 127)
    factor = most / torch.where(top > 0, top, torch.ones_like(top))
    return torch.round(x * factor[..., None]), top / most


def _aligned(q):
    """Rows of q that start on 16 bytes."""
    k = q.shape[-1]
    to = torch.zeros((*q.shape[:-1], -(-k // 16) * 16), dtype=torch.int8, device=DEVICE)
    to[..., :k] = q
    return to[..., :k]


def prepare(case, seed):
    gen = _generator(seed)
    op, n, dtype = case["op"], case["n"], TYPES[case["dtype"]]
    s = {"case": case}
    if op in ("norm", "norm_grad"):
        f, params = case["f"], TYPES[case["params"]]
        s["x"] = _features(n, f, gen).to(dtype)
        if n > 8:
            s["x"][n // 3] = 0  # a node without features
        s["g"] = (1 + 0.2 * torch.randn(f, generator=gen, device=DEVICE)).to(params)
        s["b"] = (0.1 * torch.randn(f, generator=gen, device=DEVICE)).to(params) if case["bias"] \
            else None
        if op == "norm":
            if case["residual"]:
                s["r"] = _features(n, f, gen).mul_(0.3).to(dtype)
            return s
        mean = s["x"].float().mean(-1, keepdim=True)
        h = s["x"].float() - mean
        s["stats"] = torch.cat([mean, torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS)], 1)
        del h
        s["dy"] = torch.randn((n, f), generator=gen, device=DEVICE).to(dtype)
        if case["residual"]:
            s["dh"] = torch.randn((n, f), generator=gen, device=DEVICE).to(dtype)
        return s
    if op in ("route", "combine"):
        ids, f, k = _ids(case, gen), case["f"], case["k"]
        if op == "route":
            s["ids"], s["x"] = ids, _features(n, f, gen).to(dtype)
            return s
        s["place"] = _sort(ids, case["groups"])[1]
        s["rows"] = torch.randn((n * k, f), generator=gen, device=DEVICE, dtype=dtype)
        if case["weights"]:
            w = torch.randn((n, k), generator=gen, device=DEVICE)
            s["w"] = torch.exp(w) / torch.exp(w).sum(1, keepdim=True)
        if case["grad"]:
            s["dout"] = torch.randn((n, f), generator=gen, device=DEVICE, dtype=dtype)
        return s
    fin, fout = case["fin"], case["fout"]
    s["x"] = _features(n, fin, gen).to(dtype)
    if n > 8:
        s["x"][n // 3] = 0
    shape = (case["groups"], fout, fin) if op == "grouped" else (fout, fin)
    w = (torch.rand(shape, generator=gen, device=DEVICE) * 2 - 1) * math.sqrt(6.0 / (fin + fout))
    q, s["ws"] = _quantize(w)
    s["wq"] = q.to(torch.int8) if case.get("packed") else _aligned(q)
    if op == "grouped":
        sizes = _sizes(case, seed)
        s["offsets"] = torch.tensor([0] + sizes, device=DEVICE).cumsum(0).int()
        s["most"] = max(sizes)  # the plain form pads the groups to this many rows
    return s


# --- one pass ---------------------------------------------------------------------


def _sort(ids, groups):
    """(offsets, place) of the slots in group order."""
    key = ids.reshape(-1)
    key = torch.where((key >= 0) & (key < groups), key, torch.full_like(key, groups))
    key, order = torch.sort(key, stable=True)
    at = torch.arange(key.numel(), dtype=torch.int32, device=DEVICE)
    place = torch.empty_like(at)
    place[order] = torch.where(key < groups, at, -1 - at)
    ends = torch.searchsorted(key, torch.arange(groups + 1, dtype=key.dtype, device=DEVICE))
    return ends.int(), place.view(ids.shape)


def _rows_of(place):
    """Rows that the places name, and whether each slot is kept."""
    return torch.where(place < 0, -1 - place, place).long(), place >= 0


def _plain_norm(s, case):
    h = s["x"].float()
    if case["residual"]:
        h = h + s["r"].float()
    mean = h.mean(-1, keepdim=True)
    c = h - mean
    scale = torch.rsqrt((c * c).mean(-1, keepdim=True) + EPS)
    y = c * scale * s["g"].float()
    if s["b"] is not None:
        y = y + s["b"].float()
    dtype = TYPES[case["dtype"]]
    out = {"y": y.to(dtype), "stats": torch.cat([mean, scale], 1)}
    if case["residual"]:
        out["h"] = h.to(dtype)
    return out


def _plain_norm_grad(s, case):
    mean, scale = s["stats"][:, :1], s["stats"][:, 1:]
    c = (s["x"].float() - mean) * scale
    dy = s["dy"].float()
    params = TYPES[case["params"]]
    out = {"dg": (dy * c).sum(0).to(params)}
    if s["b"] is not None:
        out["db"] = dy.sum(0).to(params)
    dc = dy * s["g"].float()
    dx = scale * (dc - dc.mean(-1, keepdim=True) - c * (dc * c).mean(-1, keepdim=True))
    if case["residual"]:
        dx = dx + s["dh"].float()
    out["dx"] = dx.to(TYPES[case["dtype"]])
    return out


def _plain_combine(s, case):
    rows, kept = _rows_of(s["place"])
    n, k, dtype = case["n"], case["k"], TYPES[case["dtype"]]
    if not case["grad"]:
        out = torch.zeros((n, case["f"]), device=DEVICE)
        for c in range(k):
            part = s["rows"][rows[:, c]].float()
            if case["weights"]:
                part = part * s["w"][:, c:c + 1]
            out = out + torch.where(kept[:, c:c + 1], part, torch.zeros_like(part))
        return {"out": out.to(dtype)}
    dout = s["dout"].float()
    drows, dw = torch.empty_like(s["rows"]), []
    for c in range(k):
        here = kept[:, c:c + 1]
        drows[rows[:, c]] = torch.where(here, dout * s["w"][:, c:c + 1],
                                        torch.zeros_like(dout)).to(dtype)
        part = (dout * s["rows"][rows[:, c]].float()).sum(1, keepdim=True)
        dw.append(torch.where(here, part, torch.zeros_like(part)))
    return {"drows": drows, "dw": torch.cat(dw, 1)}


def _plain(s):
    case = s["case"]
    op = case["op"]
    if op == "norm":
        return _plain_norm(s, case)
    if op == "norm_grad":
        return _plain_norm_grad(s, case)
    if op == "combine":
        return _plain_combine(s, case)
    if op == "route":
        offsets, place = _sort(s["ids"], case["groups"])
        rows, kept = _rows_of(place)
        x = s["x"]
        out = torch.empty((case["n"] * case["k"], case["f"]), dtype=x.dtype, device=DEVICE)
        for c in range(case["k"]):
            out[rows[:, c]] = torch.where(kept[:, c:c + 1], x, torch.zeros_like(x))
        return {"offsets": offsets, "place": place, "rows": out}
    q, scale = _quantize(s["x"].float())
    if op == "linear":
        y = (q @ s["wq"].float().t()) * s["ws"]
    else:
        # Each group's rows, padded to the largest group, in one batched product.
        offsets, at = s["offsets"].long(), torch.arange(case["n"], device=DEVICE)
        group = torch.searchsorted(offsets[1:], at, right=True)
        used = group < case["groups"]
        group = group.clamp(max=case["groups"] - 1)
        place = torch.where(used, at - offsets[group], torch.full_like(at, s["most"]))
        padded = torch.zeros((case["groups"], s["most"] + 1, case["fin"]), device=DEVICE)
        padded[group, place] = q
        y = torch.bmm(padded, s["wq"].float().transpose(1, 2).contiguous())[group, place]
        y = torch.where(used[:, None], y * s["ws"][group], torch.zeros_like(y))
    y = y * scale[:, None]
    if case["act"] == "relu":
        y = y.clamp(min=0)
    return {"y": y.to(TYPES[case["dtype"]])}


def run(s):
    if not own:
        return _plain(s)
    import paper_2308_11825_amd as agcn
    case = s["case"]
    op = case["op"]
    if op == "norm":
        if case["residual"]:
            y, h, stats = agcn.layer_norm(s["x"], s["g"], s["b"], residual=s["r"], eps=EPS,
                                          stats=True)
            return {"y": y, "stats": stats, "h": h}
        y, stats = agcn.layer_norm(s["x"], s["g"], s["b"], eps=EPS, stats=True)
        return {"y": y, "stats": stats}
    if op == "norm_grad":
        dx, dg, db = agcn.layer_norm_backward(s["dy"], s["x"], s["stats"], s["g"],
                                              bias=case["bias"], grad_hidden=s.get("dh"))
        return {"dg": dg, "db": db, "dx": dx} if case["bias"] else {"dg": dg, "dx": dx}
    if op == "route":
        offsets, place = agcn.sort_groups(s["ids"], case["groups"])
        return {"offsets": offsets, "place": place, "rows": agcn.dispatch(s["x"], place)}
    if op == "combine":
        if not case["grad"]:
            return {"out": agcn.combine(s["rows"], s["place"], s.get("w"))}
        drows, dw = agcn.combine_backward(s["dout"], s["rows"], s["place"], s["w"])
        return {"drows": drows, "dw": dw}
    q, scale = agcn.quantize_int(s["x"])
    dtype = TYPES[case["dtype"]]
    if op == "linear":
        return {"y": agcn.int_linear(q, scale, s["wq"], s["ws"], dtype=dtype, act=case["act"])}
    return {"y": agcn.grouped_int_linear(q, scale, s["wq"], s["ws"], s["offsets"], dtype=dtype,
                                         act=case["act"])}


# --- the work a pass cannot do without, and its results in 64 bits -----------------


def work(case):
    op, n = case["op"], case["n"]
    size = 4 if case["dtype"] == "float32" else 2
    if op in ("norm", "norm_grad"):
        f = case["f"]
        param = 4 if case["params"] == "float32" else 2
        if op == "norm":
            moved = 4 if case["residual"] else 2
            return {"bytes": n * f * size * moved + 8 * n + f * param * (2 if case["bias"] else 1),
                    "flops": 8 * n * f}
        moved = 4 if case["residual"] else 3
        return {"bytes": n * f * size * moved + 8 * n + f * param * (3 if case["bias"] else 2),
                "flops": 14 * n * f}
    if op in ("route", "combine"):
        f, slots = case["f"], n * case["k"]
        if op == "route":
            return {"bytes": (n + slots) * f * size + 8 * slots + 4 * case["groups"], "flops": 0}
        kept = int(slots * (1 - case["dropped"]))
        weights = 4 * slots if case["weights"] else 0
        if not case["grad"]:
            return {"bytes": (n + kept) * f * size + 4 * slots + weights, "flops": 2 * kept * f}
        return {"bytes": (n + kept + slots) * f * size + 4 * slots + 2 * weights,
                "flops": 3 * kept * f}
    fin, fout = case["fin"], case["fout"]
    groups, rows = case.get("groups", 1) - case.get("empty", 0), n - case.get("spare", 0)
    groups = min(groups, max(rows, 1))  # weights that no row takes are not read
    return {"bytes": n * fin * size + groups * fout * (fin + 4) + n * fout * size,
            "flops": 2 * rows * fin * fout}


def _exact_quantize(x):
    """The integers and scales of the rows of x, their two roundings to 32 bits (127 / top
    and its product with x) carried out on 64-bit values."""
    top = x.double().abs().amax(1, keepdim=True)
    factor = (127.0 / torch.where(top == 0, torch.ones_like(top), top)).float().double()
    return torch.round((x.double() * factor).float().double()), (top / 127.0)


def exact(case, seed):
    s = prepare(case, seed)
    op, n = case["op"], case["n"]
    if op == "norm":
        h = s["x"].double()
        if case["residual"]:
            h = h.add_(s["r"].double())
        mean = torch.sum(h, dim=1, keepdim=True) / case["f"]
        var = torch.sum((h - mean) ** 2, dim=1, keepdim=True) / case["f"]
        y = (h - mean) / torch.sqrt(var + EPS) * s["g"].double()
        if case["bias"]:
            y += s["b"].double()
        out = {"y": y, "stats": torch.cat([mean, 1 / torch.sqrt(var + EPS)], 1)}
        return {**out, "h": h} if case["residual"] else out
    if op == "norm_grad":
        h = s["x"].double()
        h -= torch.sum(h, dim=1, keepdim=True) / case["f"]
        scale = 1 / torch.sqrt(torch.sum(h ** 2, dim=1, keepdim=True) / case["f"] + EPS)
        h *= scale
        dy = s["dy"].double()
        out = {"dg": torch.sum(h * dy, dim=0)}
        if case["bias"]:
            out["db"] = torch.sum(dy, dim=0)
        dy *= s["g"].double()
        along = torch.sum(dy * h, dim=1, keepdim=True) / case["f"]
        dx = (dy - torch.sum(dy, dim=1, keepdim=True) / case["f"] - h * along) * scale
        out["dx"] = dx.add_(s["dh"].double()) if case["residual"] else dx
        return out
    if op == "route":
        # Slot by slot on the host: counts, their running sum, and each group's next place.
        ids, groups = s["ids"].reshape(-1).cpu(), case["groups"]
        if ids.numel() > 300000:
            return None
        x = s["x"].double()
        rows = torch.zeros((ids.numel(), case["f"]), dtype=torch.float64, device=DEVICE)
        kept = [e if 0 <= e < groups else groups for e in ids.tolist()]
        next_, total = [0] * (groups + 1), 0
        for e in kept:
            next_[e] += 1
        for e in range(groups + 1):
            next_[e], total = total, total + next_[e]
        offsets, place, at = torch.tensor(next_, dtype=torch.int32), [], []
        for e in kept:
            at.append(next_[e])
            place.append(next_[e] if e < groups else -1 - next_[e])
            next_[e] += 1
        used = torch.tensor([p >= 0 for p in place]).to(DEVICE)
        slots = torch.arange(len(place), device=DEVICE)[used]
        rows[torch.tensor(at).to(DEVICE)[used]] = x[slots // case["k"]]
        return {"offsets": offsets.to(DEVICE), "rows": rows,
                "place": torch.tensor(place, dtype=torch.int32).view(n, case["k"]).to(DEVICE)}
    if op == "combine":
        place, f = s["place"], case["f"]
        w = s["w"].double() if case["weights"] else torch.ones(place.shape, device=DEVICE).double()
        w = w * (place >= 0)
        at = torch.where(place >= 0, place, -1 - place).long()
        if not case["grad"]:
            out = torch.zeros((n, f), dtype=torch.float64, device=DEVICE)
            for c in range(case["k"]):
                out.addcmul_(w[:, c, None], s["rows"][at[:, c]].double())
            return {"out": out}
        drows = torch.zeros((n * case["k"], f), dtype=torch.float64, device=DEVICE)
        dw = torch.zeros(place.shape, dtype=torch.float64, device=DEVICE)
        for c in range(case["k"]):
            drows.index_copy_(0, at[:, c], w[:, c, None] * s["dout"].double())
            dw[:, c] = torch.sum(s["dout"].double() * s["rows"][at[:, c]].double(), dim=1)
        return {"drows": drows, "dw": dw * (place >= 0)}
    q, scale = _exact_quantize(s["x"])
    if op == "linear":
        y = q @ s["wq"].double().t() * s["ws"].double()
    else:
        y = torch.zeros((n, case["fout"]), dtype=torch.float64, device=DEVICE)
        at = 0
        for e, rows in enumerate(_sizes(case, seed)):
            if rows:
                y[at:at + rows] = (q[at:at + rows] @ s["wq"][e].double().t()) * s["ws"][e].double()
            at += rows
    y *= scale
    return {"y": y.clamp(min=0) if case["act"] == "relu" else y}
