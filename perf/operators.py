"""The layer operators' workloads: layer norm (forward; backward with per-example gain and bias gradients), per-example
gradients of linear layers, and the orthogonalised update, each in a plain form of elementary torch operations and as the
calls that a user of the library makes.

Shapes: the 785 x 10 softmax regression on 60 000 examples, a small transformer of width 128 with contexts of 128 tokens
and 64 workers, one of width 768 with contexts of 1024, and generic sizes between and beside them.
"""
import math

import torch

own = False

EPS = 1e-5
STEPS = 5
COEFFS = (3.4445, -4.775, 2.0315)
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    """`layout`: "dense" = examples of `tokens` rows each; "padded" = the same rows, of which an example has `count`;
    "packed" = rows of all examples one after the other."""
    return [
        # one context of the small transformer: latency
        {"name": "norm 128x128 f32", "op": "norm", "rows": 128, "width": 128, "type": "f32"},
        # a step's contexts of the wider transformer
        {"name": "norm 65536x768 bf16", "op": "norm", "rows": 65536, "width": 768, "type": "bf16"},
        # 64 workers' examples of the small transformer
        {"name": "norm grad 64x128x128 f32", "op": "norm_grad", "examples": 64, "tokens": 128, "width": 128, "type": "f32",
         "layout": "dense"},
        # a step's contexts of the wider transformer
        {"name": "norm grad 64x1024x768 bf16", "op": "norm_grad", "examples": 64, "tokens": 1024, "width": 768,
         "type": "bf16", "layout": "dense"},
        # documents of uneven length, one after the other, and an odd width
        {"name": "norm grad 257x200x515 f16", "op": "norm_grad", "examples": 257, "tokens": 200, "width": 515,
         "type": "f16", "layout": "packed"},
        # the small transformer's query/key/value layer, 64 workers
        {"name": "linear 64x128 128-384 f32", "op": "linear", "examples": 64, "tokens": 128, "in": 128, "out": 384,
         "type": "f32", "layout": "dense"},
        # the wider transformer's, 32 workers
        {"name": "linear 32x1024 768-2304 bf16", "op": "linear", "examples": 32, "tokens": 1024, "in": 768, "out": 2304,
         "type": "bf16", "layout": "dense"},
        # the softmax regression's examples: one row each
        {"name": "linear 60000x1 784-10 f32", "op": "linear", "examples": 60000, "tokens": 1, "in": 784, "out": 10,
         "type": "f32", "layout": "dense"},
        # a padded batch of short texts, odd sizes
        {"name": "linear 100x63 301-1001 f16", "op": "linear", "examples": 100, "tokens": 63, "in": 301, "out": 1001,
         "type": "f16", "layout": "padded"},
        # the softmax regression's velocity: latency
        {"name": "orth 785x10 f32", "op": "orth", "batch": 1, "rows": 785, "cols": 10, "type": "f32"},
        # the small transformer's square layers
        {"name": "orth 8x128x128 bf16", "op": "orth", "batch": 8, "rows": 128, "cols": 128, "type": "bf16"},
        # the wider transformer's query/key/value layers
        {"name": "orth 12x768x2304 f32", "op": "orth", "batch": 12, "rows": 768, "cols": 2304, "type": "f32"},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "linear", "orth"])
    kind = rng.choice(["f32", "bf16", "f16"])
    if op == "norm":
        width = _log(rng, 1, 8192)
        return {"op": op, "rows": _log(rng, 1, min(65536, (50 << 20) // width)), "width": width, "type": kind}
    if op == "norm_grad":
        width = _log(rng, 8, 8192)  # (of two features the gradient is rounding: x-hat is +1 and -1)
        examples = _log(rng, 1, min(1024, (50 << 20) // width))
        return {"op": op, "examples": examples, "tokens": _log(rng, 1, min(4096, (50 << 20) // width // examples)),
                "width": width, "type": kind, "layout": rng.choice(["dense", "padded", "packed"])}
    if op == "linear":
        n_in, n_out = _log(rng, 1, 2500), _log(rng, 1, 2500)
        examples = _log(rng, 1, max(1, min(4096, (50 << 20) // ((n_in + 1) * n_out))))
        most = min(2048, max(1, (25 << 20) // (examples * (n_in + n_out))), max(1, 50_000_000_000 // (examples * n_in * n_out)))
        return {"op": op, "examples": examples, "tokens": _log(rng, 1, most), "in": n_in, "out": n_out, "type": kind,
                "layout": rng.choice(["dense", "padded", "packed"])}
    rows, cols = _log(rng, 1, 2500), _log(rng, 1, 2500)
    short, long = min(rows, cols), max(rows, cols)
    most = max(1, min(64, 12 * 768 * 768 * 2304 // (short * short * long), (20 << 20) // (rows * cols)))
    return {"op": op, "batch": _log(rng, 1, most), "rows": rows, "cols": cols, "type": kind}


def _counts(case, gen):
    """Rows of each example: evenly from none to `tokens`, in any order (so that their sum goes by the case alone)."""
    n = case["examples"]
    even = torch.arange(n, 0, -1, device="cuda") * case["tokens"] // n if n > 1 else torch.tensor([case["tokens"]], device="cuda")
    even[-1] = 0 if n > 1 else case["tokens"]
    return even[torch.randperm(n, generator=gen, device="cuda")].to(torch.int32)


def _spans(case, gen):
    """(leading shape of the rows, first row of each example, rows of each example); None where an example's place and
    length follow from the shape."""
    n, t = case["examples"], case["tokens"]
    if case["layout"] == "dense":
        return (n, t), None, None
    count = _counts(case, gen)
    if case["layout"] == "padded":
        return (n, t), None, count
    end = count.to(torch.int64).cumsum(0)
    return (int(end[-1]),), (end - count).contiguous(), count


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape, scale=1.0, offset=0.0):
        return torch.randn(*shape, generator=gen, device="cuda") * scale + offset

    kind = TYPES[case["type"]]
    s = {"case": case}
    if case["op"] in ("norm", "norm_grad"):
        width = case["width"]
        s["gain"], s["bias"] = normal(width, scale=0.1, offset=1.0), normal(width, scale=0.1)
        column = normal(width, scale=0.5)  # features have means and scales of their own
        spread = torch.exp(normal(width, scale=0.3))
        if case["op"] == "norm":
            s["x"] = (normal(case["rows"], width) * spread + column).to(kind)
        else:
            lead, s["first"], s["count"] = _spans(case, gen)
            s["x"] = (normal(*lead, width) * spread + column).to(kind)
            s["dy"] = normal(*lead, width, scale=0.01).to(kind)
            s["dx"] = torch.zeros_like(s["x"])  # rows of no example stay as they are
    elif case["op"] == "linear":
        lead, s["first"], s["count"] = _spans(case, gen)
        s["x"] = normal(*lead, case["in"], offset=0.2).to(kind)
        s["dy"] = normal(*lead, case["out"], scale=0.01).to(kind)
    else:
        b, rows, cols = case["batch"], case["rows"], case["cols"]
        # a momentum: noise and a few directions that the batches agree on
        few = max(1, min(rows, cols) // 32)
        s["m"] = (0.01 * (normal(b, rows, cols) + 0.3 * torch.bmm(normal(b, rows, few), normal(b, few, cols)))).to(kind)
    if own:
        import paper_2302_00845_amd as cdgrab

        s["handle"] = cdgrab.Handle()  # a program makes one for its life
    return s


def run(s):
    case = s["case"]
    if own:
        import paper_2302_00845_amd as cdgrab

        h = s["handle"]
        if case["op"] == "norm":
            return cdgrab.cdgrab_layernorm(h, s["x"], s["gain"], s["bias"], eps=EPS)
        if case["op"] == "norm_grad":
            dx, g = cdgrab.cdgrab_pergrad_layernorm(h, s["x"], s["dy"], s["gain"], eps=EPS, first=s["first"],
                                                    count=s["count"], tokens=case["tokens"], dX=s["dx"])
            return {"dx": dx, "g": g}
        if case["op"] == "linear":
            return cdgrab.cdgrab_pergrad_linear(h, s["x"], s["dy"], first=s["first"], count=s["count"],
                                                tokens=case["tokens"])
        return cdgrab.cdgrab_orthogonalize(h, s["m"], steps=STEPS, coeffs=COEFFS)
    if case["op"] == "norm":
        return _norm(s)
    if case["op"] == "norm_grad":
        return _norm_grad(s)
    return _linear(s) if case["op"] == "linear" else _orth(s)


# ---- the plain forms ----------------------------------------------------------------------------

def _norm(s):
    x = s["x"].float()
    x = x - x.mean(-1, keepdim=True)
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * s["gain"] + s["bias"]
    return y.to(s["x"].dtype)


def _places(s):
    """For rows that do not fill [examples][tokens]: (row of every place, whether the place has one)."""
    case = s["case"]
    at = torch.arange(case["tokens"], device="cuda")
    have = at < s["count"].unsqueeze(1)
    start = s["first"] if s["first"] is not None else torch.arange(case["examples"], device="cuda") * case["tokens"]
    return (start.unsqueeze(1) + at) * have, have


def _by_example(s, rows):
    """[examples][tokens][width] in 32 bits, zero where there is no row."""
    rows = rows.float()
    if s["count"] is None:
        return rows
    place, have = _places(s)
    flat = rows.reshape(-1, rows.shape[-1])
    if not flat.shape[0]:
        return rows.new_zeros(*place.shape, rows.shape[-1])
    return torch.where(have.unsqueeze(-1), flat[place], rows.new_zeros(()))


def _norm_grad(s):
    x, dy = _by_example(s, s["x"]), _by_example(s, s["dy"])
    x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    xh, g = x * r, dy * s["gain"]
    dx = (r * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))).to(s["x"].dtype)
    grads = torch.cat([(dy * xh).sum(1), dy.sum(1)], 1)
    if s["count"] is None:
        s["dx"].copy_(dx)
    else:
        place, have = _places(s)
        s["dx"].view(-1, dx.shape[-1])[place[have]] = dx[have]
    return {"dx": s["dx"], "g": grads}


def _linear(s):
    x, dy = _by_example(s, s["x"]), _by_example(s, s["dy"])
    x = torch.cat([x, x.new_ones(*x.shape[:2], 1)], 2)  # the bias's input
    return torch.bmm(x.transpose(1, 2), dy).flatten(1)


def _orth(s):
    m = s["m"].float()
    wide = m.shape[1] <= m.shape[2]
    x = m if wide else m.transpose(1, 2).contiguous()
    x = x / (x * x).sum((1, 2), keepdim=True).sqrt()
    a, b, c = COEFFS
    for _ in range(STEPS):
        p = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.bmm(b * p + c * torch.bmm(p, p), x)
    return (x if wide else x.transpose(1, 2)).contiguous().to(s["m"].dtype)


# ---- what the results are, in 64 bits -------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        var, mean = torch.var_mean(s["x"].double(), -1, correction=0, keepdim=True)
        return (s["x"].double() - mean) / (var + EPS).sqrt() * s["gain"].double() + s["bias"].double()
    if case["op"] == "orth":
        # through the singular values: X0 = U S V^T gives U f(f(..f(S))) V^T; by products in 64 bits, whose
        # rounding is far below, since a decomposition of large matrices takes minutes
        if case["batch"] * case["rows"] * case["cols"] * min(case["rows"], case["cols"]) > 2 ** 24:
            return torch.stack([_exact_products(m) for m in s["m"].double()])
        u, v, w = torch.linalg.svd(s["m"].double().cpu(), full_matrices=False)
        v = v / v.square().sum(-1, keepdim=True).sqrt()
        for _ in range(STEPS):
            v = COEFFS[0] * v + COEFFS[1] * v ** 3 + COEFFS[2] * v ** 5
        return (u * v.unsqueeze(-2) @ w).cuda()
    n, t = case["examples"], case["tokens"]
    first = s["first"].tolist() if s["first"] is not None else [e * t for e in range(n)]
    count = s["count"].tolist() if s["count"] is not None else [t] * n
    x, dy = s["x"].flatten(0, -2).double(), s["dy"].flatten(0, -2).double()
    if case["op"] == "linear":
        if t == 1 and s["count"] is None:
            return torch.cat([x.unsqueeze(2) * dy.unsqueeze(1), dy.unsqueeze(1)], 1).flatten(1)
        out = x.new_zeros(n, case["in"] + 1, case["out"])
        for e in range(n):
            rows = slice(first[e], first[e] + count[e])
            out[e, :-1] = x[rows].t() @ dy[rows]
            out[e, -1] = dy[rows].sum(0)
        return out.flatten(1)
    width = case["width"]
    dx, g = torch.zeros_like(x), x.new_zeros(n, 2, width)
    for e in range(n):
        rows = slice(first[e], first[e] + count[e])
        var, mean = torch.var_mean(x[rows], -1, correction=0, keepdim=True)
        sd = (var + EPS).sqrt()
        hat, up = (x[rows] - mean) / sd, dy[rows] * s["gain"].double()
        dx[rows] = (up - (up.sum(-1, keepdim=True) + hat * (up * hat).sum(-1, keepdim=True)) / width) / sd
        g[e, 0], g[e, 1] = (dy[rows] * hat).sum(0), dy[rows].sum(0)
    return {"dx": dx.view(s["x"].shape), "g": g.flatten(1)}


def _exact_products(m):
    flip = m.shape[0] > m.shape[1]
    x = (m.t() if flip else m) / torch.linalg.matrix_norm(m)
    eye = torch.eye(x.shape[0], dtype=x.dtype, device=x.device)
    for _ in range(STEPS):
        p = x @ x.t()
        x = (COEFFS[0] * eye + p @ (COEFFS[1] * eye + COEFFS[2] * p)) @ x
    return x.t().contiguous() if flip else x


# ---- what a pass cannot do without ------------------------------------------------------------------

def work(case):
    size = torch.empty((), dtype=TYPES[case["type"]]).element_size()
    if case["op"] == "norm":
        cells = case["rows"] * case["width"]
        return {"bytes": 2 * cells * size + 8 * case["width"], "flops": 8 * cells}
    if case["op"] == "orth":
        cells = case["rows"] * case["cols"]
        short, long = min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
        # X X^T and A^2 are symmetric: half of their entries
        return {"bytes": 2 * case["batch"] * cells * size,
                "flops": case["batch"] * STEPS * (3 * short * short * long + short ** 3)}
    n = case["examples"]
    # (padded and packed examples have half of `tokens` on average)
    rows = n * case["tokens"] if case["layout"] == "dense" else (n * case["tokens"] + case["tokens"]) / 2
    if case["op"] == "linear":
        return {"bytes": rows * (case["in"] + case["out"]) * size + 4 * n * (case["in"] + 1) * case["out"],
                "flops": 2 * rows * case["in"] * case["out"]}
    cells = rows * case["width"]
    return {"bytes": 3 * cells * size + 8 * n * case["width"] + 4 * case["width"], "flops": 14 * cells}
