"""The sequence operators' workloads: causal attention of grouped heads, the norms of queries and keys with the position
rotation, and the embedding of token ids, each forward and backward (per example where there are parameters), in a plain form
of elementary torch operations and as the calls that a user of the library makes.

Shapes: a small transformer of width 128 with contexts of 128 tokens and 64 workers, one of width 768 with contexts of 1024,
and generic sizes between and beside them.  An attention step is the forward call and the backward call behind it.
"""
import math

import torch

own = False

EPS = 1e-6
BASE = 10000.0
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    """`layout`: "dense" = examples of `tokens` rows each; "padded" = the same rows, of which an example has `count`;
    "packed" = rows of all examples one after the other."""
    return [
        # the small transformer's contexts of 64 workers, evaluation: latency
        {"name": "attention 64x128 4/4x32 f32", "op": "attention", "examples": 64, "tokens": 128, "q_heads": 4, "kv_heads": 4,
         "dim": 32, "type": "f32", "layout": "dense"},
        # long prompts with keys and values shared by four heads
        {"name": "attention 2x8192 32/8x128 bf16", "op": "attention", "examples": 2, "tokens": 8192, "q_heads": 32,
         "kv_heads": 8, "dim": 128, "type": "bf16", "layout": "dense"},
        # a training step's contexts of the wider transformer
        {"name": "attention step 64x1024 12/12x64 bf16", "op": "attention_step", "examples": 64, "tokens": 1024,
         "q_heads": 12, "kv_heads": 12, "dim": 64, "type": "bf16", "layout": "dense"},
        # documents of uneven length, one after the other, and heads of an unusual width
        {"name": "attention step 24x1500 8/2x80 f16", "op": "attention_step", "examples": 24, "tokens": 1500, "q_heads": 8,
         "kv_heads": 2, "dim": 80, "type": "f16", "layout": "packed"},
        # the small transformer's queries and keys, one worker's context
        {"name": "heads 1x128 4/4x32 f32", "op": "heads", "examples": 1, "tokens": 128, "q_heads": 4, "kv_heads": 4,
         "dim": 32, "type": "f32", "layout": "dense"},
        # a training step's queries and keys of the wider transformer
        {"name": "heads 64x1024 12/12x64 bf16", "op": "heads", "examples": 64, "tokens": 1024, "q_heads": 12, "kv_heads": 12,
         "dim": 64, "type": "bf16", "layout": "dense"},
        # and their backward pass
        {"name": "heads grad 64x1024 12/12x64 bf16", "op": "heads_grad", "examples": 64, "tokens": 1024, "q_heads": 12,
         "kv_heads": 12, "dim": 64, "type": "bf16", "layout": "dense"},
        # a padded batch of short texts, shared keys
        {"name": "heads grad 257x200 8/2x80 f16", "op": "heads_grad", "examples": 257, "tokens": 200, "q_heads": 8,
         "kv_heads": 2, "dim": 80, "type": "f16", "layout": "padded"},
        # one context of the small transformer: latency
        {"name": "embed 128 of 5000x128 f32", "op": "embed", "rows": 128, "vocab": 5000, "width": 128, "type": "f32"},
        # a step's contexts of the wider transformer
        {"name": "embed 65536 of 50000x768 bf16", "op": "embed", "rows": 65536, "vocab": 50000, "width": 768, "type": "bf16"},
        # the small transformer's table, a row of gradients for each of 64 workers
        {"name": "embed grad 64x128 5000x128 f32", "op": "embed_grad", "examples": 64, "tokens": 128, "vocab": 5000,
         "width": 128, "type": "f32", "layout": "dense"},
        # the wider transformer's table, a step's gradient of the whole batch
        {"name": "embed grad 1x65536 50000x768 bf16", "op": "embed_grad", "examples": 1, "tokens": 65536, "vocab": 50000,
         "width": 768, "type": "bf16", "layout": "dense"},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["attention", "attention_step", "heads", "heads_grad", "embed", "embed_grad"])
    case = {"op": op, "type": rng.choice(["f32", "bf16", "f16"])}
    if op in ("embed", "embed_grad"):
        width = _log(rng, 1, 2048)
        if op == "embed":
            vocab = _log(rng, 2, min(100000, (40 << 20) // width))
            case.update(rows=_log(rng, 1, min(65536, (48 << 20) // width)))
        else:
            examples = _log(rng, 1, 512)
            vocab = _log(rng, 2, max(2, min(100000, (36 << 20) // width // examples)))
            case.update(examples=examples, tokens=_log(rng, 1, max(1, min(65536, (36 << 20) // width) // examples)),
                        layout=rng.choice(["dense", "padded", "packed"]))
        case.update(vocab=vocab, width=width)
        return case
    kv = rng.choice([1, 2, 3, 4, 8])
    heads = kv * rng.choice([1, 1, 2, 3, 4])
    dim = rng.choice([32, 64, 128, 16, 48, 80, 96, 2 * rng.randint(4, 64)])
    examples = _log(rng, 1, 256)
    if op in ("heads", "heads_grad"):
        most = max(1, (48 << 20) // ((heads + kv) * dim) // examples)
    else:  # by the products, and by the plain form's matrices of scores
        most = int((((1 << 30) if op == "attention" else (1 << 28)) / (examples * heads)) ** 0.5)
    case.update(examples=examples, tokens=_log(rng, 1, max(1, min(8192, most))), q_heads=heads, kv_heads=kv, dim=dim,
                layout=rng.choice(["dense", "padded", "packed"]))
    return case


def _count(case):
    """Rows of each example: evenly from none to `tokens`."""
    n, t = case["examples"], case["tokens"]
    if case["layout"] == "dense" or n == 1:
        return [t] * n
    return [(n - i) * t // n for i in range(n - 1)] + [0]


def _spans(case, gen):
    """(leading shape of the rows, first row of each example, rows of each example); None where an example's place and
    length follow from the shape."""
    n, t = case["examples"], case["tokens"]
    if case["layout"] == "dense":
        return (n, t), None, None
    count = torch.tensor(_count(case), device="cuda")[torch.randperm(n, generator=gen, device="cuda")].to(torch.int32)
    if case["layout"] == "padded":
        return (n, t), None, count
    end = count.to(torch.int64).cumsum(0)
    return (int(end[-1]),), (end - count).contiguous(), count


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape, scale=1.0, offset=0.0):
        return torch.randn(*shape, generator=gen, device="cuda") * scale + offset

    def ids(*shape):  # ranks of words: the first ones often, most of them hardly ever
        u = torch.rand(*shape, generator=gen, device="cuda", dtype=torch.float64)
        return (torch.exp(u * math.log(case["vocab"] + 1.0)) - 1.0).clamp(0, case["vocab"] - 1).to(torch.int32)

    kind = TYPES[case["type"]]
    s = {"case": case}
    if case["op"] == "embed":
        s["ids"], s["table"] = ids(case["rows"]), normal(case["vocab"], case["width"], scale=0.02)
    else:
        lead, s["first"], s["count"] = _spans(case, gen)
        if case["op"] == "embed_grad":
            s["ids"], s["dy"] = ids(*lead), normal(*lead, case["width"], scale=0.01).to(kind)
        else:
            heads, kv, dim = case["q_heads"], case["kv_heads"], case["dim"]
            # the rows of a projection: queries, keys and values of a token side by side
            qkv = torch.cat([normal(*lead, heads * dim), normal(*lead, kv * dim), normal(*lead, kv * dim)], -1)
            if case["op"] in ("heads", "heads_grad"):
                qkv += normal(qkv.shape[-1], scale=0.5)  # features have means of their own
                s["gain_q"], s["gain_k"] = normal(dim, scale=0.1, offset=1.0), normal(dim, scale=0.1, offset=1.0)
                s["x"] = qkv.to(kind)[..., :(heads + kv) * dim]
                if case["op"] == "heads_grad":
                    s["dy"] = normal(*lead, (heads + kv) * dim, scale=0.01).to(kind)
                    s["dx"] = torch.zeros_like(s["dy"])  # rows of no example stay as they are
            else:
                qkv = qkv.to(kind)
                s["q"], s["k"], s["v"] = qkv.split([heads * dim, kv * dim, kv * dim], -1)
                if case["op"] == "attention_step":
                    s["do"] = normal(*lead, heads * dim, scale=0.01).to(kind)
    if own:
        import paper_2302_00845_amd as cdgrab

        s["handle"] = cdgrab.Handle()  # a program makes one for its life
    return s


def run(s):
    case = s["case"]
    if own:
        import paper_2302_00845_amd as cdgrab

        h = s["handle"]
        if case["op"] == "embed":
            return cdgrab.cdgrab_embed(h, s["ids"], s["table"], scale=_scale(case), dtype=TYPES[case["type"]])
        at = {"first": s["first"], "count": s["count"], "tokens": case["tokens"]}
        if case["op"] == "embed_grad":
            return cdgrab.cdgrab_pergrad_embed(h, s["ids"], s["dy"], case["vocab"], scale=_scale(case), **at)
        if case["op"] in ("heads", "heads_grad"):
            kw = dict(at, q_heads=case["q_heads"], k_heads=case["kv_heads"], eps=EPS, base=BASE)
            if case["op"] == "heads":
                return cdgrab.cdgrab_headnorm(h, s["x"], s["gain_q"], s["gain_k"], **kw)
            dx, g = cdgrab.cdgrab_pergrad_headnorm(h, s["x"], s["dy"], s["gain_q"], s["gain_k"], dX=s["dx"], **kw)
            return {"dx": dx, "g": g}
        kw = dict(at, q_heads=case["q_heads"], kv_heads=case["kv_heads"])
        if case["op"] == "attention":
            return cdgrab.cdgrab_attention(h, s["q"], s["k"], s["v"], want_lse=False, **kw)[0]
        o, lse = cdgrab.cdgrab_attention(h, s["q"], s["k"], s["v"], **kw)
        dq, dk, dv = cdgrab.cdgrab_attention_backward(h, s["q"], s["k"], s["v"], o, lse, s["do"], **kw)
        return {"o": o, "dq": dq, "dk": dk, "dv": dv}
    if case["op"] == "embed":
        return (s["table"][s["ids"].long()] * _scale(case)).to(TYPES[case["type"]])
    if case["op"] == "embed_grad":
        return _embed_grad(s)
    if case["op"] == "heads":
        return _heads(s)
    return _heads_grad(s) if case["op"] == "heads_grad" else _attention(s)


# ---- the plain forms ----------------------------------------------------------------------------

def _scale(case):
    return math.sqrt(case["width"])


def _places(s):
    """For rows that do not fill [examples][tokens]: (row of every place, whether the place has one)."""
    case = s["case"]
    at = torch.arange(case["tokens"], device="cuda")
    have = at < s["count"].unsqueeze(1)
    start = s["first"] if s["first"] is not None else torch.arange(case["examples"], device="cuda") * case["tokens"]
    return (start.unsqueeze(1) + at) * have, have


def _by_example(s, rows):
    """[examples][tokens][width] in 32 bits, zero where there is no row."""
    if s["count"] is None:
        return rows.float()
    place, have = _places(s)
    flat = rows.reshape(-1, rows.shape[-1])
    if not flat.shape[0]:
        return torch.zeros(*place.shape, rows.shape[-1], device="cuda")
    return flat[place].float() * have.unsqueeze(-1)


def _to_rows(s, out, like):
    """[examples][tokens][width] back to where the rows lie, zero elsewhere."""
    out = out.to(like.dtype)
    if s["count"] is None:
        return out
    place, have = _places(s)
    rows = torch.zeros(*like.shape[:-1], out.shape[-1], dtype=like.dtype, device="cuda")
    rows.view(-1, out.shape[-1])[place[have]] = out[have]
    return rows


def _embed_grad(s):
    case = s["case"]
    n, vocab, width = case["examples"], case["vocab"], case["width"]
    g = torch.zeros(n * vocab, width, device="cuda")
    which = torch.arange(n, device="cuda").unsqueeze(1) * vocab
    if s["count"] is None:
        g.index_add_(0, (which + s["ids"]).flatten(), s["dy"].float().flatten(0, 1))
    else:
        place, have = _places(s)
        place = place[have]
        at = which.expand(have.shape)[have] + s["ids"].flatten()[place]
        g.index_add_(0, at, s["dy"].reshape(-1, width)[place].float())
    return g.mul_(_scale(case)).view(n, vocab * width)


def _turns(case):
    """cos and sin [tokens][1][dim / 2] of position * base^(-2 i / dim), the angles in 64 bits."""
    half = case["dim"] // 2
    rate = BASE ** (torch.arange(half, device="cuda", dtype=torch.float64) * (-1.0 / half))
    angle = torch.arange(case["tokens"], device="cuda", dtype=torch.float64).view(-1, 1, 1) * rate
    return angle.cos().float(), angle.sin().float()


def _heads_parts(s):
    case = s["case"]
    x = _by_example(s, s["x"]).unflatten(-1, (-1, case["dim"]))
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    gain = torch.cat([s["gain_q"].expand(case["q_heads"], -1), s["gain_k"].expand(case["kv_heads"], -1)])
    return x, r, gain, *_turns(case)


def _heads(s):
    x, r, gain, cos, sin = _heads_parts(s)
    a, b = (x * r * gain).chunk(2, -1)
    return _to_rows(s, torch.cat([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), s["x"])


def _heads_grad(s):
    case = s["case"]
    x, r, gain, cos, sin = _heads_parts(s)
    a, b = _by_example(s, s["dy"]).unflatten(-1, (-1, case["dim"])).chunk(2, -1)
    u = torch.cat([a * cos + b * sin, b * cos - a * sin], -1)  # back by the angle
    hat = x * r
    per_head = (u * hat).sum(1)
    g = u * gain
    dx = r * (g - hat * (g * hat).mean(-1, keepdim=True))
    s["dx"].copy_(_to_rows(s, dx.flatten(-2), s["dx"]))
    heads = case["q_heads"]
    return {"dx": s["dx"], "g": torch.cat([per_head[:, :heads].sum(1), per_head[:, heads:].sum(1)], -1)}


def _split(x, heads, dim):
    """[examples][tokens][heads * dim] -> [examples * heads][tokens][dim]"""
    return x.unflatten(-1, (heads, dim)).transpose(1, 2).reshape(-1, x.shape[1], dim)


def _join(x, examples, tokens):
    return x.view(examples, -1, tokens, x.shape[-1]).transpose(1, 2).reshape(examples, tokens, -1)


def _attention(s):
    case = s["case"]
    n, t, heads, kv, dim = (case[k] for k in ("examples", "tokens", "q_heads", "kv_heads", "dim"))
    group, scale = heads // kv, 1.0 / math.sqrt(dim)
    q = _split(_by_example(s, s["q"]), heads, dim).view(n * kv, group * t, dim)  # the heads that share keys
    k, v = (_split(_by_example(s, s[x]), kv, dim) for x in "kv")
    step = case["op"] == "attention_step"
    do = _split(_by_example(s, s["do"]), heads, dim).view(n * kv, group * t, dim) if step else None
    later = torch.ones(t, t, dtype=torch.bool, device="cuda").triu(1).unsqueeze(0)
    parts = []
    at_once = max(1, (1 << 28) // (group * t * t))
    for i in range(0, n * kv, at_once):
        part = slice(i, i + at_once)
        w = torch.bmm(q[part], k[part].transpose(1, 2).contiguous()).mul_(scale)
        w.view(-1, t, t).masked_fill_(later, -math.inf)
        w = w.sub_(w.amax(-1, keepdim=True)).exp_()
        w = w.div_(w.sum(-1, keepdim=True))
        out = [torch.bmm(w, v[part])]
        if step:
            dw = torch.bmm(do[part], v[part].transpose(1, 2).contiguous())
            dw = dw.sub_((do[part] * out[0]).sum(-1, keepdim=True)).mul_(w).mul_(scale)
            out += [torch.bmm(dw, k[part]), torch.bmm(dw.transpose(1, 2).contiguous(), q[part]),
                    torch.bmm(w.transpose(1, 2).contiguous(), do[part])]
        parts.append(out)
    whole = [_join(torch.cat(p).view(-1, t, dim), n, t) for p in zip(*parts)]
    whole = [_to_rows(s, x, s["q"]) for x in whole]
    return dict(zip(("o", "dq", "dk", "dv"), whole)) if step else whole[0]


# ---- what the results are, in 64 bits -------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "embed":
        return torch.nn.functional.embedding(s["ids"].long(), s["table"].double()) * case["width"] ** 0.5
    n, t = case["examples"], case["tokens"]
    first = s["first"].tolist() if s["first"] is not None else [e * t for e in range(n)]
    spans = list(zip(first, s["count"].tolist() if s["count"] is not None else [t] * n))
    if case["op"] == "embed_grad":
        out = torch.zeros(n, case["vocab"], case["width"], dtype=torch.float64, device="cuda")
        ids, dy = s["ids"].flatten().long(), s["dy"].flatten(0, -2).double() * case["width"] ** 0.5
        for e, (at, count) in enumerate(spans):
            out[e].index_put_((ids[at:at + count],), dy[at:at + count], accumulate=True)
        return out.flatten(1)
    return _exact_heads(s, spans) if case["op"] in ("heads", "heads_grad") else _exact_attention(s, spans)


def _exact_heads(s, spans):
    """Pairs of features as complex numbers, turned by exp(i angle); gradients by autograd."""
    case = s["case"]
    dim, heads = case["dim"], case["q_heads"]
    half = dim // 2
    i = torch.arange(half, dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.ones(1, dtype=torch.float64, device="cuda"),
                       torch.outer(torch.arange(case["tokens"], dtype=torch.float64, device="cuda"), BASE ** (-2 * i / dim)))
    gains = [s["gain_q"].double().requires_grad_(), s["gain_k"].double().requires_grad_()]
    x = s["x"].flatten(0, -2).double()
    out, g = torch.zeros_like(x), []
    dy = s["dy"].flatten(0, -2).double() if case["op"] == "heads_grad" else None
    for at, count in spans:
        part = x[at:at + count].unflatten(-1, (-1, dim)).requires_grad_(dy is not None)
        hat = part / (part.square().sum(-1, keepdim=True) / dim + EPS).sqrt()
        hat = torch.cat([hat[:, :heads] * gains[0], hat[:, heads:] * gains[1]], 1)
        z = torch.complex(hat[..., :half], hat[..., half:]) * turn[:count].unsqueeze(1)
        y = torch.cat([z.real, z.imag], -1).flatten(1)
        if dy is None:
            out[at:at + count] = y.detach()
        else:
            dpart, *dgains = torch.autograd.grad(y, [part] + gains, dy[at:at + count])
            out[at:at + count] = dpart.flatten(1)
            g.append(torch.cat(dgains))
    out = out.view(s["x"].shape)
    return out if dy is None else {"dx": out, "g": torch.stack(g)}


def _exact_attention(s, spans):
    case = s["case"]
    heads, kv, dim = case["q_heads"], case["kv_heads"], case["dim"]
    step = case["op"] == "attention_step"
    q, k, v = (s[x].flatten(0, -2).unflatten(-1, (-1, dim)) for x in "qkv")
    do = s["do"].flatten(0, -2).unflatten(-1, (-1, dim)) if step else None
    o, dq, dk, dv = (torch.zeros(x.shape, dtype=torch.float64, device="cuda") for x in (q, q, k, v))
    for at, count in spans:
        rows = slice(at, at + count)
        seen = torch.ones(count, count, dtype=torch.bool, device="cuda").tril()
        for g in range(kv):
            kk, vv = k[rows, g].double().requires_grad_(step), v[rows, g].double().requires_grad_(step)
            for j in range(g * heads // kv, (g + 1) * heads // kv):
                qq = q[rows, j].double().requires_grad_(step)
                score = (qq @ kk.t() / dim ** 0.5).where(seen, -torch.inf)
                out = torch.softmax(score, 1) @ vv
                o[rows, j] = out.detach()
                if step:
                    grads = torch.autograd.grad(out, [qq, kk, vv], do[rows, j].double())
                    dq[rows, j] = grads[0]
                    dk[rows, g] += grads[1]
                    dv[rows, g] += grads[2]
    o, dq, dk, dv = (x.flatten(1).view(*like.shape) for x, like in zip((o, dq, dk, dv), (s["q"], s["q"], s["k"], s["v"])))
    return {"o": o, "dq": dq, "dk": dk, "dv": dv} if step else o


# ---- what a pass cannot do without ------------------------------------------------------------------

def work(case):
    size = torch.empty((), dtype=TYPES[case["type"]]).element_size()
    if case["op"] == "embed":
        cells = case["rows"] * case["width"]
        # (ids by rank: about as many rows of the table are read as are drawn, or there are)
        return {"bytes": cells * size + 4 * min(case["rows"], case["vocab"]) * case["width"] + 4 * case["rows"], "flops": cells}
    rows = sum(_count(case))
    if case["op"] == "embed_grad":
        cells = rows * case["width"]
        return {"bytes": cells * size + 4 * rows + 4 * case["examples"] * case["vocab"] * case["width"], "flops": cells}
    heads, kv, dim = case["q_heads"], case["kv_heads"], case["dim"]
    if case["op"] == "heads":
        cells = rows * (heads + kv) * dim
        return {"bytes": 2 * cells * size, "flops": 8 * cells}
    if case["op"] == "heads_grad":
        cells = rows * (heads + kv) * dim
        return {"bytes": 3 * cells * size + 8 * case["examples"] * dim, "flops": 16 * cells}
    pairs = heads * sum(c * (c + 1) // 2 for c in _count(case))
    cells = rows * dim * 2 * (heads + kv)  # queries, keys, values, outputs
    if case["op"] == "attention":
        return {"bytes": cells * size, "flops": 4 * dim * pairs}
    # the forward pass's two products and the backward pass's five; dO is read, and dQ, dK, dV are written, besides
    return {"bytes": (2 * cells + rows * dim * heads) * size, "flops": 14 * dim * pairs}
