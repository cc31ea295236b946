"""What the speed of the operators before and after the stack of blocks is measured on: the orthogonalised update of the weights from
the gradients that the compressor hands back, the embedding of the tokens with its gradient, and the norms of queries and keys with the
rotation by position.

``run`` computes an operator in its plain form (32 bits, angles in 64, elementary torch operations, one rounding at the end), or, where
``own`` is set, through the public entry points of ``paper_2511_10333_amd``.

Fields of a case: ``op`` ("ortho", "embed", "qk"), ``dtype`` ("f32", "bf16") and
  ortho: ``shapes`` ("MxN" a matrix, ",": the next one), ``steps``
  embed: ``dir`` ("fwd", "bwd"), ``tokens``, ``vocab``, ``hidden``, ``ids`` (32 or 64 bits each), ``outside`` (the share of the tokens whose
         row is not in this part of the table, padding among them), ``first`` (id of the table's first row), ``scale``
  qk:    ``dir``, ``tokens``, ``heads_q``, ``heads_k``, ``dim``, ``rot`` (dimensions that are rotated), ``interleaved`` (neighbours are a
         pair, instead of the two halves), ``packed`` (queries, keys and values of a token in one row, as one product gives them), ``far``
         (positions begin up to there)
"""
import math

import torch

own = False

EPS = 1e-6                                  # of the norms, beside the mean square
NS_EPS = 1e-7                               # of the orthogonalised update, beside the gradient's norm
NS_COEFS = (3.4445, -4.7750, 2.0315)        # x <- a x + (b A + c A^2) x, A = x x^T
BASE = 10000.0


# ---------------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------------
def _block(hidden):
    """The four 2-D gradients of a block."""
    h = hidden
    return [(h, 3 * h), (h, h), (h, 4 * h), (4 * h, h)]


def _ortho(name, shapes, dtype, steps=5):
    c = {"op": "ortho", "shapes": ",".join("%dx%d" % s for s in shapes), "dtype": dtype, "steps": steps}
    return dict(c, name=name) if name else c


def _embed(name, direction, tokens, vocab, hidden, dtype, ids=64, outside=0.0, first=0, scale=1.0):
    c = {"op": "embed", "dir": direction, "tokens": tokens, "vocab": vocab, "hidden": hidden, "dtype": dtype, "ids": ids,
         "outside": outside, "first": first, "scale": scale}
    return dict(c, name=name) if name else c


def _qk(name, direction, tokens, heads_q, heads_k, dim, dtype, rot=None, interleaved=False, packed=True, far=0):
    c = {"op": "qk", "dir": direction, "tokens": tokens, "heads_q": heads_q, "heads_k": heads_k, "dim": dim, "dtype": dtype,
         "rot": dim if rot is None else rot, "interleaved": interleaved, "packed": packed, "far": far}
    return dict(c, name=name) if name else c


def listed():
    return [
        # a small block's four matrices: launches and latency
        _ortho("ortho_block_h512_f32", _block(512), "f32"),
        # a block of a middling model, fp32 gradients
        _ortho("ortho_block_h2048_f32", _block(2048), "f32"),
        # a block of a large model, bf16 gradients
        _ortho("ortho_block_h4096_bf16", _block(4096), "bf16"),
        # matrices of unlike and odd shapes in one list: wide, tall, a single row, nothing that ends with a tile
        _ortho("ortho_odd_f32", [(1001, 997), (130, 2731), (2500, 333), (1, 77), (65, 64)], "f32"),
        # one token of a request being answered
        _embed("embed_fwd_token_h4096_bf16", "fwd", 1, 50000, 4096, "bf16"),
        # a large micro-batch's rows
        _embed("embed_fwd_16384_h5120_bf16", "fwd", 16384, 65536, 5120, "bf16", scale=8.0),
        # the gradient of a large table: most tokens are few words, and most words have no token
        _embed("embed_bwd_16384_h4096_bf16", "bwd", 16384, 50000, 4096, "bf16"),
        # one rank's part of a table, odd everywhere, a third of the tokens elsewhere or padding
        _embed("embed_bwd_odd_f32", "bwd", 2999, 5003, 1001, "f32", ids=32, outside=0.35, first=5003, scale=0.5),
        # eight requests being answered, one token each, far into their texts
        _qk("qk_fwd_tokens8_d128_bf16", "fwd", 8, 32, 8, 128, "bf16", far=1 << 20),
        # a large micro-batch, eight queries' heads to a key's
        _qk("qk_fwd_16384_d128_bf16", "fwd", 16384, 40, 8, 128, "bf16", far=4096),
        # its backward, gradients of the shared weights among the outputs
        _qk("qk_bwd_8192_d128_bf16", "bwd", 8192, 32, 8, 128, "bf16"),
        # heads of odd number and size, part of a head rotated, neighbours as pairs
        _qk("qk_bwd_odd_f32", "bwd", 1001, 7, 3, 72, "f32", rot=40, interleaved=True, far=100000),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size in [lo, hi]: as it comes, or a multiple of 64."""
    d = _log_int(rng, lo, hi)
    return max(64, d // 64 * 64) if rng.random() < 0.5 else d


def draw(rng):
    op = rng.choice(["ortho", "embed", "qk"])
    dtype = rng.choice(["f32", "bf16"])
    if op == "ortho":
        steps = rng.choice([3, 5, 5, 5, 6])
        if rng.random() < 0.5:
            return _ortho(None, _block(_size(rng, 128, 2048)), dtype, steps)
        while True:
            shapes = [(_size(rng, 1, 6000), _size(rng, 1, 6000)) for _ in range(rng.randint(1, 8))]
            if 6 * sum(min(s) ** 2 * max(s) for s in shapes) <= 1.5e11:
                return _ortho(None, shapes, dtype, steps)
    direction = rng.choice(["fwd", "bwd"])
    tokens = _log_int(rng, 1, 16384)
    if op == "embed":
        vocab, hidden = _log_int(rng, 100, 65536), _size(rng, 64, 5120)
        first = rng.choice([0, 0, vocab])
        return _embed(None, direction, tokens, vocab, hidden, dtype, rng.choice([32, 64, 64]), rng.choice([0.0, 0.0, 0.1, 0.6]), first,
                      rng.choice([1.0, 1.0, 0.25, 45.25]))
    heads_k = rng.choice([1, 2, 3, 4, 8, 16])
    heads_q = heads_k * rng.choice([1, 2, 4, 5, 7])
    dim = rng.choice([32, 64, 64, 72, 80, 96, 128, 128, 192, 256])
    tokens = min(tokens, 16384 * 48 * 128 // ((heads_q + 2 * heads_k) * dim))
    rot = rng.choice([dim, dim, dim // 2, dim // 4 // 2 * 2])
    return _qk(None, direction, tokens, heads_q, heads_k, dim, dtype, rot, rng.random() < 0.4, rng.random() < 0.7,
               rng.choice([0, 4096, 1 << 20]))


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def _shapes(case):
    return [tuple(int(d) for d in s.split("x")) for s in case["shapes"].split(",")]


def _tdtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _parts(flat, shapes):
    """Views of a slab of gradients, one behind the other."""
    return [p.view(s) for p, s in zip(torch.split(flat, [math.prod(s) for s in shapes]), shapes)]


def _scales(case):
    """What the update of a matrix is multiplied by, so that tall matrices' rows move as far as wide ones'."""
    return [math.sqrt(max(1.0, m / n)) for m, n in _shapes(case)]


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed * 1000003 + 31)
    dt = _tdtype(case)

    def randn(*s, std=1.0):
        return torch.randn(*s, generator=g, device="cuda").mul_(std).to(dt)

    if case["op"] == "ortho":
        shapes = _shapes(case)
        flat = torch.empty(sum(math.prod(s) for s in shapes), device="cuda", dtype=dt)
        for p in _parts(flat, shapes):      # a gradient: a few strong directions, each weaker than the one before, above noise
            m, n = p.shape
            k = min(32, m, n)
            u, v = (torch.randn(d, k, generator=g, device="cuda") for d in (m, n))
            w = torch.randn(m, n, generator=g, device="cuda")
            p.copy_(((u * 0.8 ** torch.arange(k, device="cuda")) @ v.t()).add_(w).mul_(1e-4))
        return {"grads": flat}
    t = case["tokens"]
    if case["op"] == "embed":
        v, h, first = case["vocab"], case["hidden"], case["first"]
        # words by their rank: the i-th has 1 / i of the first one's tokens
        u = torch.rand(t, generator=g, device="cuda", dtype=torch.float64)
        ids = first + torch.clamp(torch.exp(u * math.log(v + 1)).long() - 1, 0, v - 1)
        if case["outside"]:
            away = torch.rand(t, generator=g, device="cuda") < case["outside"]
            pad = torch.rand(t, generator=g, device="cuda") < 0.5
            ids = torch.where(away, torch.where(pad, -1, first + v + ids % 7), ids)
        ids = ids.to(torch.int32 if case["ids"] == 32 else torch.int64)
        return {"ids": ids, "dy": randn(t, h, std=1e-3)} if case["dir"] == "bwd" else {"ids": ids, "table": randn(v, h, std=0.02)}
    hq, hk, dim = case["heads_q"], case["heads_k"], case["dim"]
    if case["packed"]:
        row = randn(t, (hq + 2 * hk) * dim, std=2.0)
        q, k = row[:, :hq * dim].view(t, hq, dim), row[:, hq * dim:(hq + hk) * dim].view(t, hk, dim)
    else:
        q, k = randn(t, hq, dim, std=2.0), randn(t, hk, dim, std=2.0)
    d = {"q": q, "k": k, "w_q": 1 + randn(dim, std=0.1), "w_k": 1 + randn(dim, std=0.1)}
    begin = torch.randint(0, case["far"] + 1, (), generator=g, device="cuda")
    d["positions"] = begin + torch.arange(t, device="cuda")
    if t <= 64:                             # tokens of different texts
        d["positions"] = torch.randint(0, case["far"] + 4096, (t,), generator=g, device="cuda")
    r = case["rot"]
    d["inv_freq"] = BASE ** (-torch.arange(0, r, 2, device="cuda", dtype=torch.float64) / max(r, 1))
    if case["dir"] == "bwd":
        d |= {"dq_out": randn(t, hq, dim, std=1e-3), "dk_out": randn(t, hk, dim, std=1e-3)}
    return d


def prepare(case, seed):
    state = {"case": case, "in": _inputs(case, seed)}
    if not own:
        return state
    import paper_2511_10333_amd as edgc
    d, dt = state["in"], _tdtype(case)
    ctx = state["ctx"] = edgc.Context(0, max_bins=256, max_rank=16, max_rows=64, max_cols=64)
    if case["op"] == "ortho":
        shapes = _shapes(case)
        state["out"] = {"updates": torch.empty_like(d["grads"])}
        ctx.reserve_orthogonalize(dt, shapes, steps=case["steps"])
        state["batch"] = edgc.PreparedBatch([edgc.Tensor(a, b) for a, b in zip(_parts(d["grads"], shapes),
                                                                             _parts(state["out"]["updates"], shapes))])
        state["scales"] = _scales(case)
        return state
    t = case["tokens"]
    if case["op"] == "embed":
        if case["dir"] == "fwd":
            state["out"] = {"x": torch.empty((t, case["hidden"]), device="cuda", dtype=dt)}
        else:
            ctx.reserve_embed(t, case["vocab"], case["hidden"])
            state["out"] = {"dtable": torch.empty((case["vocab"], case["hidden"]), device="cuda", dtype=dt)}
        return state
    state["out"] = {n: torch.empty(d[n[-1]].shape, device="cuda", dtype=dt) for n in (("q", "k") if case["dir"] == "fwd" else ("dq", "dk"))}
    if case["dir"] == "bwd":
        ctx.reserve_qk_norm(t, case["heads_q"], case["heads_k"], case["dim"])
        state["out"] |= {n: torch.empty(case["dim"], device="cuda", dtype=dt) for n in ("dw_q", "dw_k")}
    return state


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------
def run(state):
    case, d = state["case"], state["in"]
    if not own:
        return {"ortho": _plain_ortho, "embed": _plain_embed, "qk": _plain_qk}[case["op"]](case, d)
    ctx, out = state["ctx"], state["out"]
    if case["op"] == "ortho":
        ctx.orthogonalize_batch(state["batch"], steps=case["steps"], coefficients=NS_COEFS, eps=NS_EPS, scales=state["scales"])
    elif case["op"] == "embed" and case["dir"] == "fwd":
        ctx.embed_forward(d["table"], d["ids"], out["x"], scale=case["scale"], first_id=case["first"])
    elif case["op"] == "embed":
        ctx.embed_backward(d["ids"], d["dy"], out["dtable"], scale=case["scale"], first_id=case["first"])
    elif case["dir"] == "fwd":
        ctx.qk_norm_forward(d["q"], d["k"], d["w_q"], d["w_k"], d["positions"], d["inv_freq"], out["q"], out["k"], eps=EPS,
                            interleaved=case["interleaved"])
    else:
        ctx.qk_norm_backward(d["dq_out"], d["dk_out"], d["q"], d["k"], d["w_q"], d["w_k"], d["positions"], d["inv_freq"], out["dq"],
                             out["dk"], out["dw_q"], out["dw_k"], eps=EPS, interleaved=case["interleaved"])
    return out


def _plain_ortho(case, d):
    shapes = _shapes(case)
    a, b, c = NS_COEFS
    out = torch.empty_like(d["grads"])
    for g, o, scale in zip(_parts(d["grads"], shapes), _parts(out, shapes), _scales(case)):
        x = g.float()
        x = x / (x.square().sum().sqrt() + NS_EPS)
        x = x.t() if x.shape[0] > x.shape[1] else x
        for _ in range(case["steps"]):
            gram = x @ x.t()
            x = a * x + (b * gram + c * (gram @ gram)) @ x
        x = x.t() if g.shape[0] > g.shape[1] else x
        o.copy_(x * scale)
    return {"updates": out}


def _plain_embed(case, d):
    dt, v = _tdtype(case), case["vocab"]
    row = d["ids"].long() - case["first"]
    inside = (row >= 0) & (row < v)
    row = torch.where(inside, row, 0)
    if case["dir"] == "fwd":
        return {"x": (d["table"][row].float() * (inside[:, None] * case["scale"])).to(dt)}
    dtable = torch.zeros((v, case["hidden"]), device="cuda")
    dtable.index_add_(0, row, d["dy"].float() * inside[:, None])
    return {"dtable": (dtable * case["scale"]).to(dt)}


def _rotate(x, cos, sin, interleaved):
    """The first 2 n dimensions of a head by n angles, the others as they are."""
    n = cos.shape[-1]
    turned, rest = x[..., :2 * n], x[..., 2 * n:]
    a, b = (turned[..., 0::2], turned[..., 1::2]) if interleaved else (turned[..., :n], turned[..., n:])
    a, b = a * cos - b * sin, b * cos + a * sin
    return torch.cat([torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1), rest], -1)


def _plain_qk(case, d):
    dt, il = _tdtype(case), case["interleaved"]
    angle = d["positions"].double()[:, None] * d["inv_freq"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    out = {}
    for n in ("q", "k"):
        x, w = d[n].float(), d["w_" + n].float()
        r = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
        if case["dir"] == "fwd":
            out[n] = _rotate(x * r * w, cos, sin, il).to(dt)
            continue
        dn = _rotate(d["d" + n + "_out"].float(), cos, -sin, il)        # back by the same angles
        xh, u = x * r, dn * w
        out["d" + n] = (r * (u - xh * (u * xh).mean(-1, keepdim=True))).to(dt)
        out["dw_" + n] = (dn * xh).sum((0, 1)).to(dt)
    return out


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------
def work(case):
    b = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "ortho":
        # a symmetric product costs half.  Either every step by itself (A, A^2, the product with x), or all of them on the smaller
        # side, four symmetric products a step, and one product with x
        flops, steps = 0, case["steps"]
        for m, n in _shapes(case):
            s, l = min(m, n), max(m, n)
            flops += min(steps * (3 * s * s * l + s ** 3), 3 * s * s * l + max(1, 4 * steps - 3) * s ** 3)
        return {"bytes": 2 * b * sum(math.prod(s) for s in _shapes(case)), "flops": flops}
    t = case["tokens"]
    if case["op"] == "embed":
        h, ids = case["hidden"], case["ids"] // 8 * t
        if case["dir"] == "fwd":
            return {"bytes": 2 * b * t * h + ids, "flops": t * h}
        return {"bytes": b * (t + case["vocab"]) * h + ids, "flops": t * h}
    n = t * (case["heads_q"] + case["heads_k"]) * case["dim"]
    if case["dir"] == "fwd":
        return {"bytes": 2 * b * n + 8 * t, "flops": 8 * n}
    return {"bytes": 3 * b * n + 8 * t, "flops": 16 * n}


# ---------------------------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# ---------------------------------------------------------------------------------------------
def exact(case, seed):
    d = _inputs(case, seed)
    return {"ortho": _exact_ortho, "embed": _exact_embed, "qk": _exact_qk}[case["op"]](case, d)


def _exact_ortho(case, d):
    """Products from the other side for tall matrices, and the polynomial from its highest power down."""
    a, b, c = NS_COEFS
    out = []
    for g, scale in zip(_parts(d["grads"], _shapes(case)), _scales(case)):
        x = g.double()
        x /= torch.linalg.vector_norm(x) + NS_EPS
        tall = x.shape[0] > x.shape[1]
        for _ in range(case["steps"]):
            gram = x.t().mm(x) if tall else x.mm(x.t())
            eye = torch.eye(gram.shape[0], device="cuda", dtype=torch.float64)
            poly = gram.mm(c * gram + b * eye) + a * eye
            x = x.mm(poly) if tall else poly.mm(x)
        out.append((scale * x).reshape(-1))
    return {"updates": torch.cat(out)}


def _exact_embed(case, d):
    row = d["ids"].long() - case["first"]
    row = torch.where((row < 0) | (row >= case["vocab"]), case["vocab"], row)         # one row more, of zeros
    if case["dir"] == "fwd":
        table = torch.cat([d["table"].double(), torch.zeros(1, case["hidden"], device="cuda", dtype=torch.float64)])
        return {"x": torch.nn.functional.embedding(row, table) * case["scale"]}
    # running sums over the tokens in the order of their rows: a row's sum is the difference across its tokens
    order = torch.argsort(row, stable=True)
    sums = torch.cat([torch.zeros(1, case["hidden"], device="cuda", dtype=torch.float64), d["dy"].double()[order].cumsum(0)])
    ends = torch.searchsorted(row[order], torch.arange(case["vocab"] + 1, device="cuda"))
    return {"dtable": (sums[ends[1:]] - sums[ends[:-1]]) * case["scale"]}


def _exact_qk(case, d):
    """The rotation as a product of complex numbers, gradients by the rules of torch's differentiation."""
    turn = torch.polar(torch.ones((), device="cuda", dtype=torch.float64), d["positions"].double()[:, None] * d["inv_freq"])[:, None]
    n, out = turn.shape[-1], {}
    for name in ("q", "k"):
        x, w = d[name].double().requires_grad_(), d["w_" + name].double().requires_grad_()
        y = x / torch.sqrt((x * x).sum(-1, keepdim=True) / case["dim"] + EPS) * w
        pairs = y[..., :2 * n].unflatten(-1, (n, 2)) if case["interleaved"] else y[..., :2 * n].unflatten(-1, (2, n)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        z = (z if case["interleaved"] else z.transpose(-1, -2)).flatten(-2)
        y = torch.cat([z, y[..., 2 * n:]], -1)
        if case["dir"] == "fwd":
            out[name] = y.detach()
        else:
            out["d" + name], out["dw_" + name] = torch.autograd.grad(y, (x, w), d["d" + name + "_out"].double())
    return out
