"""What the speed of the training-block operators is measured on: the gated feed-forward block and the norms around it, whose
backward passes make the gradients that the compressor takes, and the global norm and clipping of what it hands back.

``run`` computes an operator in its plain form (32 bits, elementary torch operations, one rounding at the end), or, where
``own`` is set, through the public entry points of ``paper_2511_10333_amd``.

Fields of a case: ``op`` ("clip", "ff", "norm"), ``dtype`` ("f32", "bf16") and
  clip: ``shapes`` ("MxN" a matrix, "N" a vector, ";KxMxN" the list K times), ``max_norm``
  ff:   ``dir`` ("fwd", "bwd"), ``tokens``, ``hidden``, ``ff``, ``act`` ("silu", "gelu", "gelu_tanh"), ``pad`` (columns by which
        the rows of the activations are further apart than they are long), ``keep`` (forward: the two projections are kept for
        the backward pass)
  norm: ``dir``, ``tokens``, ``hidden``, ``rows_per_gate`` (0: no gate; else tokens that share a row of the gate), ``scale``
"""
import math

import torch

own = False

EPS = 1e-6          # of the norms, beside the mean square; of the clipping, beside the norm


# ---------------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------------
def _text(shapes):
    return ",".join("x".join(str(d) for d in s) for s in shapes)


def _block(hidden):
    """The four 2-D gradients of a block."""
    h = hidden
    return [(h, 3 * h), (h, h), (h, 4 * h), (4 * h, h)]


def _vectors(hidden):
    """Its norm weights and biases."""
    h = hidden
    return [(h,), (h,), (3 * h,), (h,), (h,), (h,), (4 * h,), (h,)]


def _clip(name, shapes, layers, dtype, max_norm):
    c = {"op": "clip", "shapes": _text(shapes), "layers": layers, "dtype": dtype, "max_norm": max_norm}
    return dict(c, name=name) if name else c


def _ff(name, direction, tokens, hidden, ff, dtype, act, pad=0, keep=False):
    c = {"op": "ff", "dir": direction, "tokens": tokens, "hidden": hidden, "ff": ff, "dtype": dtype, "act": act, "pad": pad,
         "keep": keep}
    return dict(c, name=name) if name else c


def _norm(name, direction, tokens, hidden, dtype, rows_per_gate, scale):
    c = {"op": "norm", "dir": direction, "tokens": tokens, "hidden": hidden, "dtype": dtype, "rows_per_gate": rows_per_gate,
         "scale": scale}
    return dict(c, name=name) if name else c


def listed():
    return [
        # a small block's gradients, 4 matrices and 8 vectors: launches and latency
        _clip("clip_block_h512_bf16", _block(512) + _vectors(512), 1, "bf16", 1.0),
        # a whole pipeline stage of 8 layers, 32 tensors, 1.6e9 elements: what a large job clips every step
        _clip("clip_stage8_h4096_f32", _block(4096), 8, "f32", 1.0),
        # one token of a request being answered: the weights are read once and that is all
        _ff("ff_fwd_token_h4096_bf16", "fwd", 1, 4096, 16384, "bf16", "silu"),
        # a few requests at once, fp32
        _ff("ff_fwd_24_h2048_f32", "fwd", 24, 2048, 8192, "f32", "gelu"),
        # a large model's micro-batch, the forward pass of a training step
        _ff("ff_fwd_8192_h5120_bf16", "fwd", 8192, 5120, 20480, "bf16", "silu", keep=True),
        # a training step's backward, bf16
        _ff("ff_bwd_4096_h4096_bf16", "bwd", 4096, 4096, 16384, "bf16", "silu"),
        # a training step's backward, fp32 gradients
        _ff("ff_bwd_2048_h2048_f32", "bwd", 2048, 2048, 8192, "f32", "silu"),
        # ragged on every side, rows further apart than they are long
        _ff("ff_bwd_odd_f32", "bwd", 1001, 997, 2731, "f32", "gelu", pad=3),
        # one token between two blocks
        _norm("norm_fwd_token_h4096_bf16", "fwd", 1, 4096, "bf16", 0, 1.0),
        # a large micro-batch between two blocks, a gate for each sequence
        _norm("norm_fwd_16384_h5120_bf16", "fwd", 16384, 5120, "bf16", 2048, 0.25),
        # its backward, gradients of shared gates and weights among the outputs
        _norm("norm_bwd_8192_h4096_bf16", "bwd", 8192, 4096, "bf16", 2048, 0.25),
        # ragged rows in fp32, one gate for all tokens
        _norm("norm_bwd_odd_f32", "bwd", 3001, 1001, "f32", 3001, 0.5),
    ]


def _log_int(rng, lo, hi):
    d = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return d + 1 if d == 3072 else d        # (a size that nothing here has)


def _size(rng, lo, hi):
    """A size in [lo, hi]: as it comes, or a multiple of 64."""
    d = _log_int(rng, lo, hi)
    d = max(64, d // 64 * 64) if rng.random() < 0.5 else d
    return d + 64 if d == 3072 else d


def draw(rng):
    op = rng.choice(["clip", "ff", "ff", "norm"])
    dtype = rng.choice(["f32", "bf16"])
    if op == "clip":
        max_norm = rng.choice([0.25, 1.0, 1.0, 1e6])
        if rng.random() < 0.5:
            hidden, layers = _size(rng, 128, 4096), rng.choice([1, 2, 4])
            shapes = [s for s in _block(hidden) + _vectors(hidden) if 3072 not in s]
            return _clip(None, shapes, layers, dtype, max_norm)
        shapes = [(_size(rng, 1, 8192), _size(rng, 1, 8192)) if rng.random() < 0.7 else (_log_int(rng, 1, 100000),)
                  for _ in range(rng.randint(1, 12))]
        return _clip(None, shapes, 1, dtype, max_norm)
    direction = rng.choice(["fwd", "bwd"])
    if op == "norm":
        tokens, hidden = _log_int(rng, 1, 16384), _size(rng, 64, 8192)
        rows = rng.choice([0, 1, tokens, max(1, tokens // 4), _log_int(rng, 1, tokens)])
        return _norm(None, direction, tokens, hidden, dtype, rows, rng.choice([1.0, 0.5, 0.1]))
    while True:
        tokens, hidden, ff = _log_int(rng, 1, 8192), _size(rng, 64, 5120), _size(rng, 128, 20480)
        if rng.random() < 0.5:
            tokens = (tokens + 31) // 32 * 32 + (32 if 3040 < tokens <= 3072 else 0)
        work = (6 if direction == "fwd" else 12) * tokens * hidden * ff
        if work <= (4e12 if dtype == "bf16" else 1e12):
            return _ff(None, direction, tokens, hidden, ff, dtype, rng.choice(["silu", "silu", "gelu", "gelu_tanh"]),
                       rng.choice([0, 0, 0, 64, 5]), direction == "fwd" and rng.random() < 0.5)


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def _shapes(case):
    return case["layers"] * [tuple(int(d) for d in s.split("x")) for s in case["shapes"].split(",")]


def _tdtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _parts(flat, shapes):
    """Views of a slab of gradients, one behind the other."""
    sizes = [math.prod(s) for s in shapes]
    return [p.view(s) for p, s in zip(torch.split(flat, sizes), shapes)]


def _groups(case):
    """Rows of the gate."""
    r = case["rows_per_gate"]
    return -(-case["tokens"] // r) if r else 0


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed * 1000003 + 29)
    dt = _tdtype(case)

    def randn(*s, std=1.0, pad=0):
        x = torch.randn(*s[:-1], s[-1] + pad, generator=g, device="cuda").mul_(std).to(dt)
        return x[..., :s[-1]]

    if case["op"] == "clip":
        shapes = _shapes(case)
        flat = torch.empty(sum(math.prod(s) for s in shapes), device="cuda", dtype=dt)
        for i, p in enumerate(_parts(flat, shapes)):      # layers differ in the scale of their gradients
            p.copy_(torch.randn(p.shape, generator=g, device="cuda").mul_(1e-3 * (1 + i % 5)))
        return {"grads": flat}
    t, h = case["tokens"], case["hidden"]
    if case["op"] == "ff":
        f, pad = case["ff"], case["pad"]
        d = {"x": randn(t, h, pad=pad), "w_gate": randn(f, h, std=h ** -0.5), "w_up": randn(f, h, std=h ** -0.5),
             "w_down": randn(h, f, std=f ** -0.5)}
        if case["dir"] == "bwd":
            # what the forward pass kept: the two projections, of about unit variance under such weights
            d |= {"gate": randn(t, f), "up": randn(t, f), "dy": randn(t, h, std=1e-3, pad=pad)}
        return d
    groups = _groups(case)
    d = {"y": randn(t, h, std=3.0), "w_post": 1 + randn(h, std=0.1), "w_pre": 1 + randn(h, std=0.1),
         "gate": randn(groups, h) if groups else None}
    if case["dir"] == "fwd":
        return d | {"x": randn(t, h)}
    # backward: what the forward pass left (the sum and both reciprocal roots) and the two gradients that come in
    d |= {"x_out": randn(t, h), "dx_out": randn(t, h, std=1e-3), "dn": randn(t, h, std=1e-3)}
    for k, of in (("rstd_post", "y"), ("rstd_pre", "x_out")):
        d[k] = (d[of].float().square().mean(1) + EPS).rsqrt()
    return d


def prepare(case, seed):
    state = {"case": case, "in": _inputs(case, seed)}
    if not own:
        return state
    import paper_2511_10333_amd as edgc
    d, dt = state["in"], _tdtype(case)
    ctx = state["ctx"] = edgc.Context(0, max_bins=256, max_rank=16, max_rows=64, max_cols=64)
    like = lambda *names: {"d" + n if n[0] != "d" else n: torch.empty(d[n].shape, device="cuda", dtype=dt) for n in names if d[n] is not None}
    if case["op"] == "clip":
        state["out"] = {"grads": torch.empty_like(d["grads"]), "norm_coef": torch.empty(2, device="cuda")}
        shapes = _shapes(case)
        state["batch"] = edgc.PreparedBatch([edgc.Tensor(a, b) for a, b in zip(_parts(d["grads"], shapes),
                                                                             _parts(state["out"]["grads"], shapes))])
        return state
    t, h = case["tokens"], case["hidden"]
    if case["op"] == "ff":
        state["ff"] = edgc.FeedForward(d["w_gate"], d["w_up"], d["w_down"], case["act"])
        ctx.reserve_ff(dt, t, h, case["ff"], backward=case["dir"] == "bwd")
        if case["dir"] == "bwd":
            state["out"] = like("x", "w_gate", "w_up", "w_down")
            return state
        state["out"] = {"y": torch.empty((t, h), device="cuda", dtype=dt)}
        if case["keep"]:
            state["out"] |= {k: torch.empty((t, case["ff"]), device="cuda", dtype=dt) for k in ("gate", "up")}
        return state
    if case["dir"] == "fwd":
        state["out"] = {k: torch.empty((t, h), device="cuda", dtype=dt) for k in ("x_out", "n")}
        state["out"] |= {k: torch.empty(t, device="cuda") for k in ("rstd_post", "rstd_pre")}
    else:
        ctx.reserve_block_norm(t, h)
        state["out"] = like("y", "w_post", "w_pre", "gate") | {"dx": torch.empty((t, h), device="cuda", dtype=dt)}
    return state


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------
def run(state):
    case, d = state["case"], state["in"]
    if not own:
        return {"clip": _plain_clip, "ff": _plain_ff, "norm": _plain_norm}[case["op"]](case, d)
    ctx, out = state["ctx"], state["out"]
    if case["op"] == "clip":
        ctx.grad_sumsq_batch(state["batch"])
        ctx.clip_batch(state["batch"], case["max_norm"], out["norm_coef"])
    elif case["op"] == "ff" and case["dir"] == "fwd":
        ctx.ff_forward(state["ff"], d["x"], out["y"], out.get("gate"), out.get("up"))
    elif case["op"] == "ff":
        ctx.ff_backward(state["ff"], d["x"], d["gate"], d["up"], d["dy"], out["dx"], out["dw_gate"], out["dw_up"], out["dw_down"])
    elif case["dir"] == "fwd":
        ctx.block_norm_forward(d["x"], d["y"], d["w_post"], d["gate"], d["w_pre"], out["x_out"], out["n"], out["rstd_post"],
                               out["rstd_pre"], scale=case["scale"], eps=EPS, rows_per_gate=case["rows_per_gate"])
    else:
        ctx.block_norm_backward(d["dx_out"], d["dn"], d["x_out"], d["y"], d["w_post"], d["gate"], d["w_pre"], d["rstd_post"],
                                d["rstd_pre"], out["dx"], out["dy"], out["dw_post"], out.get("dgate"), out["dw_pre"],
                                scale=case["scale"], rows_per_gate=case["rows_per_gate"])
    return out


def _plain_clip(case, d):
    parts = _parts(d["grads"], _shapes(case))
    norm = torch.stack([p.float().square().sum() for p in parts]).sum().sqrt()
    coef = (case["max_norm"] / (norm + EPS)).clamp(max=1.0)
    coef = torch.where(torch.isfinite(norm), coef, 1.0)
    return {"grads": (d["grads"].float() * coef).to(_tdtype(case)), "norm_coef": torch.stack([norm, coef])}


def _act(name, z):
    """The activation and its derivative."""
    if name == "silu":
        s = 1 / (1 + torch.exp(-z))
        return z * s, s * (1 + z * (1 - s))
    if name == "gelu":
        cdf = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
        return z * cdf, cdf + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    k = math.sqrt(2 / math.pi)
    th = torch.tanh(k * (z + 0.044715 * z * z * z))
    return 0.5 * z * (1 + th), 0.5 * (1 + th) + 0.5 * z * (1 - th * th) * k * (1 + 3 * 0.044715 * z * z)


def _plain_ff(case, d):
    dt = _tdtype(case)
    x, wg, wu, wd = (d[k].float() for k in ("x", "w_gate", "w_up", "w_down"))
    if case["dir"] == "fwd":
        gate, up = x @ wg.t(), x @ wu.t()
        y = (_act(case["act"], gate)[0] * up) @ wd.t()
        return {"y": y.to(dt), "gate": gate.to(dt), "up": up.to(dt)} if case["keep"] else {"y": y.to(dt)}
    gate, up, dy = (d[k].float() for k in ("gate", "up", "dy"))
    a, da = _act(case["act"], gate)
    dh = dy @ wd
    dgate, dup = dh * up * da, dh * a
    return {"dx": (dgate @ wg + dup @ wu).to(dt), "dw_gate": (dgate.t() @ x).to(dt), "dw_up": (dup.t() @ x).to(dt),
            "dw_down": (dy.t() @ (a * up)).to(dt)}


def _rows_of(case, gate):
    """The gate of each token."""
    r = case["rows_per_gate"]
    return 1.0 if gate is None else gate.repeat_interleave(r, 0)[:case["tokens"]]


def _plain_norm(case, d):
    dt, s = _tdtype(case), case["scale"]
    y, wpost, wpre = (d[k].float() for k in ("y", "w_post", "w_pre"))
    gate = _rows_of(case, None if d["gate"] is None else d["gate"].float())
    if case["dir"] == "fwd":
        r1 = (y.square().mean(1) + EPS).rsqrt()
        x1 = d["x"].float() + s * gate * (y * r1[:, None] * wpost)
        r2 = (x1.square().mean(1) + EPS).rsqrt()
        return {"x_out": x1.to(dt), "n": (x1 * r2[:, None] * wpre).to(dt), "rstd_post": r1, "rstd_pre": r2}
    r1, r2 = d["rstd_post"][:, None], d["rstd_pre"][:, None]
    dn, xh, yh = d["dn"].float(), d["x_out"].float() * r2, y * r1
    u = dn * wpre
    dx = d["dx_out"].float() + r2 * (u - xh * (u * xh).mean(1, keepdim=True))
    v = s * gate * dx * wpost
    dy = r1 * (v - yh * (v * yh).mean(1, keepdim=True))
    out = {"dx": dx.to(dt), "dy": dy.to(dt), "dw_pre": (dn * xh).sum(0).to(dt), "dw_post": (s * gate * dx * yh).sum(0).to(dt)}
    if d["gate"] is not None:
        per = s * wpost * dx * yh
        pad = _groups(case) * case["rows_per_gate"] - case["tokens"]
        per = torch.cat([per, per.new_zeros(pad, case["hidden"])])
        out["dgate"] = per.view(_groups(case), case["rows_per_gate"], -1).sum(1).to(dt)
    return out


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------
def work(case):
    b = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "clip":
        n = sum(math.prod(s) for s in _shapes(case))
        return {"bytes": 2 * b * n + 8, "flops": 3 * n}
    t, h = case["tokens"], case["hidden"]
    if case["op"] == "ff":
        f = case["ff"]
        if case["dir"] == "fwd":
            return {"bytes": b * (2 * t * h + 3 * h * f + (2 * t * f if case["keep"] else 0)), "flops": 6 * t * h * f}
        return {"bytes": b * (3 * t * h + 2 * t * f + 6 * h * f), "flops": 12 * t * h * f}
    groups = _groups(case)
    if case["dir"] == "fwd":
        return {"bytes": b * (4 * t * h + 2 * h + groups * h) + 8 * t, "flops": 10 * t * h}
    return {"bytes": b * (6 * t * h + 4 * h + 2 * groups * h) + 8 * t, "flops": 24 * t * h}


# ---------------------------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# ---------------------------------------------------------------------------------------------
def exact(case, seed):
    d = {k: None if v is None else v.double() for k, v in _inputs(case, seed).items() if k != "grads"}
    if case["op"] == "clip":
        return _exact_clip(case, _inputs(case, seed)["grads"])
    return (_exact_ff if case["op"] == "ff" else _exact_norm)(case, d)


def _exact_clip(case, flat):
    chunks = torch.split(flat, 1 << 26)
    norm = math.sqrt(math.fsum(float((c.double() ** 2).sum()) for c in chunks))
    coef = min(1.0, case["max_norm"] / (norm + EPS)) if math.isfinite(norm) else 1.0
    return {"grads": flat.double() * coef, "norm_coef": torch.tensor([norm, coef], dtype=torch.float64)}


def _exact_ff(case, d):
    """Gradients by the rules of torch's differentiation, of the same block written with torch's own activations."""
    act = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu,
           "gelu_tanh": lambda z: torch.nn.functional.gelu(z, approximate="tanh")}[case["act"]]
    if case["dir"] == "fwd":
        gate, up = d["x"].mm(d["w_gate"].t()), d["x"].mm(d["w_up"].t())
        y = (act(gate) * up).mm(d["w_down"].t())
        return {"y": y, "gate": gate, "up": up} if case["keep"] else {"y": y}
    gate, up = d["gate"].requires_grad_(), d["up"].requires_grad_()
    h = act(gate) * up
    dh = d["dy"].mm(d["w_down"])
    dgate, dup = torch.autograd.grad(h, (gate, up), dh)
    return {"dx": torch.cat([dgate, dup], 1).mm(torch.cat([d["w_gate"], d["w_up"]], 0)), "dw_gate": dgate.t().mm(d["x"]),
            "dw_up": dup.t().mm(d["x"]), "dw_down": d["dy"].t().mm(h.detach())}


def _exact_norm(case, d):
    t, h, s, r = case["tokens"], case["hidden"], case["scale"], case["rows_per_gate"]
    row = torch.arange(t, device="cuda") // r if r else None
    root = lambda z: 1 / torch.sqrt((z * z).sum(1, keepdim=True) / h + EPS)
    if case["dir"] == "fwd":
        a = s * d["w_post"] * (d["gate"][row] if r else 1.0)
        r1 = root(d["y"])
        x1 = d["x"] + a * (d["y"] * r1)
        r2 = root(x1)
        return {"x_out": x1, "n": x1 * r2 * d["w_pre"], "rstd_post": r1.view(-1), "rstd_pre": r2.view(-1)}
    yh, xh = d["y"] * d["rstd_post"][:, None], d["x_out"] * d["rstd_pre"][:, None]
    u = d["dn"] * d["w_pre"]
    dx = d["dx_out"] + d["rstd_pre"][:, None] * (u - xh * ((u * xh).sum(1, keepdim=True) / h))
    gate = d["gate"][row] if r else torch.ones_like(dx)
    v = s * gate * d["w_post"] * dx
    out = {"dx": dx, "dy": d["rstd_post"][:, None] * (v - yh * ((v * yh).sum(1, keepdim=True) / h)),
           "dw_pre": (d["dn"] * xh).sum(0), "dw_post": (s * gate * dx * yh).sum(0)}
    if r:
        out["dgate"] = torch.zeros_like(d["gate"]).index_add_(0, row, s * d["w_post"] * dx * yh)
    return out
