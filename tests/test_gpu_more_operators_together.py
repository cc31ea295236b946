"""The operators before, in and after the stack of blocks together, as a training step runs them."""
import math

import pytest
import torch

import paper_2511_10333_amd as edgc
from paper_2511_10333_amd import train_block as tb

pytestmark = pytest.mark.gpu

T, H, V, HQ, HK, D, ROT, EPS = 96, 64, 200, 4, 2, 16, 12, 1e-6
SCALE = 3.0


def leaves(seed):
    g = torch.Generator().manual_seed(seed)
    randn = lambda *s, std=1.0, mean=0.0: mean + std * torch.randn(*s, generator=g)
    return {"table": randn(V, H, std=0.3), "w_pre": randn(H, std=0.1, mean=1.0), "w_qkv": randn((HQ + 2 * HK) * D, H, std=H ** -0.5),
            "w_q": randn(D, std=0.1, mean=1.0), "w_k": randn(D, std=0.1, mean=1.0), "w_o": randn(H, HQ * D, std=(HQ * D) ** -0.5)}


def attention(q, k, v):
    """Plain and causal, tokens x heads x dim, groups of queries' heads to a key's."""
    k, v = (x.repeat_interleave(HQ // HK, 1).transpose(0, 1).contiguous() for x in (k, v))
    s = q.transpose(0, 1).contiguous() @ k.transpose(1, 2).contiguous() / math.sqrt(D)
    s = s.masked_fill(torch.ones(T, T, device=s.device).triu(1).bool(), float("-inf"))
    return (torch.softmax(s, -1) @ v).transpose(0, 1).reshape(T, HQ * D)


def reference(w, ids, pos, f, dy):
    """The same in 64 bits by torch's differentiation."""
    w = {k: x.double().requires_grad_() for k, x in w.items()}
    norm = lambda x: x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    x = SCALE * w["table"][ids.clamp(0, V - 1)] * ((ids >= 0) & (ids < V))[:, None]
    qkv = (norm(x) * w["w_pre"]) @ w["w_qkv"].t()
    q, k, v = qkv[:, :HQ * D].view(T, HQ, D), qkv[:, HQ * D:(HQ + HK) * D].view(T, HK, D), qkv[:, (HQ + HK) * D:].view(T, HK, D)
    angle = (pos.double()[:, None] * f)[:, None]

    def turn(x):
        a, b, rest = x[..., :ROT // 2], x[..., ROT // 2:ROT], x[..., ROT:]
        return torch.cat([a * torch.cos(angle) - b * torch.sin(angle), b * torch.cos(angle) + a * torch.sin(angle), rest], -1)
    y = x + attention(turn(norm(q) * w["w_q"]), turn(norm(k) * w["w_k"]), v) @ w["w_o"].t()
    return y.detach(), dict(zip(w, torch.autograd.grad(y, list(w.values()), dy.double())))


def rel(a, b):
    return float((a.double().cpu() - b).norm() / b.norm())


def test_tokens_through_attention_and_the_gradients_into_an_update():
    """Embedding, norm, product, norms of queries and keys in the rows that the product gave, attention, and back; the gradients clipped and the matrices
    orthogonalised as lists."""
    ctx = edgc.Context(0, max_bins=64, max_rank=4, max_rows=64, max_cols=64)
    g = torch.Generator().manual_seed(1)
    host = leaves(2)
    ids, pos, f = torch.randint(-3, V + 3, (T,), generator=g), torch.arange(5000, 5000 + T), 10000.0 ** (-torch.arange(0, ROT, 2, dtype=torch.float64) / ROT)
    dy = 1e-2 * torch.randn(T, H, generator=g)
    want_y, want = reference(host, ids, pos, f, dy)

    w = {k: x.cuda() for k, x in host.items()}
    ids, pos, f, dy = ids.cuda(), pos.cuda(), f.cuda(), dy.cuda()
    new = lambda *s: torch.empty(s, device="cuda")
    x, n, r = new(T, H), new(T, H), new(T)
    ctx.embed_forward(w["table"], ids, x, scale=SCALE)
    ctx.block_norm_forward(x, None, None, None, w["w_pre"], None, n, None, r, eps=EPS)
    qkv = n @ w["w_qkv"].t()
    q, k, v = qkv[:, :HQ * D].view(T, HQ, D), qkv[:, HQ * D:(HQ + HK) * D].view(T, HK, D), qkv[:, (HQ + HK) * D:].view(T, HK, D)
    qr, kr = new(T, HQ, D), new(T, HK, D)
    ctx.qk_norm_forward(q, k, w["w_q"], w["w_k"], pos, f, qr, kr, eps=EPS)
    qr.requires_grad_(), kr.requires_grad_()
    v = v.detach().clone().requires_grad_()
    o = attention(qr, kr, v)
    y = x + o.detach() @ w["w_o"].t()
    # fp32 through two norms, two products and the softmax: some hundred units of 2^-23 in the norm
    assert rel(y, want_y) < 200 * 2.0 ** -23

    grads = {k: torch.full_like(t, 9.0) for k, t in w.items()}
    grads["w_o"].copy_(dy.t() @ o.detach())
    dqr, dkr, dv = torch.autograd.grad(o, (qr, kr, v), dy @ w["w_o"])
    dqkv = new(T, (HQ + 2 * HK) * D)
    ctx.reserve_qk_norm(T, HQ, HK, D)
    ctx.qk_norm_backward(dqr.contiguous(), dkr.contiguous(), q, k, w["w_q"], w["w_k"], pos, f, dqkv[:, :HQ * D].view(T, HQ, D),
                         dqkv[:, HQ * D:(HQ + HK) * D].view(T, HK, D), grads["w_q"], grads["w_k"], eps=EPS)
    dqkv[:, (HQ + HK) * D:] = dv.reshape(T, HK * D)
    grads["w_qkv"].copy_(dqkv.t() @ n)
    dx = new(T, H)
    ctx.reserve_block_norm(T, H)
    ctx.block_norm_backward(dy, dqkv @ w["w_qkv"], x, None, None, None, w["w_pre"], None, r, dx, None, None, None, grads["w_pre"])
    ctx.reserve_embed(T, V, H)
    ctx.embed_backward(ids, dx, grads["table"], scale=SCALE)
    for key, got in grads.items():
        assert rel(got, want[key]) < 400 * 2.0 ** -23, key

    # the list's norm, and the two projections' gradients as an update
    batch = edgc.PreparedBatch([edgc.Tensor(t, t) for t in grads.values()])
    nc = torch.zeros(2, device="cuda")
    ctx.grad_sumsq_batch(batch)
    ctx.clip_batch(batch, 0.01, nc)
    matrices = [grads["w_qkv"], grads["w_o"]]
    ctx.reserve_orthogonalize(torch.float32, [tuple(m.shape) for m in matrices])
    ctx.orthogonalize_batch([edgc.Tensor(m, m) for m in matrices])
    for key in ("w_qkv", "w_o"):
        z = torch.linalg.svdvals(grads[key].double().cpu())
        before = torch.linalg.svdvals(want[key])
        # all but the directions that the gradient hardly has come out near one
        assert float(z.max()) < 1.3 and float(z[before > 0.02 * before.norm()].min()) > 0.6
    ctx.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_short_run_on_tokens_with_the_orthogonalised_update(dtype):
    reports = []
    losses = tb.train(layers=2, hidden=128, ff=256, tokens=256, sequence=64, steps=12, window=4, dtype=dtype, lr=0.02, vocab=300, update="orthogonal",
                      report=reports.append)
    assert len(losses) == 12 and all(math.isfinite(v) for v in losses)
    assert len(reports) == 3 and all(r["clip"] <= 1.0 and r["grad_norm"] > 0 for r in reports)


def test_gradients_of_a_stack_of_blocks_over_tokens():
    """The example's own passes: the table's gradient is that of the inputs' rows, summed by token."""
    ctx = edgc.Context(0, max_bins=64, max_rank=4, max_rows=64, max_cols=64)
    model = tb.Model(ctx, 2, 64, 96, 100, 50, seed=3, vocab=17)
    ids = torch.randint(0, 17, (100,), generator=torch.Generator().manual_seed(4)).cuda()
    dn = 1e-2 * torch.randn(100, 64, generator=torch.Generator().manual_seed(5)).cuda()
    out = model.forward_tokens(ids).clone()
    model.backward_tokens(ids, dn)
    table = model.g_table.clone()
    assert torch.equal(model.forward(model.table[ids]), out)
    dx = model.backward(dn).double()
    want = torch.zeros(17, 64, dtype=torch.float64, device="cuda").index_add_(0, ids, dx)
    assert float((table.double() - want).abs().max()) <= 100 * 2.0 ** -24 * float(dx.abs().sum(0).max())
    ctx.close()


def test_a_captured_step_replays_as_it_ran_beside_an_eager_one():
    """Tokens to update in one graph, on one context, with eager calls of the same context between its replays."""
    ctx = edgc.Context(0, max_bins=64, max_rank=4, max_rows=64, max_cols=64)
    model = tb.Model(ctx, 2, 128, 256, 192, 64, torch.bfloat16, seed=7, vocab=50)
    matrices = [g[k] for g in model.grads for k in ("w_gate", "w_up", "w_down")]
    outs = [torch.empty_like(m) for m in matrices]
    ctx.reserve_orthogonalize(torch.bfloat16, [tuple(m.shape) for m in matrices])
    batch = edgc.PreparedBatch([edgc.Tensor(m, o) for m, o in zip(matrices, outs)])
    ids, dn = torch.zeros(192, dtype=torch.int64, device="cuda"), torch.zeros(192, 128, device="cuda", dtype=torch.bfloat16)

    def go():
        model.forward_tokens(ids)
        model.backward_tokens(ids, dn)
        ctx.orthogonalize_batch(batch)
    fill = lambda s: (ids.copy_(torch.randint(0, 50, (192,), generator=torch.Generator().manual_seed(s))),
                      dn.copy_(1e-2 * torch.randn(192, 128, generator=torch.Generator().manual_seed(s + 100))))
    fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for s in (1, 2, 3, 1):
        fill(s)
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in outs + [model.g_table, model.n_last]]
        go()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, outs + [model.g_table, model.n_last]))
    ctx.close()
