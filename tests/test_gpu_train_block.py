"""The operators together, as a training step runs them: gradients through a stack of blocks, and a short run."""
import pytest
import torch

import paper_2511_10333_amd as edgc
from paper_2511_10333_amd import train_block as tb

pytestmark = pytest.mark.gpu


def _reference(model, x, dn):
    """The same stack in 64 bits by torch's differentiation: its output and the gradients of x and of every weight."""
    leaf = lambda t: t.detach().double().cpu().requires_grad_()
    norm = lambda v: v * torch.rsqrt((v * v).mean(1, keepdim=True) + 1e-6)
    blocks = [{k: leaf(w) for k, w in b.items()} for b in model.blocks]
    last, x0 = leaf(model.w_last), leaf(x)
    h = x0
    row = torch.arange(model.tokens) // model.sequence
    for b in blocks:
        n = norm(h) * b["w_pre"]
        y = (torch.nn.functional.silu(n @ b["w_gate"].t()) * (n @ b["w_up"].t())) @ b["w_down"].t()
        h = h + model.scale * b["gate"][row] * (norm(y) * b["w_post"])
    out = norm(h) * last
    leaves = [b[k] for b in blocks for k in b] + [last]
    grads = torch.autograd.grad(out, leaves + [x0], dn.double().cpu())
    return out.detach(), grads[:-1], grads[-1]


@pytest.mark.parametrize("tokens", [100, 200])      # few enough for the streaming products' edge, and tiles that end inside
def test_gradients_through_a_stack_of_blocks(tokens):
    ctx = edgc.Context(0, max_bins=64, max_rank=4, max_rows=64, max_cols=64)
    model = tb.Model(ctx, 3, 96, 160, tokens, 64, seed=3)
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(tokens, 96, generator=g, device="cuda")
    dn = 1e-2 * torch.randn(tokens, 96, generator=g, device="cuda")
    out = model.forward(x)
    dx = model.backward(dn)
    want, grads, want_dx = _reference(model, x, dn)
    # fp32 through three blocks of two products and two norms each: some hundred units of 2^-23 in the norm
    rel = lambda a, b: float((a.double().cpu() - b).norm() / b.norm())
    assert rel(out, want) < 300 * 2.0 ** -23 and rel(dx, want_dx) < 300 * 2.0 ** -23
    for (_, got), w in zip(model.parameters(), grads):
        assert rel(got, w) < 300 * 2.0 ** -23
    ctx.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_short_run_learns_and_compresses(dtype):
    reports = []
    losses = tb.train(layers=2, hidden=256, ff=512, tokens=512, sequence=128, steps=30, window=5, dtype=dtype, report=reports.append)
    assert all(l == l for l in losses)
    assert sum(losses[-5:]) < 0.8 * sum(losses[:5])
    assert len(reports) == 6 and all(r["clip"] <= 1.0 and r["grad_norm"] > 0 for r in reports)


def test_a_captured_step_replays_as_it_ran():
    """Norms, feed-forward block, their backward passes, gradient norm and clipping in one graph: no call allocates, waits or
    keeps anything from one pass for the next."""
    ctx = edgc.Context(0, max_bins=64, max_rank=4, max_rows=64, max_cols=64)
    model = tb.Model(ctx, 2, 128, 256, 192, 64, torch.bfloat16, seed=7)
    grads = [g for _, g in model.parameters()]
    sent = [torch.empty_like(g) for g in grads]
    clip = edgc.PreparedBatch([edgc.Tensor(g, o) for g, o in zip(grads, sent)])
    nc = torch.zeros(2, device="cuda")
    x, dn = torch.empty(192, 128, device="cuda", dtype=torch.bfloat16), torch.empty(192, 128, device="cuda", dtype=torch.bfloat16)

    def go():
        model.forward(x)
        model.backward(dn)
        ctx.grad_sumsq_batch(clip)
        ctx.clip_batch(clip, 0.01, nc)
    fill = lambda s: (x.copy_(torch.randn(192, 128, generator=torch.Generator().manual_seed(s))),
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
        replayed = [t.clone() for t in sent + [nc, model.n_last, model.d["x"]]]
        go()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, sent + [nc, model.n_last, model.d["x"]]))
    ctx.close()
