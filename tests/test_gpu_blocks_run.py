"""A residual block's calls together, as a job runs them: against autograd in 64 bits, in a torch.autograd.Function, and through the agent."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


def autograd(job, tokens, parameters):
    """(loss, gradients) of a micro-batch in 64 bits."""
    leaves = [p.double().clone().requires_grad_() for p in job.parts(parameters)]
    table, *inner, projection = leaves
    norm = lambda v, w: v * (v.square().mean(1, keepdim=True) + 1e-6).rsqrt() * w
    stream = table[tokens[:, :-1].reshape(-1)] * job.scale
    for k in range(job.blocks):
        before, w_in, after, gate, w_out = inner[5 * k:5 * k + 5]
        both = norm(stream, before) @ w_in.t()
        g, u = both[:, :job.width], both[:, job.width:]
        stream = stream + gate * norm((torch.nn.functional.silu(g) * u) @ w_out.t(), after)
    loss = torch.nn.functional.cross_entropy(norm(stream, inner[-1]) @ projection.t(), tokens[:, 1:].reshape(-1))
    loss.backward()
    return loss, [leaf.grad for leaf in leaves]


@pytest.mark.parametrize("kept", [None, "i8", "e4m3"])
@pytest.mark.parametrize("blocks,D,width", [(1, 64, 128), (3, 64, 72), (2, 40, 96)])
def test_a_micro_batch_has_the_gradient_autograd_gives(blocks, D, width, kept):
    """bfloat16 rows between the calls: as for the bare layer, a handful of roundings of 2^-8 of independent signs a block: within 2^-4 in the 2-norm for up to three blocks.  What is kept in 8 bits is off by
    at most 1/127 of the largest of 32 (i8), about 2^-8 of the rows in the 2-norm, or by 2^-4 an element, 2^-5.3 in the mean (e4m3), of independent signs from row to row: it moves a gradient by less than that share of what it is a
    factor of, three factors a block: 2^-2.5 in all."""
    from paper_2008_12260_amd.agent import Job
    job = Job(V=500, D=D, length=16, seed=1, blocks=blocks, width=width, kept=kept)
    tokens = job.examples(9)
    rounded = job.parameters.bfloat16()
    got = torch.empty(rounded.shape, dtype=torch.bfloat16, device="cuda")
    loss = job.micro_batch(tokens, job.parts(rounded), got)
    want, grads = autograd(job, tokens, rounded)
    assert abs(float(loss) - float(want.detach())) < 2.0 ** -6 * float(want.detach())
    bound = 2.0 ** -2.5 if kept == "e4m3" else 2.0 ** -4
    for g, w in zip(job.parts(got), grads):
        assert float((g.double() - w).norm()) <= bound * float(w.norm()), (g.shape, float((g.double() - w).norm() / w.norm()))


def test_a_jobs_iterations_with_blocks():
    from paper_2008_12260_amd.agent import Job
    for kept in (None, "i8"):
        job = Job(V=300, D=32, length=8, seed=2, blocks=2, kept=kept)
        before = job.parameters.clone()
        for s in (3, 0, 0):
            loss, noise, seconds = job.iteration(5, s)
            assert np.isfinite(loss) and seconds > 0
        assert noise is not None and np.isfinite(noise).all()
        assert all(bool((p != q).any()) for p, q in zip(job.parts(job.parameters), job.parts(before)))


def test_memory_bounds_the_batch():
    from paper_2008_12260_amd.agent import Job, run
    jobs = {kept: Job(V=300, D=64, length=16, seed=3, blocks=2, kept=kept) for kept in (None, "i8")}
    assert jobs["i8"].bytes_per_example() < 0.5 * jobs[None].bytes_per_example()
    memory = 20 * jobs[None].bytes_per_example()
    for kept, most in ((None, 20), ("i8", 32)):
        chosen = []
        state = run(jobs[kept], m0=8, m_max=32, rounds=1, iterations=4, memory=memory, on_round=lambda s, more: chosen.append(int(more["m_grid"].max())))
        assert chosen == [most] and all(m <= most for m, _, _ in state.records)
    with pytest.raises(ValueError, match="bytes hold"):
        run(jobs[None], m0=8, memory=jobs[None].bytes_per_example() * 7)


def test_what_a_micro_batch_remembers_is_what_is_counted():
    """Allocated between the passes, less what is there without the blocks: within the allocator's rounding of its few tensors."""
    from paper_2008_12260_amd.agent import Job
    import paper_2008_12260_amd as px
    for kept in (None, "i8"):
        job = Job(V=300, D=256, length=64, seed=4, blocks=3, width=512, kept=kept)
        m = 16
        seen = {}
        loss = px.agent.token_loss

        def watched(rows, *args, **more):
            torch.cuda.synchronize()
            seen["bytes"] = torch.cuda.memory_allocated()
            return loss(rows, *args, **more)
        model, gradient = job.parts(job.parameters.bfloat16()), torch.empty(job.parameters.numel(), dtype=torch.bfloat16, device="cuda")
        tokens = job.examples(m)
        px.agent.token_loss = watched
        try:
            job.micro_batch(tokens, model, gradient)
            seen.clear()
            torch.cuda.synchronize()
            base = torch.cuda.memory_allocated()
            job.micro_batch(tokens, model, gradient)
        finally:
            px.agent.token_loss = loss
        rows = m * job.length
        # beside what is remembered: the tokens, the last edge's rows and stats, and the last block's product, activation and branch, which Python still names
        around = rows * (16 + 2 * 2 * job.D + 16 + 2 * 3 * job.width + 2 * 2 * job.D + 33 * 2 * (job.D // 32))
        counted = m * job.bytes_per_example()
        assert counted - 64 * 1024 <= seen["bytes"] - base <= counted + around + 64 * 1024, (seen["bytes"] - base, counted, around)


def test_a_function_made_of_the_calls_has_the_gradients_autograd_gives():
    """fp32 throughout, D = 32 and 100 rows: each value is within 2^-17 of the sizes it is made of (see the edges' test), and those are within 2^5 of what is left of them."""
    import paper_2008_12260_amd as px

    class Edge(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, branch, gate, after, before):
            y, rows, ctx.state = px.block_edge(x, branch, gate=gate, after=px.Norm(after), before=px.Norm(before))
            ctx.save_for_backward(y, branch, gate, after, before)
            return y, rows

        @staticmethod
        def backward(ctx, dy, dh):
            y, branch, gate, after, before = ctx.saved_tensors
            d = px.block_edge_grad(dy.contiguous(), dh.contiguous(), ctx.state, y=y, branch=branch, gate=gate, after=px.Norm(after), before=px.Norm(before))
            return d.x, d.branch, d.gate, d.after_weight, d.before_weight

    class Gated(torch.autograd.Function):
        @staticmethod
        def forward(ctx, gate, up):
            ctx.save_for_backward(gate, up)
            return px.gated(gate, up, "gelu")[0]

        @staticmethod
        def backward(ctx, d):
            return px.gated_grad(d.contiguous(), *ctx.saved_tensors, "gelu")[:2]

    g = torch.Generator("cuda").manual_seed(5)
    start = [torch.randn(shape, generator=g, device="cuda") for shape in ((100, 32), (100, 32), (32,), (32,), (32,), (32, 64))]

    def net(edge, gated, x, z, gate, after, before, w):
        y, h = edge(x, z, gate, after, before)
        both = h @ w
        return (gated(both[:, :32], both[:, 32:]) * y).sum()
    norm = lambda v, w: v * (v.square().mean(1, keepdim=True) + 1e-6).rsqrt() * w

    def plain(x, z, gate, after, before):
        y = x + gate * norm(z, after)
        return y, norm(y, before)
    got, want = ([t.to(dtype).clone().requires_grad_() for t in start] for dtype in (torch.float32, torch.float64))
    net(Edge.apply, Gated.apply, *got).backward()
    net(plain, lambda a, b: torch.nn.functional.gelu(a) * b, *want).backward()
    for a, b in zip(got, want):
        assert float((a.grad.double() - b.grad).abs().max()) <= 2.0 ** -12 * float(b.grad.abs().max())
