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
    with pytest.raises(ValueError, match="has none"):
        run(Job(V=300, D=64, length=16), memory=memory)
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


def test_offsets_past_32_bits():
    """Rows whose elements, and whose bytes in 8 bits, lie beyond 2^32: what is done to the last ones is what is done to them alone."""
    import paper_2008_12260_amd as px
    last, D, N = 40, 16384, 300000
    assert (N - last) * D > 1 << 32
    g = torch.Generator("cuda").manual_seed(1)
    few = [torch.randn((last, D), generator=g, device="cuda").bfloat16() for _ in range(4)]
    many = [torch.zeros((N, D), dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    for big, small in zip(many, few):
        big[-last:] = small
    w = 1.0 + 0.1 * torch.randn(D, generator=g, device="cuda")
    edge = dict(after=px.Norm(w), before=px.Norm(w), gate=w)

    def same(a, b):
        assert torch.equal(a[-last:], b)
    y, rows, state = px.block_edge(many[0], many[1], **edge, keep="i8")
    y_few, rows_few, state_few = px.block_edge(few[0], few[1], **edge, keep="i8")
    same(y, y_few)
    same(rows, rows_few)
    for a, b in ((state.y_kept, state_few.y_kept), (state.branch_kept, state_few.branch_kept)):
        same(a.values, b.values)
        same(a.scales, b.scales)
    same(px.restore(state.y_kept), px.restore(state_few.y_kept))
    del y, rows
    a, b = (px.block_edge_grad(t[2], t[3], s, **edge, need=("x", "branch")) for t, s in ((many, state), (few, state_few)))
    same(a.x, b.x)
    same(a.branch, b.branch)
    del a, state
    a, b = px.gated(many[0], many[1], keep="e4m3"), px.gated(few[0], few[1], keep="e4m3")
    same(a[0], b[0])
    same(a[1].values, b[1].values)
    a, b = px.gated_grad(many[2], *a[1:]), px.gated_grad(few[2], *b[1:])
    same(a[0], b[0])
    same(a[1], b[1])


def test_a_gradient_over_kept_rows_past_32_bits():
    """Whole numbers, so that every sum is exact in whatever order."""
    import paper_2008_12260_amd as px
    N, D, last = 600000, 8192, 100
    assert (N - last) * D > 1 << 32
    g = torch.Generator("cuda").manual_seed(2)
    values = torch.zeros((N, D), dtype=torch.uint8, device="cuda")
    values[-last:] = torch.randint(0, 8, (last, D), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.full((N, D // 32), 127, dtype=torch.uint8, device="cuda")
    d = torch.randint(-3, 4, (N, 64), generator=g, device="cuda").bfloat16()
    want = d[-last:].double().t() @ values[-last:].double()
    assert torch.equal(px.kept_grad(px.Kept(values, scales, D, "i8"), d).double(), want.bfloat16().double())


def test_many_rows_of_few_elements():
    """More rows than the chip has under way at once, in every call: as in parts."""
    import paper_2008_12260_amd as px
    g = torch.Generator("cuda").manual_seed(3)
    for N, D in ((400003, 8), (200001, 40)):
        x, z, d, dh = (torch.randn((N, D), generator=g, device="cuda").bfloat16() for _ in range(4))
        w = torch.randn(D, generator=g, device="cuda")
        edge = dict(after=px.Norm(w), before=px.Norm(w, w), gate=w)
        y, rows, state = px.block_edge(x, z, **edge, keep="i8")
        grads = px.block_edge_grad(d, dh, state, **edge)
        a = px.gated(x, z, keep="i8")
        for at in range(0, N, 70001):
            to = min(N, at + 70001)
            y2, rows2, state2 = px.block_edge(x[at:to], z[at:to], **edge, keep="i8")
            assert torch.equal(y[at:to], y2) and torch.equal(rows[at:to], rows2) and torch.equal(state.y_kept.values[at:to], state2.y_kept.values)
            grads2 = px.block_edge_grad(d[at:to], dh[at:to], state2, **edge)
            assert torch.equal(grads.x[at:to], grads2.x) and torch.equal(grads.branch[at:to], grads2.branch)
            b = px.gated(x[at:to], z[at:to], keep="i8")
            assert torch.equal(a[0][at:to], b[0]) and torch.equal(a[1].values[at:to], b[1].values) and torch.equal(a[2].scales[at:to], b[2].scales)
        # sums over all rows: each chain is at most N / 1024 + 100 long
        n = px.restore(state.y_kept, torch.float32).double()
        for got, terms in ((grads.before_weight, dh.double() * n), (grads.before_bias, dh.double())):
            assert bool(((got.double() - terms.sum(0)).abs() <= (N / 1024 + 102) * 2.0 ** -24 * terms.abs().sum(0) + 2.0 ** -24 * terms.sum(0).abs()).all())


def test_two_streams_at_once():
    """The same inputs in calls that overlap, each with scratch memory of its own."""
    import paper_2008_12260_amd as px
    g = torch.Generator("cuda").manual_seed(4)
    x, z, d, dh = (torch.randn((4000, 1000), generator=g, device="cuda").bfloat16() for _ in range(4))
    w = torch.randn(1000, generator=g, device="cuda")
    edge = dict(after=px.Norm(w, w), before=px.Norm(w, w), gate=torch.randn((8, 1000), generator=g, device="cuda"), centred=True)

    def all_of(stream=None):
        y, rows, state = px.block_edge(x, z, **edge, keep="e4m3", stream=stream)
        return [y, rows, *px.block_edge_grad(d, dh, state, **edge, stream=stream), px.kept_grad(state.y_kept, dh, w, w, stream=stream)]
    want = all_of()
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream() for _ in range(2)]
    got = [[all_of(s) for s in sides] for _ in range(5)]
    torch.cuda.synchronize()
    for pair in got:
        for one in pair:
            assert all(torch.equal(a, b) for a, b in zip(one, want))


@pytest.mark.parametrize("kept", [None, "i8", "e4m3"])
def test_a_micro_batch_holds_no_more_than_it_remembers(kept):
    """Allocated when the loss is taken: of each edge what its gradient needs, of each block its activation's inputs, and beside them the tokens and the rows that the loss takes.
    (Bytes asked for: of what is allocated, the allocator's larger blocks may be up to 1 MiB each more.)"""
    from paper_2008_12260_amd.agent import Job
    import paper_2008_12260_amd as px
    asked = lambda: torch.cuda.memory_stats()["requested_bytes.all.current"]
    for blocks, D, F in ((1, 256, 512), (2, 256, 512), (3, 136, 1000)):
        job = Job(V=300, D=D, length=64, seed=6, blocks=blocks, width=F, kept=kept)
        model, gradient, tokens = job.parts(job.parameters.bfloat16()), torch.empty(job.parameters.numel(), dtype=torch.bfloat16, device="cuda"), job.examples(16)
        seen, loss = [], px.agent.token_loss

        def watched(rows, *args, **more):
            torch.cuda.synchronize()
            seen.append(asked())
            return loss(rows, *args, **more)
        px.agent.token_loss = watched
        try:
            job.micro_batch(tokens, model, gradient)
            torch.cuda.synchronize()
            base = asked()
            job.micro_batch(tokens, model, gradient)
        finally:
            px.agent.token_loss = loss
        row = (lambda width: 2 * width) if kept is None else (lambda width: 33 * -(-width // 32))
        # norms' sums; norms before and after; the activations' inputs; without a form the rows of all products but the last too
        each = 8 * (2 * blocks + 1) + (2 * blocks + 1) * row(D) + 2 * blocks * row(F) + (blocks * row(D) if kept is None else 0)
        held, rows = seen[-1] - base, 16 * 64
        around = rows * (2 * 8 + 2 * D) + 64 * 1024
        assert rows * each <= held <= rows * each + around, (blocks, D, F)


@pytest.mark.parametrize("kept", [None, "i8", "e4m3"])
def test_bytes_of_an_example_count_every_edge(kept):
    """Another example's share of what is asked for until the loss is taken, less its tokens and the rows that the loss takes: to a byte."""
    from paper_2008_12260_amd.agent import Job
    import paper_2008_12260_amd as px
    asked = lambda: torch.cuda.memory_stats()["requested_bytes.all.current"]
    for blocks, D, F in ((1, 256, 512), (2, 64, 40), (3, 136, 1000)):
        job = Job(V=300, D=D, length=64, seed=6, blocks=blocks, width=F, kept=kept)
        model, gradient = job.parts(job.parameters.bfloat16()), torch.empty(job.parameters.numel(), dtype=torch.bfloat16, device="cuda")
        seen, loss = [], px.agent.token_loss

        def watched(rows, *args, **more):
            torch.cuda.synchronize()
            seen.append(asked())
            return loss(rows, *args, **more)
        px.agent.token_loss = watched
        try:
            job.micro_batch(job.examples(3), model, gradient)
            for m in (16, 17):
                tokens = job.examples(m)
                torch.cuda.synchronize()
                base = asked()
                job.micro_batch(tokens, model, gradient)
                seen[-1] -= base
        finally:
            px.agent.token_loss = loss
        assert seen[-1] - seen[-2] == job.bytes_per_example() + 64 * (2 * 8 + 2 * D), (blocks, D, F)
    assert Job(V=300, D=64, length=64).bytes_per_example() == 0


@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
def test_the_widest_rows(dtype):
    """Rows at the limits of their widths: as their parts, which are whole groups of 32.  The product is against 64 bits: three products of at most 2^-24 of themselves off and three additions, below
    2^-21 of the sum of their sizes, and a rounding."""
    import paper_2008_12260_amd as px
    g = torch.Generator("cuda").manual_seed(7)
    W, H = 1 << 20, 1 << 19
    both, d = (torch.randn((3, W), generator=g, device="cuda").to(dtype) for _ in range(2))
    parts = [slice(at, at + W // 4) for at in range(0, W, W // 4)]
    for form in ("i8", "e4m3"):
        kept = px.keep(both, form)
        back = px.restore(kept, dtype)
        for part in parts:
            few = px.keep(both[:, part], form)
            assert torch.equal(kept.values[:, part], few.values) and torch.equal(back[:, part], px.restore(few, dtype))
        few = px.keep(both[:, :40], form)
        got = px.kept_grad(few, d)
        assert got.shape == (W, 40)
        x = px.restore(few, torch.float32).double()
        want, size = d.double().t().contiguous() @ x, d.double().abs().t().contiguous() @ x.abs()
        half = torch.finfo(dtype).eps / 2
        assert bool(((got.double() - want).abs() <= half * want.abs() + 2.0 ** -21 * size).all())
        rows, *kept = px.gated(both[:, :H], both[:, H:], keep=form)
        for inputs in (kept, (both[:, :H], both[:, H:])):
            dg, du, again = px.gated_grad(d[:, :H], *inputs, want_rows=True)
            assert dg.stride() == (W, 1)
            for part in parts[:2]:
                up = slice(H + part.start, H + part.stop)
                few = px.gated(both[:, part], both[:, up], keep=form)
                assert torch.equal(rows[:, part], few[0])
                want = px.gated_grad(d[:, part], *(few[1:] if inputs is kept else (both[:, part], both[:, up])), want_rows=True)
                assert all(torch.equal(a[:, part], b) for a, b in zip((dg, du, again), want))
