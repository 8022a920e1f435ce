"""The edge between two blocks and its gradients against 64 bits.

A row's sum is formed by chains of at most 16 elements, 6 moves between lanes and 16 wavefronts, 38 additions of 2^-24 each: within 2^-18.7 of the sum of its terms' sizes.  Some
twelve roundings more an element are 2^-20.4.  Together below 2^-18 of the sizes of what is added up, twice that where a second norm takes the first one's errors: E.  `Sized` carries each value's size, the sum of
the sizes of the terms it is made of, through the same formulas.  Sums over rows are chains of at most 200 additions at these sizes, 2^-16.3 more.  Results are rounded once."""
import pytest

torch = pytest.importorskip("torch")

from kept import FORMS, SMALLEST, U, decoded  # noqa: E402

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
E, E_SUMS = 2.0 ** -17, 2.0 ** -15


def near(got, want, size, e=E, where=""):
    tolerance = U[got.dtype] * want.abs() + e * size + SMALLEST[got.dtype]
    off = (got.double() - want).abs()
    assert bool((off <= tolerance).all()), (where, float((off / tolerance).max()))


class Case:
    """Inputs of an edge, and its parts in 64 bits."""

    def __init__(self, N, D, x_type=BF16, dtype=BF16, weights=F32, centred=False, after=True, before=True, gates=1, biased=False, residual=1.0, scale=1.0, seed=0, branch=True):
        import paper_2008_12260_amd as px
        g = torch.Generator("cuda").manual_seed(seed + N + D)
        normal = lambda *shape, dtype=dtype: torch.randn(shape, generator=g, device="cuda").to(dtype)
        self.N, self.D, self.centred, self.residual, self.scale, self.gates = N, D, centred, residual, scale, gates
        self.x, self.branch = normal(N, D, dtype=x_type) + (0.5 if centred else 0.0), normal(N, D) * 2.0 if branch else None
        norm = lambda: px.Norm(1.0 + 0.3 * normal(D, dtype=weights), normal(D, dtype=weights) if biased else None)
        self.after, self.before = norm() if after and branch else None, norm() if before else None
        self.gate = None if gates == 0 or not branch else normal(D, dtype=weights) if gates == 1 else normal(gates, D, dtype=weights)
        self.y_grad, self.rows_grad = normal(N, D, dtype=x_type), normal(N, D) if before else None
        self.edge = dict(gate=self.gate, after=self.after, before=self.before, residual=residual, scale=scale, centred=centred)

    def norm(self, v, size, eps=1e-6):
        """(n, its size, (mean, r)) of rows and their sizes."""
        mean = v.mean(1, keepdim=True) if self.centred else torch.zeros_like(v[:, :1])
        r = ((v - mean).square().mean(1, keepdim=True) + eps).rsqrt()
        n = (v - mean) * r
        whole = size.mean(1, keepdim=True) if self.centred else 0.0
        return n, r * (size + whole) + n.abs() * (1.0 + r * size.square().mean(1, keepdim=True).sqrt() + r * whole), (mean, r)

    def weighted(self, n, size, norm):
        if norm is None:
            return n, size
        w = torch.ones((), dtype=torch.float64, device="cuda") if norm.weight is None else norm.weight.double()
        out, size = n * w, size * w.abs()
        return (out, size) if norm.bias is None else (out + norm.bias.double(), size + norm.bias.double().abs())

    def gate_rows(self):
        if self.gate is None:
            return torch.ones((), dtype=torch.float64, device="cuda")
        g = self.gate.double()
        return g if self.gates == 1 else g.repeat_interleave(self.N // self.gates, 0)

    def forward(self):
        x = self.x.double()
        if self.branch is None:
            self.n_z = self.stats_z = None
            y, size = x, x.abs()
        else:
            z = self.branch.double()
            n, n_size, self.stats_z = self.norm(z, z.abs()) if self.after is not None else (z, z.abs(), None)
            self.n_z, self.n_z_size = n, n_size
            b, b_size = self.weighted(n, n_size, self.after)
            gate = self.scale * self.gate_rows()
            y, size = self.residual * x + gate * b, (self.residual * x).abs() + gate.abs() * b_size
        self.y, self.y_size = y, size
        if self.before is not None:
            self.n_y, self.n_y_size, self.stats_y = self.norm(y, size)
            self.h, self.h_size = self.weighted(self.n_y, self.n_y_size, self.before)
        return self

    def through(self, d, size, n, r):
        along, along_size = (d * n).mean(1, keepdim=True), (size * n.abs()).mean(1, keepdim=True)
        out, size_out = d - n * along, size + n.abs() * along_size
        if self.centred:
            out, size_out = out - d.mean(1, keepdim=True), size_out + size.mean(1, keepdim=True)
        return r * out, r * size_out

    def backward(self, n_y, n_z, state, y_grad=True):
        """Names to (value, size) from given normalised rows."""
        zero = torch.zeros((self.N, self.D), dtype=torch.float64, device="cuda")
        g = self.y_grad.double() if y_grad else zero
        g_size = g.abs()
        out = {}
        if self.before is not None:
            dh = self.rows_grad.double()
            w = 1.0 if self.before.weight is None else self.before.weight.double()
            more, more_size = self.through(dh * w, (dh * w).abs(), n_y, state.y_stats[:, 1:].double())
            g, g_size = g + more, g_size + more_size
            out["before_weight"] = (dh * n_y).sum(0), (dh * n_y).abs().sum(0)
            out["before_bias"] = dh.sum(0), dh.abs().sum(0)
        out["x"] = self.residual * g, abs(self.residual) * g_size
        if self.branch is None:
            return out
        gate = self.scale * self.gate_rows()
        t, t_size = gate * g, gate.abs() * g_size
        if self.after is not None:
            w = 1.0 if self.after.weight is None else self.after.weight.double()
            out["branch"] = self.through(t * w, t_size * abs(w), n_z, state.branch_stats[:, 1:].double())
            out["after_weight"] = (t * n_z).sum(0), (t_size * n_z.abs()).sum(0)
            out["after_bias"] = t.sum(0), t_size.sum(0)
        else:
            out["branch"] = t, t_size
        if self.gate is not None:
            b, b_size = self.weighted(n_z, n_z.abs(), self.after)
            shared = lambda v: v.view(self.gates, -1, self.D).sum(1).view(self.gate.shape)
            out["gate"] = shared(self.scale * g * b), shared(abs(self.scale) * g_size * b_size)
        return out


def run(case, keep=None, y_grad=True):
    import paper_2008_12260_amd as px
    case.forward()
    y, rows, state = px.block_edge(case.x, case.branch, **case.edge, keep=keep)
    if case.branch is None:
        assert y is case.x
    else:
        near(y, case.y, case.y_size, where="y")
    if case.before is not None:
        near(rows, case.h, case.h_size, where="rows")
    for stats, want, v in ((state.branch_stats, getattr(case, "stats_z", None), case.branch), (state.y_stats, getattr(case, "stats_y", None), case.y)):
        assert (stats is None) == (want is None)
        if stats is not None:
            mean, r = (t[:, 0] for t in want)
            size = v.double().abs().mean(1) if v is case.branch else case.y_size.mean(1)
            assert bool(((stats[:, 0].double() - mean).abs() <= E * size).all())
            assert bool(((stats[:, 1].double() - r).abs() <= E * r * (1 + r * size + (r * r) * (case.y_size if v is case.y else v.double()).square().mean(1))).all())
    kept = []
    for k, n, size in ((state.y_kept, getattr(case, "n_y", None), getattr(case, "n_y_size", None)), (state.branch_kept, case.n_z, getattr(case, "n_z_size", None))):
        kept.append(None)
        if k is None:
            continue
        # within half a step of the normalised rows, whose errors may move an element to the next code and, at the border of two scales, to one of the larger
        at = decoded(*k).cuda()
        kept[-1] = at
        padded = torch.nn.functional.pad(n, (0, -case.D % 32)).unflatten(1, (-1, 32)).abs().amax(2)
        top = padded.repeat_interleave(32, 1)[:, :case.D]
        half = top / 127.0 if keep == "i8" else torch.maximum(n.abs() * 2.0 ** -4, top * 2.0 ** -17)
        assert bool(((at - n).abs() <= half * (1 + 2.0 ** -6) + E * size + 2.0 ** -126).all())
    if keep is None:
        if case.before is not None:
            kept[0] = (y.double() - state.y_stats[:, :1].double()) * state.y_stats[:, 1:].double()
        if case.branch is not None:
            z = case.branch.double()
            kept[1] = z if case.after is None else (z - state.branch_stats[:, :1].double()) * state.branch_stats[:, 1:].double()
    grads = px.block_edge_grad(case.y_grad if y_grad else None, case.rows_grad, state, y=None if keep else y, branch=None if keep else case.branch, **case.edge)
    want = case.backward(kept[0], kept[1], state, y_grad)
    for name, got in grads._asdict().items():
        has = name in want and not (name.endswith("weight") and getattr(case, name[:-7]).weight is None) and not (name.endswith("bias") and getattr(case, name[:-5]).bias is None)
        assert (got is not None) == has, name
        if got is not None:
            near(got, *want[name], E_SUMS if name not in ("x", "branch") else 2 * E, name)
    return y, rows, state, grads


SIZES = [(1, 1), (2, 7), (5, 32), (3, 33), (17, 64), (40, 100), (33, 256), (70, 512), (30, 520), (24, 1000), (16, 2048), (9, 4104), (7, 8192), (5, 8200), (4, 16384)]
TYPES = [(F32, F32), (BF16, BF16), (F16, F16), (F32, BF16), (F32, F16)]


@pytest.mark.parametrize("x_type,dtype", TYPES)
@pytest.mark.parametrize("N,D", SIZES)
def test_edges(N, D, x_type, dtype):
    for keep in (None, "i8"):
        run(Case(N, D, x_type, dtype, residual=0.75, scale=-0.5), keep)
        run(Case(N, D, x_type, dtype, centred=True, biased=True, seed=1), keep)


@pytest.mark.parametrize("centred", [False, True])
@pytest.mark.parametrize("N,D", [(1, 40), (12, 64), (60, 96), (60, 520), (24, 1000), (6, 9000)])
def test_gates_of_spans(N, D, centred):
    """One a row, one for some rows, whose ends fall within and between workgroups' rows, one for all, none."""
    for gates in [0] + [g for g in (1, 2, 3, 4, 6, 12, 30, 60) if N % g == 0]:
        for keep in (None, "e4m3"):
            run(Case(N, D, centred=centred, biased=centred, gates=gates, seed=2), keep)
        run(Case(N, D, gates=gates, after=False, centred=centred, seed=3))


def test_many_rows_to_a_gate():
    for N, D, gates in ((3003, 200, 3), (3000, 64, 50), (5000, 1000, 7 - 2), (1030, 600, 2), (4099, 32, 1), (2600, 520, 1300)):
        run(Case(N, D, F32, BF16, gates=gates, biased=True, centred=True))
        run(Case(N, D, BF16, BF16, gates=gates, before=False), "i8")


@pytest.mark.parametrize("form", (None,) + FORMS)
@pytest.mark.parametrize("dtype", (F32, BF16, F16))
def test_parts(dtype, form):
    """Each part without the others."""
    N, D = 20, 200
    run(Case(N, D, dtype, dtype, branch=False), form)
    run(Case(N, D, dtype, dtype, branch=False, centred=True, biased=True), form)
    run(Case(N, D, dtype, dtype, branch=False), form, y_grad=False)
    run(Case(N, D, dtype, dtype, before=False), form)
    run(Case(N, D, dtype, dtype, after=False), form)
    run(Case(N, D, dtype, dtype, after=False, gates=0), form)
    run(Case(N, D, dtype, dtype, after=False, before=False, gates=0), form)
    run(Case(N, D, dtype, dtype, after=False, before=False, gates=20), form)
    run(Case(N, D, dtype, dtype, gates=0, weights=dtype), form, y_grad=False)
    import paper_2008_12260_amd as px
    case = Case(N, D, dtype, dtype, gates=0)
    case.after = case.edge["after"] = px.Norm()
    case.before = case.edge["before"] = px.Norm(None, case.before.weight)
    run(case, form)


def test_strides_shapes_and_what_is_needed():
    import paper_2008_12260_amd as px
    case = Case(24, 72, gates=4)
    y, rows, state = px.block_edge(case.x, case.branch, **case.edge)
    wide = torch.zeros((24, 101), dtype=BF16, device="cuda")
    wide[:, 3:75] = case.branch
    again = px.block_edge(case.x.t().contiguous().t(), wide[:, 3:75], **case.edge)
    assert torch.equal(again[0], y) and torch.equal(again[1], rows)
    edge = {**case.edge, "gate": case.gate.view(4, 1, 72)}
    shaped = px.block_edge(case.x.view(4, 6, 72), case.branch.view(4, 6, 72), **edge)
    assert shaped[0].shape == (4, 6, 72) and torch.equal(shaped[1].view(24, 72), rows)
    want = px.block_edge_grad(case.y_grad, case.rows_grad, state, y=y, branch=case.branch, **case.edge)
    got = px.block_edge_grad(case.y_grad.view(4, 6, 72), case.rows_grad.view(4, 6, 72), shaped[2], y=shaped[0], branch=case.branch.view(4, 6, 72), **edge)
    assert got.gate.shape == (4, 1, 72) and got.x.shape == (4, 6, 72)
    for a, b in zip(got, want):
        assert (a is None) == (b is None) and (a is None or torch.equal(a.reshape(b.shape), b))
    for need in (("x",), ("branch", "gate"), ("after",), ("before", "x"), ("gate",)):
        some = px.block_edge_grad(case.y_grad, case.rows_grad, state, y=y, branch=case.branch, **case.edge, need=need)
        for name, t in some._asdict().items():
            part = name.split("_")[0]
            assert (t is not None) == (part in need and getattr(want, name) is not None)
            assert t is None or torch.equal(t, getattr(want, name))


def test_a_norm_alone_in_another_type():
    """The first edge of a stack whose residual stream is in fp32: no branch, rows in 16 bits."""
    import paper_2008_12260_amd as px
    for dtype in (BF16, F16):
        for form in (None, "i8"):
            case = Case(21, 136, F32, dtype, branch=False).forward()
            y, rows, state = px.block_edge(case.x, before=case.before, rows_dtype=dtype, keep=form)
            assert y is case.x and rows.dtype == dtype and state.x_dtype == F32 and state.dtype == dtype
            near(rows, case.h, case.h_size)
            grads = px.block_edge_grad(case.y_grad, case.rows_grad, state, y=None if form else y, before=case.before)
            n = decoded(*state.y_kept).cuda() if form else (y.double() - state.y_stats[:, :1].double()) * state.y_stats[:, 1:].double()
            want = case.backward(n, None, state)
            assert grads.x.dtype == F32 and grads.branch is None
            near(grads.x, *want["x"], 2 * E)
            near(grads.before_weight, *want["before_weight"], E_SUMS)


@pytest.mark.parametrize("form", (None,) + FORMS)
def test_a_norm_alone_under_a_residual_scale(form):
    """Without a branch y is x whatever the stack's residual is: the gradients are those of the forward call, differentiated."""
    import paper_2008_12260_amd as px
    for N, D, centred in ((12, 40, False), (9, 1000, True), (3, 9000, False)):
        case = Case(N, D, F32, F32, branch=False, centred=centred, biased=True)
        want = px.block_edge(case.x, before=case.before, centred=centred, keep=form)
        want_grads = px.block_edge_grad(case.y_grad, case.rows_grad, want[2], y=None if form else want[0], before=case.before, centred=centred)
        y, rows, state = px.block_edge(case.x, before=case.before, residual=0.75, centred=centred, keep=form)
        assert y is case.x and torch.equal(rows, want[1])
        grads = px.block_edge_grad(case.y_grad, case.rows_grad, state, y=None if form else y, before=case.before, residual=0.75, centred=centred)
        for a, b in zip(grads, want_grads):
            assert (a is None) == (b is None) and (a is None or torch.equal(a, b))
        if form is None:
            x = case.x.double().requires_grad_()
            v = x - x.mean(1, keepdim=True) if centred else x
            n = v * (v.square().mean(1, keepdim=True) + 1e-6).rsqrt()
            (x * case.y_grad + (n * case.before.weight + case.before.bias) * case.rows_grad).sum().backward()
            case.forward()
            near(grads.x, x.grad, case.backward(case.n_y, None, state)["x"][1], 2 * E)


def test_in_place_through_the_library():
    """y over x, and the gradient of x over that of y, by the C ABI."""
    import ctypes
    import paper_2008_12260_amd as px
    for N, D in ((33, 100), (9, 1000)):
        case = Case(N, D)
        y, rows, state = px.block_edge(case.x, case.branch, **case.edge)
        grads = px.block_edge_grad(case.y_grad, case.rows_grad, state, y=y, branch=case.branch, **case.edge)
        dims = px.EdgeDims(N, D, px.PX_TYPE_BF16, px.PX_TYPE_BF16, px.PX_TYPE_F32, px.PX_TYPE_F32, 0, px.PX_EDGE_AFTER | px.PX_EDGE_BEFORE, 1e-6, 1.0, 1.0, 0)
        p, L = (lambda t: t.data_ptr()), px.lib()
        x, h = case.x.clone(), torch.empty_like(rows)
        torch.cuda.synchronize()
        rc = L.pollux_block_edge(ctypes.byref(dims), p(x), p(case.branch), p(case.gate), p(case.after.weight), None, p(case.before.weight), None, p(x), p(h), None, None, None, None, None,
                                 None, None)
        assert rc == px.PX_OK
        need = ctypes.c_size_t()
        assert L.pollux_block_edge_workspace_size(ctypes.byref(dims), ctypes.byref(need)) == px.PX_OK
        ws, d, dz = torch.empty(need.value, dtype=torch.uint8, device="cuda"), case.y_grad.clone(), torch.empty_like(rows)
        torch.cuda.synchronize()
        rc = L.pollux_block_edge_grad(ctypes.byref(dims), p(d), p(case.rows_grad), p(y), None, p(case.branch), None, p(state.y_stats), p(state.branch_stats), p(case.gate), p(case.after.weight), None,
                                      p(case.before.weight), p(ws), need.value, p(d), p(dz), None, None, None, None, None, None)
        assert rc == px.PX_OK
        torch.cuda.synchronize()
        assert torch.equal(x, y) and torch.equal(h, rows) and torch.equal(d, grads.x) and torch.equal(dz, grads.branch)


def test_a_last_span_that_is_cut_short():
    """By the C ABI: a gate of ceil(N / span) rows, the last of which serves fewer; as a gate a row, whose gradients are then summed."""
    import ctypes
    import paper_2008_12260_amd as px
    L, p = px.lib(), (lambda t: None if t is None else t.data_ptr())
    for N, D, span in ((10, 72, 4), (101, 1000, 33), (50, 600, 49), (9, 40, 2)):
        case = Case(N, D, F32, F32, gates=N)
        gate = torch.randn((-(-N // span), D), device="cuda")
        case.gate = case.edge["gate"] = gate.repeat_interleave(span, 0)[:N].contiguous()
        y, rows, state = px.block_edge(case.x, case.branch, **case.edge)
        want = px.block_edge_grad(case.y_grad, case.rows_grad, state, y=y, branch=case.branch, **case.edge)
        dims = px.EdgeDims(N, D, 0, 0, 0, 0, 0, px.PX_EDGE_AFTER | px.PX_EDGE_BEFORE, 1e-6, 1.0, 1.0, span)
        y2, rows2, gate_grad, dx, dz = torch.empty_like(y), torch.empty_like(rows), torch.full_like(gate, 7.0), torch.empty_like(y), torch.empty_like(y)
        need = ctypes.c_size_t()
        assert L.pollux_block_edge_workspace_size(ctypes.byref(dims), ctypes.byref(need)) == px.PX_OK
        ws = torch.empty(need.value, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        assert L.pollux_block_edge(ctypes.byref(dims), p(case.x), p(case.branch), p(gate), p(case.after.weight), None, p(case.before.weight), None, p(y2), p(rows2), None, None, None, None, None, None,
                                   None) == px.PX_OK
        assert L.pollux_block_edge_grad(ctypes.byref(dims), p(case.y_grad), p(case.rows_grad), p(y), None, p(case.branch), None, p(state.y_stats), p(state.branch_stats), p(gate), p(case.after.weight), None,
                                        p(case.before.weight), p(ws), need.value, p(dx), p(dz), p(gate_grad), None, None, None, None, None) == px.PX_OK
        torch.cuda.synchronize()
        assert torch.equal(y2, y) and torch.equal(rows2, rows) and torch.equal(dx, want.x) and torch.equal(dz, want.branch)
        for s in range(gate.shape[0]):
            terms = want.gate[s * span:(s + 1) * span].double()
            # (each row's rounded once more there; sums of at most 49)
            assert bool(((gate_grad[s].double() - terms.sum(0)).abs() <= 64 * 2.0 ** -24 * terms.abs().sum(0) + 2.0 ** -140).all())


def test_rows_of_zeros_and_rows_that_are_not_finite():
    import paper_2008_12260_amd as px
    case = Case(40, 300, gates=0)
    case.x[5] = 0
    case.branch[5] = 0
    run(case)
    run(case, "e4m3")
    y, rows, state = px.block_edge(case.x, case.branch, **case.edge, keep="i8")
    bad = case.x.clone()
    bad[7, 3], bad[8, 299] = float("nan"), float("inf")
    y2, rows2, state2 = px.block_edge(bad, case.branch, **case.edge, keep="i8")
    others = [r for r in range(40) if r not in (7, 8)]
    assert torch.equal(rows[others], rows2[others]) and torch.equal(y[others], y2[others])
    assert bool(torch.isnan(rows2[7]).all()) and not bool(torch.isfinite(rows2[8]).all()) and bool(torch.isfinite(y2[7, 4:]).all())
    g, g2 = (px.block_edge_grad(case.y_grad, case.rows_grad, s, **case.edge) for s in (state, state2))
    assert torch.equal(g.x[others], g2.x[others]) and torch.equal(g.branch[others], g2.branch[others]) and bool(torch.isnan(g2.x[7]).all())


def test_rows_far_from_zero_keep_their_spread():
    """Centred norms of rows at 1000 with a spread of 1: in fp32 the mean is off by at most 2^-18.7 of 1000 and the rows' own steps are 2^-14."""
    import paper_2008_12260_amd as px
    x = torch.randn((20, 700), device="cuda") + 1000.0
    rows = px.block_edge(x, before=px.Norm(), centred=True)[1].double()
    v = x.double() - x.double().mean(1, keepdim=True)
    want = v * (v.square().mean(1, keepdim=True) + 1e-6).rsqrt()
    assert float((rows - want).abs().max()) < 1000 * 2.0 ** -18 + 2.0 ** -17 * 5


def test_no_rows():
    import paper_2008_12260_amd as px
    case = Case(0, 50, gates=1, biased=True)
    y, rows, state = px.block_edge(case.x, case.branch, **case.edge, keep="i8")
    assert y.shape == rows.shape == (0, 50)
    grads = px.block_edge_grad(case.y_grad, case.rows_grad, state, **case.edge)
    assert grads.x.shape == (0, 50)
    for t in grads[2:]:
        assert not bool(t.any())


@pytest.mark.parametrize("gates", [(0, 50), (3, 50), (2, 3, 50), (1, 50)])
def test_no_rows_of_gates(gates):
    import paper_2008_12260_amd as px
    case = Case(0, 50, gates=1)
    case.edge["gate"] = torch.ones(gates, device="cuda")
    y, rows, state = px.block_edge(case.x, case.branch, **case.edge, keep="i8")
    assert y.shape == rows.shape == (0, 50)
    used = torch.full((512,), float("nan"), device="cuda")      # (what the gradient is allocated from next, perhaps)
    del used
    grads = px.block_edge_grad(case.y_grad, case.rows_grad, state, **case.edge)
    assert grads.gate.shape == gates and not bool(grads.gate.any()) and not bool(grads.after_weight.any())


def test_no_rows_have_no_spans():
    """By the C ABI a gate of no rows' spans has no rows: nothing is written to its gradient."""
    import ctypes
    import paper_2008_12260_amd as px
    L = px.lib()
    gate, weight, gate_grad, weight_grad = torch.ones(64, device="cuda"), torch.ones(64, device="cuda"), torch.full((64,), 7.0, device="cuda"), torch.full((64,), 7.0, device="cuda")
    ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    for span, left in ((3, 7.0), (0, 0.0)):
        dims = px.EdgeDims(0, 64, 0, 0, 0, 0, 0, px.PX_EDGE_AFTER, 1e-6, 1.0, 1.0, span)
        need = ctypes.c_size_t()
        assert L.pollux_block_edge_workspace_size(ctypes.byref(dims), ctypes.byref(need)) == px.PX_OK and need.value <= 256
        gate_grad.fill_(7.0)
        torch.cuda.synchronize()
        assert L.pollux_block_edge_grad(ctypes.byref(dims), None, None, None, None, None, None, None, None, gate.data_ptr(), weight.data_ptr(), None, None, ws.data_ptr(), 256, None, None,
                                        gate_grad.data_ptr(), weight_grad.data_ptr(), None, None, None, None) == px.PX_OK
        torch.cuda.synchronize()
        assert bool((gate_grad == left).all()) and not bool(weight_grad.any())


def test_gradients_are_differences():
    """fp32, along random directions, steps h = 2^-6: a difference is within h^2 times a third derivative (some units here, of sums of 24 x 40 terms of size 1: below 2^-12 * 2^7) and 2^-24 * 2^10 / h of
    the derivative."""
    import paper_2008_12260_amd as px
    case = Case(24, 40, F32, F32, centred=True, biased=True, gates=3, residual=0.5, scale=1.5)
    g = torch.Generator("cuda").manual_seed(7)
    y, rows, state = px.block_edge(case.x, case.branch, **case.edge)
    grads = px.block_edge_grad(case.y_grad, case.rows_grad, state, y=y, branch=case.branch, **case.edge)
    leaves = dict(x=case.x, branch=case.branch, gate=case.gate, after_weight=case.after.weight, after_bias=case.after.bias, before_weight=case.before.weight, before_bias=case.before.bias)

    def value(changed):
        v = {**leaves, **changed}
        y, rows, _ = px.block_edge(v["x"], v["branch"], **{**case.edge, "gate": v["gate"], "after": px.Norm(v["after_weight"], v["after_bias"]),
                                                          "before": px.Norm(v["before_weight"], v["before_bias"])})
        return float((y.double() * case.y_grad.double()).sum() + (rows.double() * case.rows_grad.double()).sum())
    h = 2.0 ** -6
    for name, leaf in leaves.items():
        way = torch.randn(leaf.shape, generator=g, device="cuda")
        got = float((getattr(grads, name).double() * way.double()).sum())
        want = (value({name: leaf + h * way}) - value({name: leaf - h * way})) / (2 * h)
        assert abs(got - want) <= 2.0 ** -4 + 2.0 ** -5 * abs(want), (name, got, want)


def test_streams_graphs_and_the_same_bits():
    import paper_2008_12260_amd as px
    case = Case(1000, 600, gates=5, biased=True)
    wants = []
    sets = [(case.x * k, case.branch + k, case.y_grad * k, case.rows_grad) for k in (1, 2, 3)]

    def both(x, branch, d, dh, stream=None):
        y, rows, state = px.block_edge(x, branch, **case.edge, keep="i8", stream=stream)
        return y, rows, px.block_edge_grad(d, dh, state, **case.edge, stream=stream)
    for s in sets:
        wants.append(both(*s))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = both(*sets[0], stream=side)
    side.synchronize()
    assert torch.equal(got[1], wants[0][1]) and all(torch.equal(a, b) for a, b in zip(got[2], wants[0][2]))
    live = [t.clone() for t in sets[0]]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both(*live)
    for k in (1, 2, 0):
        for t, new in zip(live, sets[k]):
            t.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], wants[k][0]) and torch.equal(out[1], wants[k][1]) and all(torch.equal(a, b) for a, b in zip(out[2], wants[k][2]))
