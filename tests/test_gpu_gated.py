"""Gated activations and their gradients against 64 bits.

With p the factor from 0 to 1, an activation is g p and its slope p + g p'.  silu: exp of an exact argument (2 steps of 2^-23 at most), a sum, a quotient and two products: p and
p (1 - p) are within 2^-20 of themselves.  The others' exponents are rounded before they are raised: erfc(x) and exp(-x^2) move by up to 2 x^2 2^-24 of themselves, x < 10.1 where
they are not 0, tanh's by 3 roundings of an exponent below 104: 2^-15.  A product or sum more adds 2^-23 each; results are rounded once.  Where p or p' is below 2^-126, the smallest normal number, the
hardware's functions give 0: off by 2^-126 of what they are multiplied with (p' of the last is p (1 - p) times up to 1.6 (1 + 0.135 g^2))."""
import pytest

torch = pytest.importorskip("torch")

from kept import FORMS, SMALLEST, U, decoded  # noqa: E402

pytestmark = pytest.mark.gpu

TYPES = (torch.float32, torch.bfloat16, torch.float16)
ACTS = ("silu", "gelu", "gelu_tanh")
E = {"silu": 2.0 ** -19, "gelu": 2.0 ** -14.5, "gelu_tanh": 2.0 ** -14.5}


def inputs(N, F, dtype, seed, count=3):
    g = torch.Generator("cuda").manual_seed(seed)
    return [(3.0 * torch.randn((N, F), generator=g, device="cuda")).to(dtype) for _ in range(count)]


def parts(g, act):
    """(p, p') in 64 bits."""
    if act == "silu":
        return torch.sigmoid(g), torch.sigmoid(g) * torch.sigmoid(-g)
    if act == "gelu":
        return 0.5 * torch.erfc(-g * 0.5 ** 0.5), torch.exp(-0.5 * g * g) / (2 * torch.pi) ** 0.5
    k = (8 / torch.pi) ** 0.5
    t = k * (g + 0.044715 * g ** 3)
    return torch.sigmoid(t), torch.sigmoid(t) * torch.sigmoid(-t) * k * (1 + 3 * 0.044715 * g * g)


def near(got, want, size, act, factors):
    """size: the sum of the sizes of what `want` is a sum of; factors: of what p and p' are multiplied with in it."""
    dtype = got.dtype
    tolerance = U[dtype] * want.abs() + E[act] * size + SMALLEST[dtype] + 2.0 ** -120 + 2.0 ** -126 * factors
    assert bool(((got.double() - want).abs() <= tolerance).all()), float(((got.double() - want).abs() / tolerance).max())


def check(gate, up, d, act, grads, rows):
    """gate, up in 64 bits."""
    p, slope = parts(gate, act)
    u = torch.ones_like(gate) if up is None else up
    if rows is not None:
        near(rows, gate * p * u, (gate * p * u).abs(), act, (gate * u).abs())
    if grads is not None:
        inner = 1.6 * (1 + 0.135 * gate * gate) if act == "gelu_tanh" else 1.0
        near(grads[0], d * u * (p + gate * slope), (d * u).abs() * (p + (gate * slope).abs()), act, (d * u).abs() * (1 + gate.abs() * inner))
        if up is not None:
            near(grads[1], d * gate * p, (d * gate * p).abs(), act, (d * gate).abs())


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,F", [(1, 1), (3, 7), (2, 64), (5, 129), (70, 1000), (33, 4096)])
def test_rows_and_gradients(N, F, dtype, act):
    import paper_2008_12260_amd as px
    gate, up, d = inputs(N, F, dtype, N + F)
    for u in (up, None):
        rows, gate_kept, up_kept = px.gated(gate, u, act)
        assert gate_kept is None and up_kept is None
        grads = px.gated_grad(d, gate, u, act, want_rows=True)
        wide = None if u is None else u.double()
        check(gate.double(), wide, d.double(), act, grads, rows)
        assert torch.equal(grads[2], rows)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,F", [(1, 1), (4, 33), (9, 1000), (40, 2048)])
def test_gradients_from_what_is_kept(N, F, dtype, form):
    import paper_2008_12260_amd as px
    gate, up, d = inputs(N, F, dtype, 100 + N + F)
    for act in ACTS:
        for u in (up, None):
            rows, *kept = px.gated(gate, u, act, keep=form)
            assert torch.equal(rows, px.gated(gate, u, act)[0])
            for k, x in zip(kept, (gate, u)):
                if x is not None:
                    same = px.keep(x, form)
                    assert torch.equal(k.values, same.values) and torch.equal(k.scales, same.scales) and k[2:] == same[2:]
            wide = [None if k is None else decoded(*k).cuda() for k in kept]
            grads = px.gated_grad(d, *kept, act, want_rows=True)
            check(wide[0], wide[1], d.double(), act, grads, grads[2])


def test_halves_of_one_product_and_results_in_place():
    import paper_2008_12260_amd as px
    for F in (64, 77):
        both, d = torch.cat(inputs(30, F, torch.bfloat16, 1)[:2], 1), inputs(30, F, torch.bfloat16, 2)[0]
        rows, _, _ = px.gated(both[:, :F], both[:, F:])
        assert torch.equal(rows, px.gated(both[:, :F].clone(), both[:, F:].clone())[0])
        out = torch.full((30, 2 * F + 9), 5.0, dtype=torch.bfloat16, device="cuda")
        gate_grad, up_grad, none = px.gated_grad(d, both[:, :F], both[:, F:], out=out[:, 4:4 + 2 * F])
        assert none is None and gate_grad.data_ptr() == out[:, 4:].data_ptr()
        want = px.gated_grad(d, both[:, :F], both[:, F:])
        assert torch.equal(gate_grad, want[0]) and torch.equal(up_grad, want[1])
        assert bool((out[:, :4] == 5).all()) and bool((out[:, 4 + 2 * F:] == 5).all())
    cube = inputs(24, 50, torch.float32, 3)
    rows = px.gated(cube[0].view(4, 6, 50), cube[1].view(4, 6, 50))[0]
    assert rows.shape == (4, 6, 50) and torch.equal(rows.view(24, 50), px.gated(*cube[:2])[0])
    back = px.gated_grad(cube[2].view(4, 6, 50), cube[0].view(4, 6, 50), cube[1].view(4, 6, 50))
    assert back[0].shape == (4, 6, 50) and torch.equal(back[1].reshape(24, 50), px.gated_grad(cube[2], *cube[:2])[1])
    strided = px.gated(cube[0].t().contiguous().t(), cube[1])[0]
    assert torch.equal(strided, px.gated(*cube[:2])[0])


@pytest.mark.parametrize("act", ACTS)
def test_far_from_zero_and_not_finite(act):
    import paper_2008_12260_amd as px
    inf, nan = float("inf"), float("nan")
    g = torch.tensor([[-inf, -3e38, -1e20, -200.0, -0.0, 0.0, 200.0, 1e20, 3e38, inf, nan]], device="cuda")
    one = torch.ones_like(g)
    rows = px.gated(g, one, act)[0][0].tolist()
    slopes, values, _ = (None if t is None else t[0].tolist() for t in px.gated_grad(one, g, one, act))
    for k, x in enumerate(g[0].tolist()):
        if x != x:
            assert rows[k] != rows[k] and slopes[k] != slopes[k]
        else:
            assert rows[k] == values[k] == (x if x > 0 else 0.0) and slopes[k] == (1.0 if x > 0 else 0.5 if x == 0 else 0.0), (x, rows[k], slopes[k])


def test_gradients_are_the_differences_of_the_rows():
    """fp32, steps of 2^-9: the central difference is within h^2/6 times the third derivative (below 2) of the slope, 2^-19.6, and its rounding, 2 * 2^-24 * 9 * 2^8 + the rows' own 2^-14.5
    relative errors, which move little between neighbours: 2^-5 in all is more than enough to tell a wrong formula."""
    import paper_2008_12260_amd as px
    g = torch.linspace(-6, 6, 1001, device="cuda")[None]
    u = torch.full_like(g, 1.5)
    h = 2.0 ** -9
    for act in ACTS:
        want = (px.gated(g + h, u, act)[0].double() - px.gated(g - h, u, act)[0].double()) / (2 * h)
        assert float((px.gated_grad(torch.ones_like(g), g, u, act)[0].double() - want).abs().max()) < 2.0 ** -5


def test_graphs_and_no_rows():
    import paper_2008_12260_amd as px
    gate, up, d = inputs(100, 500, torch.bfloat16, 9)
    live = [torch.zeros_like(t) for t in (gate, up, d)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rows, *kept = px.gated(live[0], live[1], keep="i8")
        grads = px.gated_grad(live[2], *kept, want_rows=True)
    for k in range(3):
        new = inputs(100, 500, torch.bfloat16, 20 + k)
        for t, n in zip(live, new):
            t.copy_(n)
        graph.replay()
        torch.cuda.synchronize()
        want_rows, *want_kept = px.gated(new[0], new[1], keep="i8")
        want = px.gated_grad(new[2], *want_kept, want_rows=True)
        assert torch.equal(rows, want_rows) and all(torch.equal(a, b) for a, b in zip(grads, want))
    empty = gate[:0]
    rows, *kept = px.gated(empty, empty, keep="i8")
    assert rows.shape == (0, 500) and px.gated_grad(empty, *kept)[0].shape == (0, 500)
