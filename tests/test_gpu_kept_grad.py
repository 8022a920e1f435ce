"""The gradient of a layer's weights from its input kept in 8 bits, against 64 bits.

Kept elements are exact in every type, products of 16 bits are exact in fp32 and those of fp32 within 2^-24 of themselves, and a sum of N of them in any order is off by at most N 2^-24 of the sum of
their sizes; a weight, a bias's sum (N 2^-24 again) and product, and what is added to, a few 2^-24 more; the result is rounded once."""
import pytest

torch = pytest.importorskip("torch")

from kept import FORMS, SMALLEST, U, decoded  # noqa: E402

pytestmark = pytest.mark.gpu

TYPES = (torch.float32, torch.bfloat16, torch.float16)


def inputs(N, D, M, dtype, form, seed):
    import paper_2008_12260_amd as px
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn((N, D), generator=g, device="cuda") * torch.exp(torch.randn((N, 1), generator=g, device="cuda"))
    return px.keep(x, form), (0.1 * torch.randn((N, M), generator=g, device="cuda")).to(dtype)


def check(got, kept, d, weight=None, bias=None, added=None):
    x, d = decoded(*kept).cuda(), d.double()
    N = d.shape[0]
    want, size = torch.mm(d.t(), x), torch.mm(d.abs().t(), x.abs())
    if weight is not None:
        want, size = want * weight.double(), size * weight.double().abs()
    if bias is not None:
        want = want + torch.outer(d.sum(0), bias.double())
        size = size + torch.outer(d.abs().sum(0), bias.double().abs())
    if added is not None:
        want, size = want + added.double(), size + added.double().abs()
    tolerance = U[got.dtype] * want.abs() + (N + 12) * 2.0 ** -24 * size + SMALLEST[got.dtype]
    off = (got.double() - want).abs()
    assert bool((off <= tolerance).all()), float((off / tolerance).max())


SIZES = [(1, 1, 1), (1, 64, 8), (3, 33, 5), (64, 32, 16), (65, 100, 77), (200, 257, 130), (127, 512, 64), (1000, 96, 200), (513, 1000, 331), (2048, 256, 320)]


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,D,M", SIZES)
def test_products(N, D, M, dtype, form):
    import paper_2008_12260_amd as px
    kept, d = inputs(N, D, M, dtype, form, N + D + M)
    check(px.kept_grad(kept, d), kept, d)
    g = torch.Generator("cuda").manual_seed(1)
    weight, bias = torch.randn(D, generator=g, device="cuda"), torch.randn(D, generator=g, device="cuda")
    check(px.kept_grad(kept, d, weight, bias), kept, d, weight, bias)
    check(px.kept_grad(kept, d, bias=bias.bfloat16()), kept, d, None, bias.bfloat16())
    into = torch.randn((M, D), generator=g, device="cuda").to(dtype)
    before = into.clone()
    got = px.kept_grad(kept, d, weight.to(dtype), weight_grad=into, accumulate=True)
    assert got is into
    check(got, kept, d, weight.to(dtype), added=before)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", TYPES)
def test_each_shape_of_tile(dtype, form):
    """Large enough for tiles of 256 and 128, and long and thin enough for slices of every kind."""
    import paper_2008_12260_amd as px
    for N, D, M in ((300, 4100, 4200), (700, 1400, 1500), (9000, 256, 512), (5001, 40, 24)):
        kept, d = inputs(N, D, M, dtype, form, N)
        check(px.kept_grad(kept, d), kept, d)


def test_rows_and_results_of_any_stride():
    import paper_2008_12260_amd as px
    kept, d = inputs(100, 70, 48, torch.bfloat16, "i8", 3)
    want = px.kept_grad(kept, d)
    wide = torch.randn((100, 100), device="cuda").bfloat16()
    for at in (0, 8, 3):
        wide[:, at:at + 48] = d
        assert torch.equal(px.kept_grad(kept, wide[:, at:at + 48]), want)
    assert torch.equal(px.kept_grad(kept, d.t().contiguous().t()), want)
    assert torch.equal(px.kept_grad(kept, d.view(4, 25, 48)), want)
    out = torch.full((48, 90), 3.0, dtype=torch.bfloat16, device="cuda")
    px.kept_grad(kept, d, weight_grad=out[:, 8:78])
    assert torch.equal(out[:, 8:78], want) and bool((out[:, :8] == 3).all()) and bool((out[:, 78:] == 3).all())


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", TYPES)
def test_what_is_not_finite_stays_in_its_columns(dtype, form):
    import paper_2008_12260_amd as px
    kept, d = inputs(150, 100, 40, dtype, form, 4)
    x = px.restore(kept, torch.float32)
    x[70, 50] = float("inf")
    bad = px.keep(x, form)
    got, want = px.kept_grad(bad, d), px.kept_grad(kept, d)
    assert bool(torch.isnan(got[:, 32:64]).all())
    assert torch.equal(got[:, :32], want[:, :32]) and torch.equal(got[:, 64:], want[:, 64:])
    d[3, 7] = float("nan")
    got = px.kept_grad(kept, d)
    assert bool(torch.isnan(got[7]).all()) and torch.equal(got[:7], want[:7]) and torch.equal(got[8:], want[8:])


@pytest.mark.parametrize("form", FORMS)
def test_the_smallest_and_the_largest_scales(form):
    """Elements from 2^-124 to 2^127, and gradients that bring the products back to 1: scales whose byte is 0 (2^-127, no normal number) to the largest, in the types that hold them."""
    import paper_2008_12260_amd as px
    g = torch.Generator("cuda").manual_seed(7)
    for dtype in (torch.float32, torch.bfloat16):
        for e in (-123, -120, -118, -100, 100, 118, 125):
            x = (1.0 + torch.rand((200, 96), generator=g, device="cuda")) * 2.0 ** e
            kept, d = px.keep(x, form), (torch.randn((200, 40), generator=g, device="cuda") * 2.0 ** (-e if abs(e) < 110 else -e // 2)).to(dtype)
            assert e > -118 or int(kept.scales.min()) <= 3
            check(px.kept_grad(kept, d), kept, d)


def test_no_rows_give_zeros():
    import paper_2008_12260_amd as px
    for dtype in TYPES:
        kept, d = inputs(0, 40, 24, dtype, "i8", 5)
        assert not bool(px.kept_grad(kept, d).any())
        assert not bool(px.kept_grad(kept, d, bias=torch.ones(40, device="cuda")).any())


def test_streams_graphs_and_the_same_bits():
    import paper_2008_12260_amd as px
    kept, d = inputs(3000, 200, 300, torch.bfloat16, "e4m3", 6)
    bias = torch.randn(200, device="cuda")
    want = px.kept_grad(kept, d, bias=bias)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = px.kept_grad(kept, d, bias=bias, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    live = torch.zeros_like(d)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = px.kept_grad(kept, live, bias=bias)
    for k in range(3):
        live.copy_(d * (k + 1))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, px.kept_grad(kept, d * (k + 1), bias=bias))
