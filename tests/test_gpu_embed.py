"""Rows looked up by token, and the table's gradient, against 64 bits.

Tolerances: a looked-up row is one product, rounded once (u: half a step of the rows' type; the product itself is in fp32, 2^-24
more).  An entry's gradient is an fp32 sum of c rows, off by at most c 2^-24 of the sum of their sizes, times scale (2^-24), added
to what was held (2^-24) and rounded once."""
import pytest

pytestmark = pytest.mark.gpu

TYPES = ("float32", "bfloat16", "float16")
U = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
SMALLEST = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -24}


def tokens_of(N, V, seed, ignored=0.1, skewed=True):
    import math
    import torch
    g = torch.Generator("cuda").manual_seed(seed)
    u = torch.rand(N, generator=g, device="cuda", dtype=torch.float64)
    t = ((torch.exp(u * math.log(V + 1.0)) - 1).long() if skewed else (u * V).long()).clamp(0, V - 1)
    return torch.where(torch.rand(N, generator=g, device="cuda") < ignored, -1, t)


def gradient(tokens, rows, V, scale, held=None):
    """(value, bound before the result's own rounding) in 64 bits."""
    import torch
    keep = (tokens >= 0) & (tokens < V)
    t, r = tokens[keep].long(), rows[keep].double()
    value = torch.zeros((V, rows.shape[1]), dtype=torch.float64, device="cuda").index_add_(0, t, r)
    size = torch.zeros_like(value).index_add_(0, t, r.abs())
    count = torch.zeros(V, dtype=torch.float64, device="cuda").index_add_(0, t, torch.ones_like(t, dtype=torch.float64))
    f = 2.0 ** -24
    bound = (count[:, None] + 2) * f * size * abs(scale)
    value = value * scale
    if held is not None:
        value = value + held.double()
        bound = bound + f * value.abs()
    return value, bound


def close(got, value, bound):
    import torch
    type_ = str(got.dtype)[6:]
    assert bool(((got.double() - value).abs() <= bound + U[type_] * (value.abs() + bound) + SMALLEST[type_]).all())


@pytest.mark.parametrize("rows_type", TYPES)
@pytest.mark.parametrize("table_type", TYPES)
def test_lookup(table_type, rows_type):
    import torch
    import paper_2008_12260_amd as px
    for N, V, D, i64 in ((1, 1, 1, True), (5, 9, 8, False), (70, 300, 1000, True), (333, 50, 77, False), (3, 1000, 4096 * 3 + 5, True)):
        table = torch.randn((V, D), device="cuda").to(getattr(torch, table_type))
        tokens = tokens_of(N, V, N + D)
        for scale in (1.0, -0.37, 8.0):
            got = px.embed(tokens if i64 else tokens.int(), table, scale, dtype=getattr(torch, rows_type))
            want = torch.where(tokens[:, None] >= 0, table[tokens.clamp(min=0)].double() * float(torch.tensor(scale).float()), 0.0)
            close(got, want, 2.0 ** -24 * want.abs())
            assert bool((got[tokens < 0] == 0).all())


def test_lookup_of_many_dimensions_strided_rows_and_infinite_entries():
    import torch
    import paper_2008_12260_amd as px
    table = torch.randn((40, 33), device="cuda").bfloat16()[:, :31]
    table[7] = float("nan")
    table[8] = float("inf")
    tokens = torch.tensor([[1, -1, 39], [8, 0, 2]], device="cuda")
    out = torch.full((2, 3, 31), 5.0, dtype=torch.bfloat16, device="cuda")
    got = px.embed(tokens, table, 2.0, out=out)
    assert got.data_ptr() == out.data_ptr()
    want = torch.where(tokens[..., None] >= 0, table[tokens.clamp(min=0)] * 2.0, 0.0)
    assert torch.equal(got, want)
    assert px.embed(torch.empty((0, 4), dtype=torch.int32, device="cuda"), table).shape == (0, 4, 31)


def test_tokens_outside_the_table_are_reported_and_give_zeros():
    import torch
    import paper_2008_12260_amd as px
    table = torch.randn((40, 64), device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    tokens = torch.tensor([3, -1, 39], device="cuda")
    px.embed(tokens, table, status=status)
    assert int(status) == 0
    for bad in (40, -2, 1 << 40, -(1 << 50)):
        status.zero_()
        tokens[1] = bad
        got = px.embed(tokens, table, status=status)
        assert int(status) == px.PX_ST_BAD_TOKEN
        assert torch.equal(got[0], table[3]) and torch.equal(got[2], table[39]) and not bool(got[1].any())
        for N in (3, 3000):
            many = torch.cat([tokens, torch.full((N - 3,), 5, device="cuda")])
            dims = px.EmbedDims(N, 40, 64, px.PX_TYPE_F32, px.PX_TYPE_F32, 1, 1.0, 0, 0)
            ws = torch.full((1 << 22,), 255, dtype=torch.uint8, device="cuda")
            rows = torch.randn((N, 64), device="cuda")
            close(px.embed_grad(many, rows, 40, workspace=ws), *gradient(many, rows, 40, 1.0))
            assert px.pollux_last_status(ws) == px.PX_ST_BAD_TOKEN
            many[1] = -1
            px.embed_grad(many, rows, 40, workspace=ws)
            assert px.pollux_last_status(ws) == 0


# up to 512 tokens one workgroup ranks, beyond them several sort; windows hold 8 to 32 places, and 128 beyond 2^17 tokens
CASES = [(1, 1, 1), (1, 100, 64), (7, 3, 5), (33, 1000, 40), (1024, 50, 24), (1025, 50, 24), (1500, 1, 8), (5000, 1023, 100), (5000, 1024, 2500),
         (70001, 30000, 9), (200000, 300, 16), (3000, 1000003, 3)]


@pytest.mark.parametrize("rows_type,table_type", [("float32", "float32"), ("bfloat16", "bfloat16"), ("float16", "float16"), ("bfloat16", "float32"),
                                                  ("float32", "float16")])
@pytest.mark.parametrize("N,V,D", CASES)
def test_gradients(N, V, D, rows_type, table_type):
    import torch
    import paper_2008_12260_amd as px
    tokens = tokens_of(N, V, N + V, skewed=N % 2 == 0)
    rows = torch.randn((N, D), device="cuda", generator=torch.Generator("cuda").manual_seed(D)).to(getattr(torch, rows_type))
    got = px.embed_grad(tokens if V % 2 else tokens.int(), rows, V, 0.75, dtype=getattr(torch, table_type))
    close(got, *gradient(tokens, rows, V, 0.75))


@pytest.mark.parametrize("type_", TYPES)
def test_gradients_are_added_to(type_):
    import torch
    import paper_2008_12260_amd as px
    for N, V, D in ((50, 200, 30), (3000, 2000, 72)):
        tokens = tokens_of(N, V, 3)
        rows = torch.randn((N, D), device="cuda").to(getattr(torch, type_))
        buffer = torch.randn((V, D + 3), device="cuda").to(getattr(torch, type_))
        before = buffer.clone()
        got = px.embed_grad(tokens, rows, V, 2.5, table_grad=buffer[:, :D], accumulate=True)
        assert got.data_ptr() == buffer.data_ptr()
        close(got, *gradient(tokens, rows, V, 2.5, before[:, :D]))
        absent = torch.ones(V, dtype=torch.bool, device="cuda")
        absent[tokens[tokens >= 0]] = False
        assert torch.equal(buffer[absent], before[absent]) and torch.equal(buffer[:, D:], before[:, D:])


def test_no_tokens_one_token_everywhere_and_none_that_counts():
    import torch
    import paper_2008_12260_amd as px
    rows = torch.randn((4000, 136), device="cuda")
    for N in (0, 1, 31, 32, 33, 64, 1023, 4000):
        for tokens in (torch.full((N,), 17, device="cuda"), torch.full((N,), -1, device="cuda")):
            got = px.embed_grad(tokens, rows[:N], 100)
            close(got, *gradient(tokens, rows[:N], 100, 1.0))


def test_rows_of_masked_tokens_may_hold_anything():
    import torch
    import paper_2008_12260_amd as px
    tokens = tokens_of(3000, 500, 9, ignored=0.5)
    rows = torch.randn((3000, 64), device="cuda").bfloat16()
    want = px.embed_grad(tokens, rows, 500)
    for bad in (float("nan"), float("inf")):
        assert torch.equal(px.embed_grad(tokens, torch.where(tokens[:, None] < 0, bad, rows.float()).bfloat16(), 500), want)
    rows[5] = float("nan")
    tokens[5] = 3
    got = px.embed_grad(tokens, rows, 500)
    assert bool(torch.isnan(got[3]).all()) and not bool(torch.isnan(got[4:]).any()) and not bool(torch.isnan(got[:3]).any())


def test_the_same_call_gives_the_same_bits_on_other_streams_and_in_graphs():
    import torch
    import paper_2008_12260_amd as px
    V, D = 3000, 200
    sets = [(tokens_of(9000, V, k), torch.randn((9000, D), device="cuda").bfloat16()) for k in range(3)]
    wants = [(px.embed(t, r[:V], 3.0), px.embed_grad(t, r, V)) for t, r in sets]
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    for _ in range(3):
        got = px.embed_grad(*sets[0], V, stream=other)
        other.synchronize()
        assert torch.equal(got, wants[0][1])
    t, r = (x.clone() for x in sets[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rows, grad = px.embed(t, r[:V], 3.0), px.embed_grad(t, r, V)
    for k in (1, 2, 0, 1):
        t.copy_(sets[k][0])
        r.copy_(sets[k][1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(rows, wants[k][0]) and torch.equal(grad, wants[k][1])
        assert torch.equal(px.embed_grad(*sets[k], V), wants[k][1])


def test_the_gradient_is_the_lookups():
    """<embed(T), R> = <T, embed_grad(R)>: both sides in 64 bits from fp32 results, each element rounded once or summed in fp32."""
    import torch
    import paper_2008_12260_amd as px
    tokens = tokens_of(2000, 400, 4)
    table, rows = torch.randn((400, 96), device="cuda"), torch.randn((2000, 96), device="cuda")
    left = (px.embed(tokens, table, 1.5).double() * rows.double()).sum()
    grad = px.embed_grad(tokens, rows, 400, 1.5)
    right = (table.double() * grad.double()).sum()
    value, bound = gradient(tokens, rows, 400, 1.5)
    slack = (table.double().abs() * (bound + 2.0 ** -24 * value.abs())).sum() + 2.0 ** -23 * (px.embed(tokens, table, 1.5).double() * rows.double()).abs().sum()
    assert abs(float(left - right)) <= float(slack)


def test_wrong_tensors_are_refused():
    import torch
    import paper_2008_12260_amd as px
    table, tokens = torch.randn((50, 64), device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    rows = torch.randn((4, 64), device="cuda")
    for bad in ((tokens.cpu(), table), (tokens, table.cpu()), (tokens.float(), table), (tokens, table.double()), (tokens, table[0])):
        with pytest.raises((ValueError, TypeError)):
            px.embed(*bad)
    for more in (dict(dtype=torch.float64), dict(out=torch.empty((4, 64), dtype=torch.bfloat16, device="cuda")), dict(status=torch.zeros(2, dtype=torch.int32, device="cuda"))):
        with pytest.raises((ValueError, TypeError)):
            px.embed(tokens, table, **more)
    for args, more in (((tokens, rows[:3], 50), {}), ((tokens, rows, 50), dict(accumulate=True)), ((tokens, rows, 50), dict(table_grad=torch.empty((49, 64), device="cuda")))):
        with pytest.raises((ValueError, TypeError)):
            px.embed_grad(*args, **more)
    with pytest.raises(px.PolluxError) as e:
        px.embed(tokens, table, float("nan"))
    assert e.value.code == px.PX_E_INVALID_ARG


def test_tables_of_any_place_are_zeroed_to_their_ends_and_no_further():
    """Rows with and without gaps, of odd lengths, in fp32 and 16 bits, few and many tokens, within the memory-side cache and beyond: entries that
    no token names are zeros, what lies between the rows and behind them is left."""
    import torch
    import paper_2008_12260_amd as px
    for N, V, D, gap, type_ in ((5, 1001, 7, 0, "bfloat16"), (5, 1001, 7, 2, "float32"), (2000, 333, 33, 0, "float16"), (2000, 333, 33, 3, "bfloat16"), (3, 4097, 129, 0, "float32"),
                                (1100, 70001, 2001, 0, "bfloat16"), (9, 70001, 1001, 3, "float32")):
        tokens = tokens_of(N, V, N)
        rows = torch.randn((N, D), device="cuda").to(getattr(torch, type_))
        flat = torch.full((V * (D + gap) + 64,), 7.0, dtype=rows.dtype, device="cuda")
        table = flat[:V * (D + gap)].view(V, D + gap)
        got = px.embed_grad(tokens, rows, V, table_grad=table[:, :D])
        absent = torch.ones(V, dtype=torch.bool, device="cuda")
        absent[tokens[tokens >= 0]] = False
        assert not bool(got[absent].any())
        assert bool((table[:, D:] == 7.0).all()) and bool((flat[V * (D + gap):] == 7.0).all())
        named = torch.unique(tokens[tokens >= 0])
        value, bound = gradient(torch.searchsorted(named, tokens.clamp(min=-1)).where(tokens >= 0, -1), rows, len(named), 1.0)
        close(got[named], value, bound)


@pytest.mark.parametrize("rows_type,table_type", [("float32", "float32"), ("bfloat16", "bfloat16"), ("float16", "float32")])
@pytest.mark.parametrize("N,V,D,share", [(1, 5, 300, 0.0), (9, 2, 520, 0.3), (17, 40, 257, 0.0), (1025, 3, 264, 0.1), (8193, 700, 1000, 0.1), (16390, 9000, 513, 0.0), (33000, 50, 300, 0.9),
                                         (140001, 400, 258, 0.1)])
def test_gradients_of_wide_rows(N, V, D, share, rows_type, table_type):
    """Rows of more than 256 elements: a wavefront a window, in windows of 8 to 128 places, runs within and across them, few and most tokens masked."""
    import torch
    import paper_2008_12260_amd as px
    tokens = tokens_of(N, V, N + D, ignored=share)
    rows = torch.randn((N, D), device="cuda", generator=torch.Generator("cuda").manual_seed(D)).to(getattr(torch, rows_type))
    rows[tokens < 0] = float("nan")
    got = px.embed_grad(tokens, rows, V, 1.25, dtype=getattr(torch, table_type))
    close(got, *gradient(tokens, rows, V, 1.25))


def test_every_number_of_few_tokens_is_ranked():
    """Up to 512 tokens are ranked by threads in proportion: each count of them has its own share."""
    import torch
    import paper_2008_12260_amd as px
    rows = torch.randn((1025, 24), device="cuda")
    for N in list(range(1, 40)) + [63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 512, 513, 800, 1023, 1024, 1025]:
        tokens = tokens_of(N, 37, N, ignored=0.2)
        close(px.embed_grad(tokens, rows[:N], 37), *gradient(tokens, rows[:N], 37, 1.0))
    tokens = tokens_of(900, (1 << 20) - 1, 3, skewed=False)
    close(px.embed_grad(tokens, rows[:900, :8], (1 << 20) - 1), *gradient(tokens, rows[:900, :8], (1 << 20) - 1, 1.0))
