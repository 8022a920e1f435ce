"""Cross entropy over a vocabulary and its gradients against the formulas in 64 bits.

Tolerances, from the formats alone.  u: half a step of the type, relative (fp32 2^-24, bf16 2^-8, fp16 2^-11).  A logit is a sum of D products in fp32: off by at most D 2^-24 sum|h||w| =: dl.  lse moves by no more
than its logits, and its own sum of V exponentials (each within (|x| + 4) 2^-24 of its value, |x| e^-|x| < 1) and logarithm add
(V / 64 + 256) 2^-24 + 4 2^-24 |lse|.  q = g (p - [y]) is off by g p (dl + dlse + 8 2^-24) and rounded to the type (fp16:
no finer than 2^-25 of the largest |g| / 2^12, which the scaling leaves); each gradient is a sum of products with q in fp32, K 2^-24 of the sum of their
sizes, and is rounded once."""
import ctypes

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

TYPES = ("float32", "bfloat16", "float16")
U = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
SMALLEST = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -24}


def inputs(N, V, D, type_, seed, ignored=0.3, i64=True, pad=0):
    """hidden, weight (views of wider buffers where `pad`), targets, row weights."""
    import torch
    g = torch.Generator("cuda").manual_seed(seed)
    dt = getattr(torch, type_)
    hidden = torch.randn((N, D + pad), generator=g, device="cuda").to(dt)[:, :D]
    weight = (torch.randn((V, D + pad), generator=g, device="cuda") * (3.0 * D ** -0.5)).to(dt)[:, :D]
    targets = torch.randint(0, V, (N,), generator=g, device="cuda")
    targets = torch.where(torch.rand(N, generator=g, device="cuda") < ignored, -1, targets)
    row_weight = torch.rand(N, generator=g, device="cuda") * 2.0 - 0.5
    row_weight = torch.where(torch.rand(N, generator=g, device="cuda") < 0.1, 0.0, row_weight)
    return hidden, weight, targets if i64 else targets.int(), row_weight


def reference(hidden, weight, targets, row_weight):
    """Everything in 64 bits, and the bounds that the module's text derives."""
    import torch
    h, w, y = hidden.double(), weight.double(), targets.long()
    type_ = str(hidden.dtype)[6:]
    u, f = U[type_], 2.0 ** -24
    N, D = h.shape
    V = w.shape[0]
    has = (y >= 0) & (y < V)
    logits = torch.mm(h, w.t())
    lse = torch.logsumexp(logits, 1)
    at = torch.where(has, y, 0)
    loss = torch.where(has, lse - logits.gather(1, at[:, None])[:, 0], 0.0)
    dl = D * f * torch.mm(h.abs(), w.abs().t()).amax(1)
    dlse = dl + (V / 64 + 256) * f + 4 * f * lse.abs()
    g = torch.where(has, 1.0 if row_weight is None else row_weight.double(), 0.0)
    counts = g != 0
    p = torch.exp(logits - lse[:, None])
    q = p.clone()
    q[torch.arange(N, device="cuda")[has], y[has]] -= 1.0
    q = torch.where(counts[:, None], q * g[:, None], 0.0)
    dq = torch.where(counts[:, None], g.abs()[:, None] * p * (dl + dlse + 8 * f)[:, None], 0.0) + u * q.abs()
    if type_ == "float16":
        dq = dq + torch.where(counts[:, None], 2.0 ** -37 * g.abs().max(), 0.0)
    hz = torch.where(counts[:, None], h, 0.0)
    hidden_grad, weight_grad = torch.mm(q, w), torch.mm(q.t(), hz)
    size_h, size_w = torch.mm(q.abs(), w.abs()), torch.mm(q.abs().t(), hz.abs())
    dh = torch.mm(dq, w.abs()) + (V + 16) * f * size_h + u * hidden_grad.abs() + SMALLEST[type_]
    dw = torch.mm(dq.t(), hz.abs()) + (N + 16) * f * size_w + u * weight_grad.abs() + SMALLEST[type_]
    return dict(loss=(loss, dlse + dl + f * loss.abs()), lse=(lse, dlse), hidden_grad=(hidden_grad, dh), weight_grad=(weight_grad, dw))


def run(hidden, weight, targets, row_weight, **more):
    import paper_2008_12260_amd as px
    loss, lse = px.token_loss(hidden, weight, targets)
    hidden_grad, weight_grad = px.token_loss_grad(hidden, weight, targets, lse, row_weight, **more)
    return dict(loss=loss, lse=lse, hidden_grad=hidden_grad, weight_grad=weight_grad)


def close(got, want, names=("loss", "lse", "hidden_grad", "weight_grad")):
    for k in names:
        value, bound = want[k]
        off = (got[k].double() - value).abs()
        worst = float((off - bound).max()) if off.numel() else -1.0
        assert worst <= 0.0, (k, worst, float(off.max()), float(bound.max()))


SIZES = [(1, 1, 1), (1, 5, 8), (3, 300, 64), (17, 1000, 72), (64, 257, 128), (130, 2049, 40), (257, 513, 264), (300, 1000, 1001),
         (5, 3000, 13), (513, 700, 96), (1, 4097, 520), (2000, 129, 33)]


@pytest.mark.parametrize("type_", TYPES)
@pytest.mark.parametrize("N,V,D", SIZES)
def test_losses_and_gradients(N, V, D, type_):
    args = inputs(N, V, D, type_, N * 7 + V + D, ignored=0.3 if N > 3 else 0.0, i64=(N + V) % 2 == 0)
    close(run(*args), reference(*args))


@pytest.mark.parametrize("type_", TYPES)
def test_row_weights_of_one_when_none_are_given(type_):
    hidden, weight, targets, _ = inputs(70, 333, 128, type_, 3)
    close(run(hidden, weight, targets, None), reference(hidden, weight, targets, None))


@pytest.mark.parametrize("N,V,D", [(12, 40000, 4096), (1030, 270000, 64)])
def test_several_pieces_of_the_vocabulary(N, V, D):
    """Weights or tokens too many for one piece: the hidden rows' gradient is summed over pieces."""
    args = inputs(N, V, D, "bfloat16", 5)
    close(run(*args), reference(*args))


@pytest.mark.parametrize("type_", TYPES)
@pytest.mark.parametrize("pad", [1, 8])
def test_strided_rows(pad, type_):
    args = inputs(40, 200, 88, type_, 11, pad=pad)
    assert not args[0].is_contiguous()
    got, want = run(*args), reference(*args)
    close(got, want)


def test_results_in_a_callers_strided_buffers():
    import torch
    hidden, weight, targets, row_weight = inputs(33, 130, 70, "bfloat16", 12)
    big_h = torch.full((33, 96), 7.0, dtype=torch.bfloat16, device="cuda")
    big_w = torch.full((130, 71), 7.0, dtype=torch.bfloat16, device="cuda")
    got = run(hidden, weight, targets, row_weight, hidden_grad=big_h[:, :70], weight_grad=big_w[:, :70])
    close(got, reference(hidden, weight, targets, row_weight))
    assert bool((big_h[:, 70:] == 7.0).all()) and bool((big_w[:, 70:] == 7.0).all())


@pytest.mark.parametrize("type_", TYPES)
def test_weight_gradients_are_added_to(type_):
    import torch
    import paper_2008_12260_amd as px
    hidden, weight, targets, row_weight = inputs(50, 301, 72, type_, 13)
    held = torch.randn((301, 72), device="cuda").to(weight.dtype)
    want = reference(hidden, weight, targets, row_weight)
    _, lse = px.token_loss(hidden, weight, targets)
    into = held.clone()
    none, got = px.token_loss_grad(hidden, weight, targets, lse, row_weight, weight_grad=into, accumulate=True, need=(False, True))
    assert none is None and got.data_ptr() == into.data_ptr()
    value, bound = want["weight_grad"]
    total = value + held.double()
    assert bool(((got.double() - total).abs() <= bound + U[type_] * total.abs()).all())


def test_only_the_hidden_gradient():
    import paper_2008_12260_amd as px
    args = inputs(50, 301, 72, "bfloat16", 13)
    _, lse = px.token_loss(*args[:3])
    got, none = px.token_loss_grad(*args[:3], lse, args[3], need=(True, False))
    assert none is None
    close(dict(hidden_grad=got), reference(*args), ("hidden_grad",))


@pytest.mark.parametrize("type_", TYPES)
def test_masked_rows_count_for_nothing_whatever_they_hold(type_):
    import torch
    hidden, weight, targets, row_weight = inputs(90, 300, 64, type_, 17)
    masked = (targets < 0) | (row_weight == 0)
    assert bool(masked.any()) and not bool(masked.all())
    clean = reference(torch.where(masked[:, None], 0.0, hidden.float()).to(hidden.dtype), weight, targets, row_weight)
    for bad in (float("nan"), float("inf"), -float("inf"), torch.finfo(hidden.dtype).min):
        got = run(torch.where(masked[:, None], bad, hidden.float()).to(hidden.dtype), weight, targets, row_weight)
        close(got, clean, ("hidden_grad", "weight_grad"))
        assert bool((got["hidden_grad"][masked] == 0).all())
        assert bool((got["loss"][targets < 0] == 0).all())
    got = run(hidden, weight, torch.full_like(targets, -1), row_weight)
    assert not bool(got["loss"].any()) and not bool(got["hidden_grad"].any()) and not bool(got["weight_grad"].any())


def test_infinite_and_nan_logits_give_what_the_formula_gives():
    import torch
    import paper_2008_12260_amd as px
    inf, nan = float("inf"), float("nan")
    weight = torch.zeros((300, 8), dtype=torch.bfloat16, device="cuda")
    weight[:, 0] = 1.0
    weight[200:, 1] = 1.0
    hidden = torch.zeros((6, 8), dtype=torch.bfloat16, device="cuda")
    hidden[1, 0] = inf          # every logit inf (products of 0 and inf are NaN only where an element is 0: weight[:, 0] is 1)
    hidden[2, 0] = -inf
    hidden[3, 1] = nan
    hidden[4, 0] = 3.0e38       # logits near the largest number
    hidden[5, 0] = -3.0e38
    targets = torch.zeros(6, dtype=torch.int64, device="cuda")
    loss, lse = px.token_loss(hidden, weight, targets)
    want = torch.logsumexp(torch.mm(hidden.double(), weight.double().t()), 1)
    assert bool(torch.isnan(lse[3])) and lse[1] == inf and lse[2] == -inf
    assert abs(float(lse[0]) - np.log(300.0)) < 1e-5
    for n in (4, 5):
        assert abs(float(lse[n]) / float(want[n]) - 1) < 1e-6
    assert bool(torch.isnan(loss[1])) and bool(torch.isnan(loss[2])) and bool(torch.isnan(loss[3]))


def test_targets_outside_the_vocabulary_are_reported_and_count_as_none():
    import torch
    import paper_2008_12260_amd as px
    hidden, weight, targets, row_weight = inputs(40, 100, 64, "bfloat16", 19)
    dims = px.LossDims(40, 100, 64, px.PX_TYPE_BF16, 1, 64, 64, 0, 0)
    need = ctypes.c_size_t()
    assert px.lib().pollux_loss_workspace_size(ctypes.byref(dims), 1, ctypes.byref(need)) == px.PX_OK
    ws = torch.empty(need.value + (1 << 20), dtype=torch.uint8, device="cuda").fill_(0xFF)
    _, lse = px.token_loss(hidden, weight, targets, workspace=ws)
    assert px.pollux_last_status(ws) == 0
    px.token_loss_grad(hidden, weight, targets, lse, row_weight, workspace=ws)
    assert px.pollux_last_status(ws) == 0
    none = targets < 0
    for bad in (100, -2, 1 << 40, -(1 << 40)):
        off = torch.where(none, bad, targets)
        loss, lse = px.token_loss(hidden, weight, off, workspace=ws)
        assert px.pollux_last_status(ws) == px.PX_ST_BAD_TOKEN
        assert bool((loss[none] == 0).all())
        got = px.token_loss_grad(hidden, weight, off, lse, row_weight, workspace=ws)
        assert px.pollux_last_status(ws) == px.PX_ST_BAD_TOKEN
        want = px.token_loss_grad(hidden, weight, targets, lse, row_weight)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_no_tokens():
    import torch
    import paper_2008_12260_amd as px
    weight = torch.randn((100, 64), device="cuda").bfloat16()
    hidden = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    targets = torch.empty(0, dtype=torch.int64, device="cuda")
    loss, lse = px.token_loss(hidden, weight, targets)
    assert loss.shape == lse.shape == (0,)
    held = torch.ones((100, 64), dtype=torch.bfloat16, device="cuda")
    hidden_grad, weight_grad = px.token_loss_grad(hidden, weight, targets, lse, weight_grad=held.clone(), accumulate=True)
    assert hidden_grad.shape == (0, 64) and torch.equal(weight_grad, held)
    _, weight_grad = px.token_loss_grad(hidden, weight, targets, lse)
    assert not bool(weight_grad.any())


def test_gradients_of_tiny_row_weights_keep_their_precision_in_fp16():
    """A mean over 2^20 tokens: q is below fp16's smallest number, the gradients of a scaled loss are not."""
    hidden, weight, targets, row_weight = inputs(60, 500, 64, "float16", 23)
    close(run(hidden, weight * 64, targets, row_weight * 2.0 ** -14), reference(hidden, weight * 64, targets, row_weight * 2.0 ** -14))
    close(run(hidden, weight, targets, row_weight * 2.0 ** 12), reference(hidden, weight, targets, row_weight * 2.0 ** 12))


def test_gradients_against_differences_of_the_loss():
    """fp32, steps of 2^-6 along one direction: the loss's own rounding (some 2^-20) over the step, and the step squared."""
    import torch
    import paper_2008_12260_amd as px
    hidden, weight, targets, row_weight = inputs(48, 200, 64, "float32", 29)
    _, lse = px.token_loss(hidden, weight, targets)
    hidden_grad, weight_grad = px.token_loss_grad(hidden, weight, targets, lse, row_weight)
    total = lambda h, w: float((px.token_loss(h, w, targets)[0].double() * row_weight.double()).sum())
    step = 2.0 ** -6
    for t, grad, other in ((hidden, hidden_grad, lambda t: (t, weight)), (weight, weight_grad, lambda t: (hidden, t))):
        way = torch.randn(t.shape, generator=torch.Generator("cuda").manual_seed(1), device="cuda")
        way /= way.norm()
        slope = (total(*other(t + step * way)) - total(*other(t - step * way))) / (2 * step)
        assert abs(slope - float((grad.double() * way.double()).sum())) < 48 * 2.0 ** -20 / step + step ** 2


def test_the_same_call_gives_the_same_bits_and_streams_may_differ():
    import torch
    args = inputs(700, 5000, 256, "bfloat16", 31)
    want = run(*args)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    import paper_2008_12260_amd as px
    for _ in range(3):
        loss, lse = px.token_loss(*args[:3], stream=other)
        hidden_grad, weight_grad = px.token_loss_grad(*args[:3], lse, args[3], stream=other)
        other.synchronize()
        for k, v in dict(loss=loss, lse=lse, hidden_grad=hidden_grad, weight_grad=weight_grad).items():
            assert torch.equal(v, want[k]), k


def test_recorded_into_a_graph():
    import torch
    import paper_2008_12260_amd as px
    sets = [inputs(100, 1000, 96, "bfloat16", 40 + k) for k in range(3)]
    wants = [run(*s) for s in sets]
    live = [t.clone() for t in sets[0]]
    run(*live)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run(*live)
    for k in (1, 2, 0, 1):
        for t, s in zip(live, sets[k]):
            t.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        eager = run(*sets[k])
        for name in out:
            assert torch.equal(out[name], wants[k][name]) and torch.equal(eager[name], wants[k][name]), name


def test_wrong_tensors_are_refused():
    import torch
    import paper_2008_12260_amd as px
    hidden, weight, targets, row_weight = inputs(8, 50, 64, "bfloat16", 41)
    for bad in ((hidden.cpu(), weight, targets), (hidden.float(), weight, targets), (hidden[:, :32], weight, targets), (hidden, weight, targets[:4]),
                (hidden, weight, targets.float()), (hidden.double(), weight.double(), targets), (hidden[0], weight, targets)):
        with pytest.raises((ValueError, TypeError)):
            px.token_loss(*bad)
    loss, lse = px.token_loss(hidden, weight, targets)
    for more in (dict(row_weight=row_weight.double()), dict(weight_grad=torch.empty((50, 64), device="cuda")), dict(accumulate=True),
                 dict(hidden_grad=torch.empty((64, 8), dtype=torch.bfloat16, device="cuda").t())):
        with pytest.raises((ValueError, TypeError)):
            px.token_loss_grad(hidden, weight, targets, lse, **more)
    small = torch.empty(256, dtype=torch.uint8, device="cuda")
    with pytest.raises(px.PolluxError) as e:
        px.token_loss(hidden, weight, targets, workspace=small)
    assert e.value.code == px.PX_E_WORKSPACE


@pytest.mark.parametrize("type_", ("bfloat16", "float16"))
@pytest.mark.parametrize("N,V,D", [(40, 600, 64), (3, 9, 8), (70, 40001, 72), (300, 3000, 13), (1030, 270000, 24)])
def test_the_targets_share_of_a_hidden_gradient_is_not_rounded(N, V, D, type_):
    """Logits near 0: q is 1 / V but at the target, where it is near the row's weight.  The roundings of the other entries (u each), fp32's
    of the target's, the sum's and the result's are all that is left."""
    import torch
    hidden, weight, targets, row_weight = inputs(N, V, D, type_, 51)
    hidden = hidden * 2.0 ** -9
    u, f = U[type_], 2.0 ** -24
    h, w = hidden.double(), weight.double()
    has = (targets >= 0) & (row_weight != 0)
    logits = torch.mm(h, w.t())
    p = torch.softmax(logits, 1)
    dl = D * f * torch.mm(h.abs(), w.abs().t()).amax(1)
    dlse = dl + (V / 64 + 256) * f + 4 * f * torch.logsumexp(logits, 1).abs()
    g = torch.where(has, row_weight.double(), 0.0)[:, None]
    at = torch.zeros_like(p)
    at[has] = torch.nn.functional.one_hot(targets[has], V).double()
    q = g * (p - at)
    dq = g.abs() * p * (dl + dlse + 8 * f)[:, None] + u * q.abs() * (1 - at) + 4 * f * q.abs() * at
    if type_ == "float16":
        dq = dq + torch.where(has[:, None], 2.0 ** -37 * g.abs().max(), 0.0)
    want = torch.mm(q, w)
    bound = torch.mm(dq, w.abs()) + (V + 16) * f * torch.mm(q.abs(), w.abs()) + u * want.abs() + SMALLEST[type_]
    close(run(hidden, weight, targets, row_weight), dict(hidden_grad=(want, bound)), ("hidden_grad",))


def test_more_tokens_than_are_taken_at_a_time():
    args = inputs(32768 + 37, 300, 16, "bfloat16", 53)
    close(run(*args), reference(*args))
    args = inputs(65536 + 1, 20, 3, "float32", 54, i64=False)
    close(run(*args), reference(*args))


def test_scratch_memory_has_to_be_on_the_gpu():
    import torch
    import paper_2008_12260_amd as px
    hidden, weight, targets, _ = inputs(8, 50, 64, "bfloat16", 55)
    _, lse = px.token_loss(hidden, weight, targets)
    host = torch.empty(1 << 20, dtype=torch.uint8)
    rows = torch.randn((8, 64), device="cuda")
    for call in (lambda w: px.token_loss(hidden, weight, targets, workspace=w), lambda w: px.token_loss_grad(hidden, weight, targets, lse, workspace=w),
                 lambda w: px.embed_grad(targets, rows, 50, workspace=w), lambda w: px.orthogonalize(rows, workspace=w)):
        for bad in (host, torch.empty((1 << 20, 2), dtype=torch.uint8, device="cuda")[:, 0]):
            with pytest.raises(ValueError):
                call(bad)


@pytest.mark.parametrize("N,V,D", [(300, 9000, 300), (600, 5000, 512), (1501, 3001, 77)])
def test_fp32_in_large_tiles(N, V, D):
    """Sizes at which fp32 is multiplied in parts of 16 bits: the same tolerances, with elements of very different sizes too."""
    import torch
    args = inputs(N, V, D, "float32", 61)
    close(run(*args), reference(*args))
    hidden, weight, targets, row_weight = args
    g = torch.Generator("cuda").manual_seed(62)
    hidden = hidden * torch.exp2(torch.randint(-20, 1, (1, D), generator=g, device="cuda").float())
    weight = weight * torch.exp2(torch.randint(-30, 1, (1, D), generator=g, device="cuda").float())
    close(run(hidden, weight, targets, row_weight), reference(hidden, weight, targets, row_weight))


def test_fp32_logits_that_are_not_finite_in_large_tiles():
    import torch
    import paper_2008_12260_amd as px
    inf = float("inf")
    hidden, weight, targets, _ = inputs(600, 5000, 512, "float32", 63, ignored=0.0)
    weight = weight.abs()
    hidden[7, 5] = inf
    hidden[300, 5] = -inf
    hidden[431, 9] = float("nan")
    big = 2.0 ** 127 * (2 - 2.0 ** -23)                 # the largest number, which no bfloat16 holds
    hidden[511] = 0
    hidden[511, 0] = big
    weight[:, 0] = 2.0 ** -124
    loss, lse = px.token_loss(hidden, weight, targets)
    want = torch.logsumexp(torch.mm(hidden.double(), weight.double().t()), 1)
    assert lse[7] == inf and lse[300] == -inf and bool(torch.isnan(lse[431]))
    rest = torch.ones(600, dtype=torch.bool, device="cuda")
    rest[[7, 300, 431]] = False
    assert bool(((lse.double() - want).abs() <= 2.0 ** -10 + 2.0 ** -22 * want.abs())[rest].all())
