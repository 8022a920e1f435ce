"""A training iteration's calls record nothing for autograd: what requires grad is refused where it would be followed, and the calls make a
torch.autograd.Function where it is not."""
import pytest

import paper_2008_12260_amd as px

torch = pytest.importorskip("torch")


def calls(device):
    """(name of the tensor that requires grad, the call with it)."""
    tokens = torch.tensor([1, 0, 3], device=device)

    def new(*shape, dtype=torch.float32):
        return torch.ones(shape, dtype=dtype, device=device)

    def leaf(*shape, dtype=torch.float32):
        return new(*shape, dtype=dtype).requires_grad_()

    bf16 = torch.bfloat16
    return [("table", lambda: px.embed(tokens, leaf(4, 8))), ("out", lambda: px.embed(tokens, new(4, 8), out=leaf(3, 8))),
            ("rows_grad", lambda: px.embed_grad(tokens, leaf(3, 8), 4)), ("table_grad", lambda: px.embed_grad(tokens, new(3, 8), 4, table_grad=leaf(4, 8))),
            ("hidden", lambda: px.token_loss(leaf(3, 8), new(4, 8), tokens)), ("weight", lambda: px.token_loss(new(3, 8), leaf(4, 8), tokens)),
            ("a result of hidden", lambda: px.token_loss(leaf(3, 8) * 2.0, new(4, 8), tokens)),
            ("hidden", lambda: px.token_loss_grad(leaf(3, 8), new(4, 8), tokens, new(3))), ("weight", lambda: px.token_loss_grad(new(3, 8), leaf(4, 8), tokens, new(3))),
            ("lse", lambda: px.token_loss_grad(new(3, 8), new(4, 8), tokens, leaf(3))),
            ("row_weight", lambda: px.token_loss_grad(new(3, 8), new(4, 8), tokens, new(3), leaf(3))),
            ("hidden_grad", lambda: px.token_loss_grad(new(3, 8), new(4, 8), tokens, new(3), hidden_grad=leaf(3, 8))),
            ("weight_grad", lambda: px.token_loss_grad(new(3, 8), new(4, 8), tokens, new(3), weight_grad=leaf(4, 8))),
            ("grads", lambda: px.noise_scale(leaf(3, 8), 1.0)), ("precondition", lambda: px.noise_scale(new(3, 8), 1.0, leaf(8))),
            ("grads", lambda: px.orthogonalize(leaf(3, 8))), ("out", lambda: px.orthogonalize(new(3, 8), out=leaf(3, 8, dtype=bf16)))]


def test_what_requires_grad_is_refused():
    for name, call in calls("cpu"):
        with pytest.raises(ValueError, match="requires grad"):
            call()
            pytest.fail(name)


def test_what_has_a_tangent_is_refused():
    from torch.autograd import forward_ad
    dual = lambda *shape: forward_ad.make_dual(torch.ones(shape), torch.ones(shape))
    tokens, x = torch.tensor([1, 0, 3]), torch.ones((3, 8))
    with forward_ad.dual_level():
        for call in (lambda: px.embed(tokens, dual(4, 8)), lambda: px.embed_grad(tokens, dual(3, 8), 4), lambda: px.token_loss(dual(3, 8), torch.ones((4, 8)), tokens),
                     lambda: px.token_loss_grad(x, dual(4, 8), tokens, torch.ones(3)), lambda: px.noise_scale(dual(3, 8), 1.0), lambda: px.orthogonalize(dual(3, 8))):
            with pytest.raises(ValueError, match="tangent"):
                call()
            with torch.no_grad(), pytest.raises(ValueError, match="tangent"):
                call()


@pytest.mark.gpu
def test_what_requires_grad_is_taken_where_it_is_not_followed():
    for name, call in calls("cuda"):
        with pytest.raises(ValueError, match="requires grad"):
            call()
            pytest.fail(name)
        with torch.no_grad():
            got = call()
        for t in got if isinstance(got, tuple) else (got,):
            assert t is None or t.is_cuda


@pytest.mark.gpu
def test_a_function_made_of_the_calls_has_the_gradients_autograd_gives():
    """fp32; the bound is of sums of at most 300 products with q, each within 2^-24 of itself, and of q's own error: its logits are sums of 32 products,
    33 * 2^-24 of |h||w| < 64 in all, so that q is off by less than 2^-13 of itself."""
    class Embedded(torch.autograd.Function):
        @staticmethod
        def forward(ctx, tokens, table):
            ctx.save_for_backward(tokens)
            ctx.entries = table.shape[0]
            return px.embed(tokens, table, 2.0)

        @staticmethod
        def backward(ctx, grad):
            return None, px.embed_grad(ctx.saved_tensors[0], grad.contiguous(), ctx.entries, 2.0)

    class Loss(torch.autograd.Function):
        @staticmethod
        def forward(ctx, hidden, weight, targets):
            loss, lse = px.token_loss(hidden, weight, targets)
            ctx.save_for_backward(hidden, weight, targets, lse)
            return loss

        @staticmethod
        def backward(ctx, grad):
            return (*px.token_loss_grad(*ctx.saved_tensors, grad.contiguous()), None)

    g = torch.Generator("cuda").manual_seed(1)
    table, weight = (torch.randn((300, 32), generator=g, device="cuda") for _ in range(2))
    tokens, targets = (torch.randint(0, 300, (70,), generator=g, device="cuda") for _ in range(2))
    leaves = table.clone().requires_grad_(), weight.clone().requires_grad_()
    Loss.apply(Embedded.apply(tokens, leaves[0]), leaves[1], targets).mean().backward()
    wants = table.double().requires_grad_(), weight.double().requires_grad_()
    torch.nn.functional.cross_entropy((2.0 * wants[0][tokens]) @ wants[1].t(), targets).backward()
    for got, want in zip(leaves, wants):
        size = float(want.grad.abs().max())
        assert size > 0 and float((got.grad.double() - want.grad).abs().max()) <= 2.0 ** -12 * size
