"""Row weights many powers of two apart, against 64 bits: in fp16 q is held to half a step of its type or to 2^-37 of the largest weight,
whichever is coarser (the bound of `reference`), and each row of the hidden rows' gradient is then that much less exact."""
import pytest

from test_gpu_token_loss import TYPES, close, inputs, reference, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("type_", TYPES)
@pytest.mark.parametrize("N,V,D", [(64, 500, 64), (300, 1000, 72), (513, 3000, 40)])
def test_weights_many_powers_of_two_apart(N, V, D, type_):
    import torch
    hidden, weight, targets, row_weight = inputs(N, V, D, type_, 71)
    power = torch.randint(-30, 1, (N,), generator=torch.Generator("cuda").manual_seed(72), device="cuda").float()
    for factor in (1.0, 2.0 ** -10, 2.0 ** 10):
        scaled = row_weight * torch.exp2(power) * factor
        close(run(hidden, weight, targets, scaled), reference(hidden, weight, targets, scaled))


def test_small_ones_alone_keep_their_precision_in_fp16():
    """The largest weight of a call sets the scale: without large ones the bound is relative to the small ones.  (Weights of 2^12 bring the gradients
    well above fp16's smallest numbers, 2^-24.)"""
    hidden, weight, targets, row_weight = inputs(100, 700, 64, "float16", 73)
    args = hidden * 2.0 ** -10, weight * 2.0 ** 12, targets, row_weight * 2.0 ** -20
    want = reference(*args)
    close(run(*args), want, ("hidden_grad",))
    assert float(want["hidden_grad"][0].abs().max()) > 2.0 ** -12
