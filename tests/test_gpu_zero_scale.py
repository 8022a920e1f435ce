"""A scale of zero of either sign, one after the other: a plan is kept by a call's values, and the two are equal."""
import pytest

pytestmark = pytest.mark.gpu


def test_scales_of_both_zeros():
    import torch
    import paper_2008_12260_amd as px
    table = torch.tensor([[1.0, -2.0, 3.0], [-4.0, 5.0, -6.0]], device="cuda")
    tokens = torch.tensor([1, 0, 0, 1], device="cuda")
    rows = table[tokens]
    for scale in (0.0, -0.0, 0.0, -0.0):
        assert torch.equal(torch.signbit(px.embed(tokens, table, scale)), torch.signbit(rows * scale)), scale
        got = px.embed_grad(tokens, rows, 2, scale)
        assert not bool(got.any()) and torch.equal(torch.signbit(got), torch.signbit(2.0 * table * scale)), scale
