"""What is kept of a call's sizes and values is told apart by all of them, signs of zeros too (no GPU needed)."""
import pytest

import paper_2008_12260_amd as px

torch = pytest.importorskip("torch")


def test_zeros_of_either_sign_have_plans_of_their_own(monkeypatch):
    seen = []
    planned = px.train._planned

    class Reached(Exception):
        pass

    def watched(*args):
        seen.append(planned(*args)[0]._obj)
        raise Reached
    monkeypatch.setattr(px, "_current_device", lambda: -1)
    monkeypatch.setattr(px.train, "_planned", watched)
    tokens, table = torch.zeros(3, dtype=torch.int64), torch.ones((4, 8))

    def sign(x):
        return str(x).startswith("-")
    for zero in (0.0, -0.0, 0.0):
        for call, of in ((lambda: px.embed(tokens, table, zero), lambda d: (d.scale,)), (lambda: px.embed_grad(tokens, table[:3], 4, zero), lambda d: (d.scale,)),
                         (lambda: px.orthogonalize(table, 2, (zero, zero, zero)), lambda d: (d.a, d.b, d.c))):
            with pytest.raises(Reached):
                call()
            assert all(v == 0.0 and sign(v) == sign(zero) for v in of(seen[-1])), zero
