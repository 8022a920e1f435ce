"""Tensors of the right number of elements in a wrong shape are refused, on the host: the device is not asked, and the library not called."""
import pytest

import paper_2008_12260_amd as px

torch = pytest.importorskip("torch")


@pytest.fixture(autouse=True)
def on_the_host(monkeypatch):
    """Tensors of the host pass the question which device they are on; a call that passes all checks stops before the library."""
    class Reached(Exception):
        pass

    def planned(*args, **more):
        raise Reached
    monkeypatch.setattr(px, "_current_device", lambda: -1)
    monkeypatch.setattr(px.train, "_planned", planned)
    return Reached


def test_preconditions_have_a_gradients_shape(on_the_host):
    grads = torch.ones((4, 6, 10))
    for shape in ((10, 6), (6, 10, 1), (3, 20), (1, 60), (60, 1), (59,), ()):
        with pytest.raises(ValueError, match="precondition"):
            px.noise_scale(grads, 1.0, torch.ones(shape))
    for shape in ((6, 10), (60,)):
        with pytest.raises(on_the_host):
            px.noise_scale(grads, 1.0, torch.ones(shape))
    with pytest.raises(on_the_host):
        px.noise_scale(grads.view(4, 60), 1.0, torch.ones(60))
    with pytest.raises(ValueError, match="precondition"):
        px.noise_scale(grads.view(4, 60), 1.0, torch.ones(6, 10))
    with pytest.raises(ValueError, match="precondition"):
        px.noise_scale(torch.ones((3, 1)), 1.0, torch.ones(()))


def test_rows_have_their_tokens_shape(on_the_host):
    tokens = torch.zeros((4, 6), dtype=torch.int64)
    for shape in ((6, 4, 8), (2, 12, 8), (24, 2, 4), (192,), (4, 48), (4, 6), (1, 24, 8), (4, 6, 1, 8), ()):
        with pytest.raises(ValueError, match="rows_grad"):
            px.embed_grad(tokens, torch.ones(shape), 10)
    for shape in ((4, 6, 8), (24, 8), (24, 1)):
        with pytest.raises(on_the_host):
            px.embed_grad(tokens, torch.ones(shape), 10)
    with pytest.raises(on_the_host):
        px.embed_grad(tokens[0, 0], torch.ones(8), 10)


def test_results_have_their_tokens_shape(on_the_host):
    tokens, table = torch.zeros((4, 6), dtype=torch.int64), torch.ones((10, 8))
    for shape in ((6, 4, 8), (2, 12, 8), (8, 24), (192,), (4, 48), (4, 6), (1, 24, 8), ()):
        with pytest.raises(ValueError, match="out"):
            px.embed(tokens, table, out=torch.empty(shape))
    for shape in ((4, 6, 8), (24, 8)):
        with pytest.raises(on_the_host):
            px.embed(tokens, table, out=torch.empty(shape))
