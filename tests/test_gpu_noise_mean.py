"""The mean that the noise scale's pass gives, where an element's gradients are not finite and where it is rounded."""
import pytest

pytestmark = pytest.mark.gpu

TYPES = ("float32", "bfloat16", "float16")
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("type_", TYPES)
@pytest.mark.parametrize("B", (2, 3, 9))
def test_means_of_what_is_not_finite(B, type_):
    """The formula: infinite where an element's gradients are infinite with one sign, whichever of them is; NaN with both or with a NaN."""
    import torch
    import paper_2008_12260_amd as px
    n = 1000 + 5
    grads = torch.randn((B, n), generator=torch.Generator("cuda").manual_seed(B), device="cuda")
    cases = [({0: INF}, INF), ({0: -INF}, -INF), ({B - 1: INF}, INF), ({B - 1: -INF}, -INF), ({0: INF, B - 1: INF}, INF), ({0: -INF, B - 1: -INF}, -INF),
             ({0: INF, B - 1: -INF}, NAN), ({0: -INF, B - 1: INF}, NAN), ({0: INF, B - 1: NAN}, NAN), ({0: NAN}, NAN), ({B - 1: NAN}, NAN)]
    for k, (held, _) in enumerate(cases):
        for row, value in held.items():
            grads[row, 7 + 91 * k] = value
            if k == 0:
                grads[row, n - 1] = value           # the last element, in a group that is not whole
    grads = grads.to(getattr(torch, type_))
    for mean_dtype in (None, torch.bfloat16, torch.float16):
        mean, scale = px.noise_scale(grads, 4.0, mean_dtype=mean_dtype)
        for k, (_, want) in enumerate(cases):
            got = float(mean[7 + 91 * k])
            assert got == want or got != got and want != want, (k, got, want)
        assert float(mean[n - 1]) == INF
        finite = torch.isfinite(grads).all(0)
        assert int(finite.sum()) == n - len(cases) - 1 and bool(torch.isfinite(mean[finite]).all())
        want = grads.double().mean(0)[finite]
        u = torch.finfo(mean.dtype).eps / 2
        assert bool(((mean[finite].double() - want).abs() <= u * want.abs() + torch.finfo(mean.dtype).smallest_normal * u + 2.0 ** -50 * 8).all())
        assert bool(torch.isnan(scale).all())


def test_means_are_rounded_once():
    """Just above and below the middle of two neighbours of 16 bits, by less than fp32 can tell: 2^-28 of 0.5 + half a step."""
    import torch
    import paper_2008_12260_amd as px
    for dtype in (torch.bfloat16, torch.float16):
        step = torch.finfo(dtype).eps / 2                              # between neighbours of 0.5
        for sign in (1.0, -1.0):
            for odd in (0.0, 1.0):                                     # the lower neighbour's last bit
                for little, up in ((2.0 ** -26, True), (-2.0 ** -26, False)):
                    middle = 0.5 + odd * step + step / 2
                    grads = sign * torch.tensor([[2.0], [4.0 * odd * step], [2.0 * step], [little]], device="cuda").repeat(1, 9)
                    mean, _ = px.noise_scale(grads, 1.0, mean_dtype=dtype)
                    want = sign * (middle + (step / 2 if up else -step / 2))
                    assert bool((mean.double() == want).all()), (dtype, sign, odd, up, float(mean[0]), want)
        # the middle itself: to the neighbour whose last bit is 0
        for odd in (0.0, 1.0):
            grads = torch.tensor([[2.0], [4.0 * odd * step], [2.0 * step], [0.0]], device="cuda").repeat(1, 9)
            mean, _ = px.noise_scale(grads, 1.0, mean_dtype=dtype)
            assert bool((mean.double() == 0.5 + 2.0 * odd * step).all())
    # past the largest number, and below the smallest
    big = torch.full((2, 3), 3.3e38, device="cuda")
    assert bool(torch.isfinite(px.noise_scale(big, 1.0)[0]).all())
    assert bool((px.noise_scale(big, 1.0, mean_dtype=torch.float16)[0] == INF).all()) and bool((px.noise_scale(-big, 1.0, mean_dtype=torch.float16)[0] == -INF).all())
    tiny = torch.full((2, 3), 1e-40, device="cuda")
    assert not bool(px.noise_scale(tiny, 1.0, mean_dtype=torch.float16)[0].any())


@pytest.mark.parametrize("mean_type", TYPES)
@pytest.mark.parametrize("type_", TYPES)
def test_means_are_the_nearest_numbers(type_, mean_type):
    """B a power of two: the sum of the deviations is exact in 64 bits, and so is the mean."""
    import torch
    import paper_2008_12260_amd as px
    g = torch.Generator("cuda").manual_seed(5)
    for B in (2, 4, 8):
        grads = torch.randn((B, 20001), generator=g, device="cuda").to(getattr(torch, type_))
        mean, _ = px.noise_scale(grads, 1.0, mean_dtype=getattr(torch, mean_type))
        want = grads.double().mean(0)
        dt = mean.dtype
        away = (mean.double() - want).abs()
        for other in (INF, -INF):
            near = torch.nextafter(mean, torch.full_like(mean, other)) if dt == torch.float32 else neighbour(mean, other)
            assert bool((away <= (near.double() - want).abs()).all())


def neighbour(x, way):
    """The next number of 16 bits towards an infinity."""
    import torch
    bits = x.view(torch.int16).int()
    grow = (x > 0) == (way > 0)
    moved = torch.where(x == 0, torch.full_like(bits, 1 if way > 0 else -32767), torch.where(grow, bits + 1, bits - 1))
    return moved.to(torch.int16).view(x.dtype)
