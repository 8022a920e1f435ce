"""fp32 products in parts of 16 bits: each of them is off by at most 2^-24 of itself, as if it had been rounded to fp32.

Rows in which equal products would add their errors up: even places hold x and z, odd places -(x z rounded to fp32) and 1, whose product no split
changes.  A logit is then D / 2 times what rounding took from x z, and all partial sums are small: of 32 places some 0.25 x z at most, so that
six sums for each 32 places leave 6 (D / 32) 2^-26 |x z|, and a product's own 2^-24 counts D / 2 times."""
import pytest

pytestmark = pytest.mark.gpu


def bits(values):
    import numpy as np
    import torch
    return torch.from_numpy(np.array(values, dtype=np.uint32).view(np.float32).copy())


def test_products_of_equal_rows():
    import torch
    import paper_2008_12260_amd as px
    N, V, D = 600, 5000, 4096                     # tiles of 128
    g = torch.Generator().manual_seed(1)
    low = torch.tensor([0xff80, 0x7f80, 0x8080, 0x7fff, 0x8000, 0x00ff, 0x807f, 0xffff])
    top = torch.randint(0, 128, (N,), generator=g) << 16
    lows = torch.where(torch.arange(N) < 300, low[torch.arange(N) % 8], torch.randint(0, 1 << 16, (N,), generator=g))
    x = bits((0x3f800000 + top + lows).tolist())
    x[0] = bits([0x3f80ff80])[0]
    for z in bits([0x3f80ff80, 0x3f807f80, 0x3fabff80, 0x3fff7f7f, 0x3f9e3779, 0x3f800000]):
        product = x.double() * z.double()
        rounded = product.float()
        hidden, weight = torch.empty((N, D)), torch.empty((V, D))
        hidden[:, 0::2], hidden[:, 1::2] = x[:, None], -rounded[:, None]
        weight[:, 0::2], weight[:, 1::2] = z, 1.0
        want = D / 2 * (product - rounded.double()) + torch.log(torch.tensor(float(V), dtype=torch.float64))
        _, lse = px.token_loss(hidden.cuda(), weight.cuda(), torch.zeros(N, dtype=torch.int64, device="cuda"))
        bound = product * (D / 2 * 2.0 ** -24 + 6 * (D / 32) * 2.0 ** -26) + (V / 64 + 256) * 2.0 ** -24 + 4 * 2.0 ** -24 * want
        off = (lse.double().cpu() - want).abs()
        assert bool((off <= bound).all()), (float(z), int((off - bound).argmax()), float(off.max()), float(bound.max()))
