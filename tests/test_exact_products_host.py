"""Without a GPU: the operands of the bit-for-bit tests show a product of parts that is left out, and the bound on random ones does."""
import math

import pytest
import torch

from exact_products import BITS, SIX, numbers, one_place, parts

U32 = 2.0 ** -24


def test_every_one_of_the_six_products_shows():
    g = torch.Generator().manual_seed(1)
    shown = set()
    for bits, other in BITS["f32"]:
        a, b = numbers(64, 1, bits, g), numbers(64, 1, other, g)
        pa, pb = parts(a), parts(b)
        assert torch.equal(sum(pa), a) and torch.equal(sum(pb), b)
        want = a.double() * b.double()
        assert torch.equal(want.float().double(), want)
        total = torch.zeros_like(a)
        for i, j in SIX:                                   # in fp32, smallest first: exact
            total = total + pa[i] * pb[j]
        assert torch.equal(total.double(), want)
        for i, j in SIX:
            if (pa[i] * pb[j] != 0).any():
                shown.add((i, j))
    assert shown == set(SIX)


def test_one_number_a_row():
    places, m = one_place(50, 33, 12, torch.Generator().manual_seed(1))
    assert (m != 0).sum(1).eq(1).all() and (m.gather(1, places[:, None]) != 0).all() and len(set(places.tolist())) == 33


@pytest.mark.parametrize("k", [128, 256, 300])
def test_a_random_product_without_one_of_the_six_is_beyond_the_bound(k):
    """The bound of the GPU's test: sqrt(k) + 4 half steps in the root of the mean square."""
    g = torch.Generator().manual_seed(2)
    a, b = torch.randn(200, k, generator=g), torch.randn(300, k, generator=g)
    pa, pb = parts(a), parts(b)
    exact = a.double() @ b.double().t()
    bound = (math.sqrt(k) + 4) * U32 * exact.norm()
    all_six = sum(pa[i].double() @ pb[j].double().t() for i, j in SIX)
    assert (all_six - exact).norm() < 0.05 * bound
    for i, j in SIX:
        assert (all_six - pa[i].double() @ pb[j].double().t() - exact).norm() > 1.5 * bound
