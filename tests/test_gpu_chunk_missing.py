"""Attention of new tokens where visible places of the table hold no page (a page of zeros: score 0, value 0), by either form of the
call: one token a sequence without `first`, and rows by `first`."""
import pytest
import torch

from test_gpu_chunk import Case, kvp  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


def take_out(c, places):
    """places: (sequence, place) pairs whose number becomes one outside the pool."""
    for i, (b, place) in enumerate(places):
        c.bt[b, place] = (-1, c.desc.n_pages, 1 << 30, -7, -(1 << 31), (1 << 31) - 1)[i % 6]
    c.table = c.bt.cuda()


LENS = {
    "short": [70, 1, 33, 64, 65, 0, 200, 17, 16],
    "long": [20000],                                          # over many shares
    "many": [40 + 7 * (i % 50) for i in range(150)],
    "mixed": [9000, 300, 20, 5000, 64],
}


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dh,page,G,window,sinks", [(64, 16, 4, 0, 0), (128, 48, 4, 0, 0), (128, 16, 2, 150, 20), (64, 64, 1, 100, 0), (128, 32, 16, 0, 0)])
@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("one_each", [True, False])
def test_visible_places_without_a_page(kvp, lens, one_each, dh, page, G, window, sinks, bits):
    """The first, the last (the row's own token's), every third and all places of a sequence."""
    lens = LENS[lens]
    c = Case(kvp, [0, 0] if G < 16 else [0], lens, [min(n, 1) for n in lens], 2 * G, 2, dh, page, bits, window, sinks, one_each=one_each, freed=False)
    places = []
    for b, n in enumerate(lens):
        k = -(-n // page)
        places += [(b, i) for i in range(k) if (i == 0, i == k - 1, i % 3 == 1, True, i < k // 2)[b % 5]]
    take_out(c, places)
    c.check(*c.run())


@pytest.mark.parametrize("bits", [16, 8])
def test_rows_of_a_chunk(kvp, bits):
    """Several tokens a sequence, whose own places are among the missing ones."""
    c = Case(kvp, [0, 0, 2], [300, 90, 1000], [70, 90, 3], 4, 2, 64, 16, bits, freed=False)
    take_out(c, [(0, 0), (0, 15), (0, 18), (1, 0), (1, 1), (2, 5), (2, 62)] + [(2, i) for i in range(20, 50)])
    c.check(*c.run())


@pytest.mark.parametrize("one_each", [True, False])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("power", [-100, -40, 0, 60])
def test_small_scales_beside_a_missing_page(kvp, power, dh, one_each):
    """The zeros of a missing page take no bits from values of any size: V's scales around 2^power in the 8-bit cache."""
    lens = [90, 300, 7000]
    c = Case(kvp, [0, 0], lens, [1] * 3 if one_each else [1, 80, 3], 4, 2, dh, 32, 8, one_each=one_each, freed=False)
    g = torch.Generator().manual_seed(11)
    for x in c.scales[1]:
        x.copy_(torch.randint(127 + power, 130 + power, x.shape, generator=g, dtype=torch.uint8))
    take_out(c, [(0, 0), (1, 2), (1, 9)] + [(2, i) for i in range(0, 219, 4)])
    c.check(*c.run())
