"""Attention of new tokens over the 8-bit cache with scales, queries and powers of K far from 1."""
import pytest
import torch

from test_gpu_chunk import Case, kvp  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("one_each", [True, False])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("scale,gain,power", [
    (0.25, 1.0, -6), (3.0, 1.0, -6), (0.0, 40.0, -6), (0.0, 2.0 ** -100, -6), (0.0, 0.0, -6), (1e-30, 1e30, -6),     # as over the bf16 cache
    (0.0, 2.0 ** 100, -100), (0.0, 2.0 ** -105, 100), (0.0, 2.0 ** -100, -100), (2.0 ** 90, 2.0 ** -96, 0), (2.0 ** -100, 2.0 ** 50, 48), (0.0, 2.0 ** -115, 113),
])
def test_scales(kvp, scale, gain, power, dh, one_each):
    """K of magnitudes around 2^power to 2^(power + 4)."""
    lens = [1000, 77]
    c = Case(kvp, [0], lens, [1, 1] if one_each else [20, 77], 4, 1, dh, 16, 8, gain=gain, one_each=one_each)
    g = torch.Generator().manual_seed(8)
    s = c.scales[0][0]
    live = s != 255                                           # (blocks that no row sees stay as they are)
    s.copy_(torch.where(live, torch.randint(127 + power - 6, 127 + power - 2, s.shape, generator=g, dtype=torch.uint8).cuda(), s))
    c.check(*c.run(scale=scale), scale)


@pytest.mark.parametrize("dh", [64, 128])
def test_powers_of_rows_side_by_side(kvp, dh):
    """Rows of 2^-110 to 2^110 in one tile, K's powers to match none of them."""
    c = Case(kvp, [0, 0], [700, 90], [90, 33], 4, 2, dh, 16, 8)
    g = torch.Generator().manual_seed(9)
    for l in range(2):
        c.q[l].copy_(c.q[l].float() * torch.exp2(torch.randint(-110, 13, (c.T, 4, 1), generator=g).float()).cuda())
    c.check(*c.run(scale=2.0 ** -12), 2.0 ** -12)
