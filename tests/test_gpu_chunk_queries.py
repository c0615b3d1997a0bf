"""Attention of new tokens over the 8-bit cache: how exactly a query's elements enter the scores."""
import pytest
import torch

from test_gpu_chunk import Case, kvp  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("one_each", [True, False])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("below", range(1, 31))
def test_small_elements_beside_a_large_one(kvp, below, dh, one_each):
    """The row's largest meets zeros in K, so that the scores are those of elements around 2^-below of it, with every mantissa.  An
    element counts exactly down to 2^-13 of the row's largest and is off by 2^-21 of that below (2^-31 and 2^-39 for single tokens, by
    f16); K's magnitude is 1, so a score is off by dh times that where elements are below, and by the roundings of its sum, 64 * 2^-23
    of sum |q k|, as everywhere."""
    exact, step = (31, 39) if one_each else (13, 21)
    lens = [200, 40]
    new = [1, 1] if one_each else [129, 40]
    c = Case(kvp, [0], lens, new, 2, 1, dh, 16, 8, one_each=one_each, freed=False)
    g = torch.Generator().manual_seed(below)
    q = torch.randint(128, 256, c.q[0].shape, generator=g) / 128.0 * 2.0 ** -below
    q[..., 0] = 1.0
    if not one_each:
        q[3::4, :, 0] = 0.0                                   # and rows whose largest is among them
    c.q[0].copy_(q)
    assert torch.equal(c.q[0].cpu().float(), q)
    k = torch.where(torch.rand(c.pools[0][0].shape, generator=g) < 0.5, -1.0, 1.0)
    k[:, :, ::2] = k[:, :, ::2].abs()                         # (every second token: all elements of one sign add up)
    k[..., 0] = 0.0
    c.pools[0][0].copy_(k.to(c.pools[0][0].dtype))
    c.scales[0][0].fill_(127)
    scale = 2.0 ** (below - 5)                                # scores of some units
    o, lse = c.run(scale=scale)
    ro, rl, _, _ = c.exact(0, scale)
    rows = torch.tensor([r for r, _, _ in c.rows()], device="cuda")
    large = c.q[0].float().abs().amax(-1)
    size = (c.q[0].double().abs().sum(-1) - c.q[0][..., 0].double().abs()) * scale
    smallest = c.q[0].float().abs().masked_fill(c.q[0] == 0, 1.0).amin(-1)
    off = torch.where(smallest < large * 2.0 ** -exact, dh * 2.0 ** -step * large * scale, 0.0).double()
    # (the factor, the difference to the maximum and ex2: as much again, and 2^-22 of the score)
    tol = off + 2 * 64 * 2.0 ** -23 * size + 2.0 ** -20 * (1 + rl.abs())
    assert (lse[0].double() - rl).abs()[rows].sub(tol[rows]).max() <= 0
