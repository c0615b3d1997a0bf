"""Attention of new tokens with scores of great magnitude, whose rounding alone is far more than a power of two."""
import numpy as np
import pytest
import torch

from test_gpu_chunk import Case, kvp  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("one_each", [False, True])
@pytest.mark.parametrize("dh,Hq,lens,new", [(64, 4, [40, 3], [40, 1]), (128, 4, [32, 1000], [5, 300]), (128, 12, [20000], [2]), (64, 1, [300], [300])])
@pytest.mark.parametrize("power", [10, 16, 22, 28, 34, 50, 90])
def test_scores_of_great_magnitude_that_are_rounded(kvp, dh, Hq, lens, new, power, one_each, bits):
    """Two keys in turn, whose scores are numbers like any others times 2^power: tokens of the larger one have one weight, the others none.
    (Every query has an element of 1 or -1 along the keys' difference: scores 2^power and more apart, far more than their errors.)
    The largest of a row have the weight 1, which P holds exactly: 2^-8 and 2^-11 are room for P, 2^-13 for the sums, as elsewhere."""
    c = Case(kvp, [0], lens, [1] * len(lens) if one_each else new, Hq, 1, dh, 16, bits, one_each=one_each, freed=False)
    g = torch.Generator(device="cuda").manual_seed(power)
    two = torch.randn(2, dh, device="cuda", generator=g)
    two = (two * 64).to(torch.float8_e4m3fn).float() if bits == 8 else two.bfloat16().float()
    q, along = torch.randn(c.T, Hq, dh, device="cuda", generator=g), torch.nn.functional.normalize(two[0] - two[1], dim=0)
    sign = torch.tensor([1.0, -1.0, -1.0] * Hq, device="cuda")[:Hq, None]
    q = (q - (q @ along)[..., None] * along + sign * along).bfloat16()
    of_key = 2.0 ** (-6 if bits == 8 else 0)
    y = q.double() @ two.double().T * of_key * 0.25           # [T, Hq, 2]
    assert ((y[..., 0] - y[..., 1]).abs() > 1).all()
    c.q[0][:] = q * 2.0 ** (power // 2)
    up = power - power // 2
    if bits == 8:
        c.scales[0][0].fill_(127 - 6 + up)
    else:
        two = two * 2.0 ** up
    c.pools[0][0][:, :, 0::2] = two[0].to(c.pools[0][0].dtype)
    c.pools[0][0][:, :, 1::2] = two[1].to(c.pools[0][0].dtype)
    o, lse = c.run(scale=0.25)
    part = 2.0 ** (-11 if bits == 8 else -8) + 2.0 ** -13
    for row, b, pos in list(c.rows())[::7] + list(c.rows())[-3:]:
        v = c.keys(b, pos + 1, 0)[1][0]
        for h in range(Hq):
            best = int(y[row, h].argmax()) if pos > 0 else 0
            won = v[best::2]
            want, size = won.mean(0), won.abs().mean(0)
            assert ((o[0][row, h].double() - want).abs() <= 2.0 ** -8 * want.abs() + size * part).all(), (b, pos, h)
            assert abs(float(lse[0][row, h]) - float(y[row, h, best]) * 2.0 ** power - np.log(len(won))) <= 2.0 ** -16 * float(y[row, h].abs().max() + 16) * 2.0 ** power
