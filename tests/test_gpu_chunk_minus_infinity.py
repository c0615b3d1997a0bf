"""Attention of new tokens: rows whose scores are all -infinity have output 0 and LSE -infinity, by either form of the call."""
import pytest
import torch

from test_gpu_chunk import Case, kvp  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.mark.parametrize("lens", [[80], [5, 16, 17, 1], [20000], [3000] * 3 + [10] * 40, [64] * 200])
@pytest.mark.parametrize("one_each", [True, False])
@pytest.mark.parametrize("dh,window,sinks", [(64, 0, 0), (128, 0, 0), (128, 100, 5)])
def test_scores_that_are_all_minus_infinity(kvp, dh, window, sinks, one_each, lens):
    """Of every second sequence; the others' are finite.  Whole units, and units cut into shares."""
    c = Case(kvp, [0, 0], lens, [1] * len(lens), 2, 1, dh, 16, 16, window, sinks, one_each=one_each, freed=False)
    for q in c.q:
        q.copy_(q.abs() + 0.1)
    finite = c.run()
    for b in range(0, len(lens), 2):
        c.pools[0][0][c.bt[b, :-(-lens[b] // 16)].long().cuda()] = -INF
    o, lse = c.run()
    for l in range(2):
        assert (o[l][::2] == 0).all() and (lse[l][::2] == -INF).all()
        assert torch.equal(o[l][1::2], finite[0][l][1::2]) and torch.equal(lse[l][1::2], finite[1][l][1::2])


@pytest.mark.parametrize("one_each", [True, False])
def test_some_scores_that_are_minus_infinity(kvp, one_each):
    """Whole granules and shares of them, in front, in the middle and at the end: those tokens have no part."""
    for lens, dead in (([20000], slice(0, 900)), ([20000], slice(300, 1100)), ([20000], slice(700, 1250)), ([100], slice(0, 3)), ([100], slice(2, 7))):
        c = Case(kvp, [0], lens, [1], 2, 1, 128, 16, 16, one_each=one_each, freed=False)
        c.q[0].copy_(c.q[0].abs() + 0.1)
        pages = c.bt[0, dead].long().cuda()
        c.pools[0][0][pages] = -INF
        o, lse = c.run()
        k, v = c.keys(0, lens[0], 0)
        x = torch.einsum("hd,nd->hn", c.q[0][0].double(), k[0]) * 128 ** -0.5      # (-infinity where the keys are)
        p = torch.softmax(x, -1)
        assert torch.isfinite(o[0]).all() and torch.isfinite(lse[0]).all()
        # sums of 128 products of numbers around 1: 2^-16 of their magnitudes (about 128) at the most in a score, twice that in a weight;
        # P in bf16 2^-8 of sum p |v|, and 2^-8 of the output
        ds = 2.0 ** -16 * (c.q[0][0].double().abs().sum(-1) * k[0][torch.isfinite(k[0])].abs().max() * 128 ** -0.5).max()
        a = p @ v[0].abs()
        assert ((o[0][0].double() - p @ v[0]).abs() <= a * (2.0 ** -8 + 2.0 ** -13 + 2 * ds) + 2.0 ** -8 * (p @ v[0]).abs()).all()
        want = torch.logsumexp(x, -1)
        assert ((lse[0][0].double() - want).abs() <= ds + 2.0 ** -20 * (1 + want.abs())).all()
