"""Attention of new tokens where numbers, rows and sequences are at the edges of what the kernel takes apart."""
import pytest
import torch

from test_gpu_chunk import Case, kvp  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("new", [1, 7, 130])
def test_every_code(kvp, dh, new):
    """All finite codes of the 8-bit cache, subnormal ones among them, in every column of V and in K; the steps with masks and without."""
    c = Case(kvp, [0], [600], [new], 2, 1, dh, 16, 8, freed=False)
    codes = torch.tensor([i for i in range(256) if i & 0x7f != 0x7f], dtype=torch.uint8, device="cuda")
    for i, pool in enumerate((c.pools[0][0], c.pools[1][0])):
        at = torch.arange(pool.numel(), device="cuda")
        pool.view(torch.uint8).copy_(codes[(at * (7 + 4 * i) + at // dh) % len(codes)].view(pool.shape))
        c.scales[i][0].fill_(118 + i)
    c.check(*c.run())


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dh", [64, 128])
def test_queries_of_any_size(kvp, dh, bits):
    """Elements of a row down to 2^-40 of the largest, in any column; K of magnitudes between 1/2 and 1.  What the row's largest drowns in
    the 8-bit cache's products, 2^-25 of it for each of up to 128 columns, is 2^-18 of it and so below 2^-17 of sum |q k|, which is
    half of it at least: half of what is allowed for anyway."""
    c = Case(kvp, [0], [500], [90], 4, 2, dh, 16, bits, freed=False)
    g = torch.Generator().manual_seed(3)
    q = torch.randn(c.q[0].shape, generator=g) * torch.exp2(-torch.randint(0, 40, c.q[0].shape, generator=g).float())
    c.q[0].copy_(q)
    k = (torch.rand(c.pools[0][0].shape, generator=g) / 2 + 0.5) * torch.randint(0, 2, c.pools[0][0].shape, generator=g).mul(2).sub(1)
    if bits == 8:
        c.scales[0][0].fill_(127)
    c.pools[0][0].copy_(k.to(c.pools[0][0].dtype))
    c.check(*c.run())


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
def test_queries_that_are_not_finite(kvp, bits, what):
    """They reach their own row and no other."""
    c = Case(kvp, [0, 0], [400, 90], [150, 3], 4, 2, 64, 16, bits)
    want = c.run()
    for row, head in ((0, 0), (3, 1), (77, 2), (149, 3), (150, 0), (152, 2)):
        c.q[1][row, head, (row * 5) % 64] = what
    o, lse = c.run()
    hit = ~torch.isfinite(c.q[1].float()).all(-1)
    assert torch.isnan(o[1][hit]).all() and torch.isnan(lse[1][hit]).all()
    assert torch.equal(o[1][~hit], want[0][1][~hit]) and torch.equal(lse[1][~hit], want[1][1][~hit])
    assert torch.equal(o[0], want[0][0]) and torch.equal(lse[0], want[1][0])


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("new", [8, 15, 16, 17, 24, 31, 32, 33, 47, 48, 49, 63, 64, 65])
def test_rows_around_halves_of_tiles(kvp, new, bits):
    """4 rows a token: units of a quarter of a tile to two tiles, alone and cut into many shares, of one step and of many."""
    for lens in ([new], [3000], [64 + new, 700]):
        c = Case(kvp, [0], lens, [new] * len(lens), 4, 1, 128 if new % 2 else 64, 16, bits)
        c.check(*c.run())


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("donor,lens,new,Hq,Hkv", [
    ([0, 0], [1843, 181, 1452, 2063, 1986], [539, 118, 849, 226, 684], 128, 16),
    ([0], [2371, 1671, 830, 2609, 634, 1004, 1534, 582, 2695, 1720, 1016], [836, 513, 746, 638, 487, 332, 888, 119, 865, 69, 491], 256, 16),
    ([0, 0, 0, 0], [1571, 545, 314, 2191, 480], [555, 227, 125, 418, 369], 256, 16),
    ([0, 0], [2079, 2204, 1238, 567, 2314, 708], [898, 579, 482, 73, 604, 263], 128, 16),
])
def test_units_over_shares_without_places(kvp, donor, lens, new, Hq, Hkv, bits):
    """A unit goes from a share over one that has been left nothing, the second of its shares, into a third."""
    c = Case(kvp, donor, lens, new, Hq, Hkv, 64, 16, bits)
    o, lse = c.run()
    c.check(o, lse, layers=[0, len(donor) - 1])


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("one_each", [True, False])
def test_windows_of_any_size(kvp, bits, one_each):
    """A window that reaches behind every token is none; more first tokens than there are tokens."""
    new = [1, 1, 0, 1] if one_each else [200, 3, 0, 64]
    c = Case(kvp, [0, 0], [700, 3, 0, 64], new, 8, 2, 64, 16, bits, one_each=one_each, freed=False)
    want = c.run()
    most = (1 << 31) - 1
    for window, sinks in ((most, 0), (most, most), (c.desc.max_pages * 16, 7), (5, most), (1, c.desc.max_pages * 16)):
        o, lse = c.run(window=window, sinks=sinks)
        for x, y in zip(o + lse, want[0] + want[1]):
            some = ~torch.isnan(y)
            assert torch.equal(torch.isnan(x), torch.isnan(y))
            if window >= c.desc.max_pages * 16:
                assert torch.equal(x[some], y[some])
    c.window, c.sinks = 5, most
    c.check(*c.run(window=5, sinks=most))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("B", [33, 300, 1 << 14])
def test_many_sequences(kvp, B, bits):
    """Up to as many as a call takes, of a few tokens, some without rows."""
    new = [(i * 7 + i // 3) % 3 for i in range(B)]
    c = Case(kvp, [0], [n + (i * 5) % 9 for i, n in enumerate(new)], new, 2, 1, 64, 16, bits)
    o, lse = c.run()
    if B <= 300:
        return c.check(o, lse)
    rows = [r for r, _, _ in c.rows()]
    assert torch.isfinite(o[0][rows]).all() and torch.isfinite(lse[0][rows]).all()
    # each sequence by itself: a call of 64 of them
    for b0 in (0, 5000, B - 64):
        r0, r1 = c.first_host[b0], c.first_host[b0 + 64]
        part = kvp.DecodeDesc(1, 64, 2, 1, 64, 16, c.desc.max_pages, c.desc.n_pages, 0, kvp.BF16)
        q, po, pl = c.q[0][r0:r1].contiguous(), torch.empty_like(o[0][r0:r1]), torch.empty_like(lse[0][r0:r1])
        ws = torch.empty(kvp.attn_chunk_workspace_bytes(part, [0], r1 - r0), dtype=torch.uint8, device="cuda")
        kvp.attn_chunk(part, [0], [q], c.lists["k"], c.lists["v"], c.table[b0:b0 + 64].contiguous(), c.lengths[b0:b0 + 64].contiguous(), [po], [pl], ws,
                       **{**c.kw, "first": (c.first[b0:b0 + 65] - r0).contiguous()})
        assert torch.equal(po, o[0][r0:r1]) and torch.equal(pl, lse[0][r0:r1])


def test_two_streams_at_once(kvp):
    """Calls of both caches run beside one another, each with its own workspace."""
    cases = [Case(kvp, [0, 0], [6000, 900], [40, 600], 8, 2, 128, 16, bits, seed=s) for s, bits in ((91, 16), (92, 8), (93, 16), (94, 8))]
    outs, streams = [c.outputs() for c in cases], [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, (o, lse, ws), s in zip(cases, outs, streams):
            with torch.cuda.stream(s):
                c.call(o, lse, ws)
    torch.cuda.synchronize()
    for c, (o, lse, _) in zip(cases, outs):
        c.check(o, lse)
