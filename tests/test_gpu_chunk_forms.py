"""Attention of new tokens in the forms that a serving program mixes: single tokens in ranges of layers, in captured graphs that share a
workspace, on streams side by side, over far pages and large ones; numbers that the kernel ahead is still writing; the most tokens."""
import numpy as np
import pytest
import torch

from ahead import Ahead
from test_gpu_chunk import Case, kvp  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("window,sinks", [(0, 0), (60, 5)])
@pytest.mark.parametrize("begin,end", [(0, 1), (1, 2), (1, 4), (2, 3), (3, 4), (0, 4)])
def test_layer_ranges_of_single_tokens(kvp, begin, end, window, sinks, bits):
    c = Case(kvp, [0, 0, 2, 0], [900, 40, 0, 17], [1, 1, 0, 1], 8, 2, 64, 16, bits, window, sinks, one_each=True)
    o, lse = c.run(layer_begin=begin, layer_end=end)
    c.check(o, lse, layers=range(begin, end))
    for l in set(range(4)) - set(range(begin, end)):
        assert torch.isnan(o[l]).all() and torch.isnan(lse[l]).all()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("window", [0, 300])
@pytest.mark.parametrize("lens", [[3000, 40, 0, 700], [20 + 9 * i for i in range(70)]])
def test_graphs_of_single_tokens_that_share_a_workspace(kvp, lens, window, bits):
    one = [min(n, 1) for n in lens]
    cases = [Case(kvp, [0, 0, 2], lens, one, 8, 2, 128, 16, bits, window, 4 if window else 0, seed=s, columns=60, one_each=True, freed=False) for s in (91, 92)]
    for c in cases:                                           # (the lengths change: what lies behind or before may be seen)
        for x in c.pools[0] + c.pools[1]:
            x.copy_(torch.randn(x.shape, device="cuda").to(x.dtype))
        for x in c.scales[0] + c.scales[1]:
            x.fill_(121)
    (oc, lc, ws), (od, ld, _) = cases[0].outputs(), cases[1].outputs()
    outs, graphs = [(oc, lc), (od, ld)], []
    for c, (o, l) in zip(cases, outs):
        c.call(o, l, ws)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.call(o, l, ws)
        graphs.append(g)
    for turn in range(4):
        for c, g, (o, l) in zip(cases, graphs, outs):
            c.lens = [max(0, n - 13 * turn * (i % 3)) for i, n in enumerate(lens)]
            for t in o + l:
                t.fill_(float("nan"))
            c.lengths.copy_(torch.tensor(c.lens, dtype=torch.int32))
            g.replay()
        for c, (o, l) in zip(cases, outs):
            c.check(o, l)


def test_single_tokens_on_streams_side_by_side(kvp):
    forms = [(16, 0, True), (8, 0, True), (16, 200, True), (8, 200, True), (16, 200, False), (8, 0, False)]
    cases = [Case(kvp, [0, 0], [6000, 900, 3], [1, 1, 1] if one else [9, 40, 3], 8, 2, 128, 16, bits, window, 3 if window else 0, seed=90 + i, one_each=one)
             for i, (bits, window, one) in enumerate(forms)]
    outs, streams = [c.outputs() for c in cases], [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(6):
        for c, (o, lse, ws), s in zip(cases, outs, streams):
            with torch.cuda.stream(s):
                c.call(o, lse, ws)
    torch.cuda.synchronize()
    for c, (o, lse, _) in zip(cases, outs):
        c.check(o, lse)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
def test_queries_of_single_tokens_that_are_not_finite(kvp, bits, what):
    """They reach their own row and no other: NaN, but for scores that are all -infinity."""
    for lens in ([400, 90, 17], [9000, 3]):
        c = Case(kvp, [0, 0], lens, [1] * len(lens), 4, 2, 64, 16, bits, one_each=True)
        for b, head in ((0, 0), (1, 3), (len(lens) - 1, 2)):
            c.q[1][b, head, (b * 5 + head) % 64] = what
        o, lse = c.run()
        hit = ~torch.isfinite(c.q[1].float()).all(-1)
        for b, head in hit.nonzero().tolist():
            x = what * c.keys(b, lens[b], 0)[0][head // 2, :, (b * 5 + head) % 64]
            if (x == -float("inf")).all():
                assert (o[1][b, head] == 0).all() and lse[1][b, head] == -float("inf")
            else:
                assert torch.isnan(o[1][b, head]).all() and torch.isnan(lse[1][b, head])
        c.q[1][hit] = 0.5
        for l in range(2):
            ro, rl, to, tl = c.exact(l)
            fine = ~hit if l else torch.ones_like(hit)
            assert ((o[l].double() - ro).abs() <= to)[fine].all() and ((lse[l].double() - rl).abs() <= tl)[fine].all()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("page", [144, 1024, 4096])
@pytest.mark.parametrize("one_each", [True, False])
def test_large_pages(kvp, page, one_each, bits):
    for window, sinks in ((0, 0), (500, 9)):
        c = Case(kvp, [0, 0], [5000, 1, 4096, 1023], [1] * 4 if one_each else [70, 1, 130, 0], 8, 2, 64, page, bits, window, sinks, one_each=one_each)
        c.check(*c.run())


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("one_each", [True, False])
def test_far_pages(kvp, one_each, bits):
    """Numbers beyond 2^32 bytes of a pool."""
    page, Hkv, dh, n_pages = 128, 8, 128, 18000 if bits == 16 else 34000
    if torch.cuda.mem_get_info()[0] < 20e9:
        pytest.skip("needs 20 GB")
    c = Case(kvp, [0], [500, 200], [1, 1] if one_each else [9, 200], 16, 8, dh, page, bits, freed=False)
    far = [n_pages - 1 - 3 * i for i in range(int((c.bt >= 0).sum()))]
    table, old = c.bt.clone(), c.bt[c.bt >= 0].tolist()
    table[c.bt >= 0] = torch.tensor(far, dtype=torch.int32)
    for held in (c.pools, c.scales):
        for i in range(2):
            if held[i]:
                big = torch.empty((n_pages,) + held[i][0].shape[1:], dtype=held[i][0].dtype, device="cuda")
                big.view(torch.uint8)[far] = held[i][0].view(torch.uint8)[old]
                held[i][0] = big
    c.bt, c.table, c.lists = table, table.cuda(), dict(k=[c.pools[0][0]], v=[c.pools[1][0]])
    if bits == 8:
        c.kw.update(k_scale=[c.scales[0][0]], v_scale=[c.scales[1][0]])
    c.desc.n_pages = n_pages
    c.check(*c.run())


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("window", [0, 100])
@pytest.mark.parametrize("B,one", [(3, True), (70, True), (3, False), (40, False)])
def test_numbers_that_a_kernel_of_the_library_writes(kvp, B, one, window, bits):
    """Lengths and first rows that the kernel ahead is still writing when this one comes up: what it writes counts."""
    r = np.random.default_rng(B)
    new = [1] * B if one else [128 + int(x) for x in r.integers(0, 40, B)]
    most = [700 + int(x) for x in r.integers(0, 300, B)]
    c = Case(kvp, [0, 0], most, new, 4, 2, 64, 16, bits, window, 5 if window else 0, one_each=one, freed=False)
    for x in c.pools[0] + c.pools[1]:
        x.copy_(torch.randn(x.shape, device="cuda").to(x.dtype))
    for x in c.scales[0] + c.scales[1]:
        x.fill_(121)
    lens = [most, [n - int(x) for n, x in zip(most, r.integers(1, 400, B))]]
    lens[1][B // 2] = 0 if one else 200
    lists = [[torch.tensor(x, dtype=torch.int32)] + ([] if one else [c.first.cpu()]) for x in lens]
    ahead = Ahead(kvp, *lists)
    runs = [c.outputs() for _ in range(8)]
    torch.cuda.synchronize()
    for i, (o, lse, ws) in enumerate(runs):
        ahead.write(i)
        c.lengths = ahead.views[0]
        c.call(o, lse, ws, **({} if one else {"first": ahead.views[1]}))
    assert kvp.device_status() == kvp.OK
    for i, (o, lse, _) in enumerate(runs):
        c.lens = lens[i % 2]
        if one:
            c.first_host = list(range(B + 1))
        c.check(o, lse)


def test_the_most_tokens(kvp):
    """2^24 - 1 rows of one sequence under a window: the rows at both ends and around 2^23 against the window's tokens in 64 bits."""
    T, page, window, dh = (1 << 24) - 1, 1024, 50, 64
    if torch.cuda.mem_get_info()[0] < 24e9:
        pytest.skip("needs 24 GB")
    n_pages = (T + page - 1) // page
    g = torch.Generator(device="cuda").manual_seed(5)
    normal = lambda *s: torch.randn(*s, dtype=torch.bfloat16, device="cuda", generator=g)
    k, v, q = normal(n_pages, 1, page, dh), normal(n_pages, 1, page, dh), normal(T, 1, dh)
    table = torch.randperm(n_pages, generator=torch.Generator().manual_seed(6)).int().view(1, -1).cuda()
    o, lse = torch.full_like(q, float("nan")), torch.full((T, 1), float("nan"), device="cuda")
    desc = kvp.DecodeDesc(1, 1, 1, 1, dh, page, n_pages, n_pages, 0, kvp.BF16)
    ws = torch.empty(kvp.attn_chunk_workspace_bytes(desc, [0], T), dtype=torch.uint8, device="cuda")
    kvp.attn_chunk(desc, [0], [q], [k], [v], table, torch.tensor([T], dtype=torch.int32, device="cuda"), [o], [lse], ws,
                   first=torch.tensor([0, T], dtype=torch.int32, device="cuda"), window=window)
    assert torch.isfinite(o).all() and torch.isfinite(lse).all() and kvp.device_status() == kvp.OK
    for at in (0, 1 << 23, T - 300):
        pos = torch.arange(at, at + 300, device="cuda")
        j = torch.arange(max(0, at - window), at + 300, device="cuda")
        kk, vv = (x[table[0, j // page].long(), 0, j % page].double() for x in (k, v))
        seen = (j <= pos[:, None]) & (j > pos[:, None] - window)
        qq = q[pos, 0].double()
        x = torch.where(seen, qq @ kk.T * dh ** -0.5, -float("inf"))
        ds = 2.0 ** -16 * torch.where(seen, qq.abs() @ kk.abs().T * dh ** -0.5, 0.0).amax(-1, keepdim=True)
        p = torch.softmax(x, -1)
        want = p @ vv
        assert ((o[pos, 0].double() - want).abs() <= (p @ vv.abs()) * (2.0 ** -8 + 2.0 ** -13 + 2 * ds) + 2.0 ** -8 * want.abs()).all()
        lw = torch.logsumexp(x, -1)
        assert ((lse[pos, 0].double() - lw).abs() <= ds[:, 0] + 2.0 ** -20 * (1 + lw.abs())).all()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("one_each", [True, False])
@pytest.mark.parametrize("window", [0, 5000])
def test_keys_that_are_not_numbers_over_whole_shares(kvp, window, one_each, bits):
    """NaN in K of so many tokens that whole shares of a long unit have nothing else."""
    for dead in (slice(0, 700), slice(300, 1200), slice(1100, 1250), slice(0, 1250)):
        c = Case(kvp, [0], [20000, 50], [1, 1], 2, 1, 128, 16, bits, window, one_each=one_each, freed=False)
        pages = c.bt[0, dead].long().cuda()
        c.pools[0][0].view(torch.uint8)[pages] = 0x7f if bits == 8 else 0xff
        o, lse = c.run()
        sees = not window or dead.stop * 16 > 20000 - window
        assert torch.isnan(o[0][0]).all() == sees and torch.isnan(lse[0][0]).all() == sees, dead
        assert torch.isfinite(o[0][1]).all() and torch.isfinite(lse[0][1]).all()
