"""Decode attention over the cache held in 8 bits, against attention in 64 bits over the numbers that the cache stands for."""
import numpy as np
import pytest
import torch

from ahead import Ahead
from guard import Guarded
from paper_2608_15943_b200 import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvp():
    from paper_2608_15943_b200 import kvp as mod
    return mod


def cache8(lens, n_own, Hkv, dh, page, seed, lo=117, hi=124, poison=True, columns=1):
    """Pools [n_own][n_pages, Hkv, page, dh] of e4m3, scale bytes lo..hi-1, scattered pages; what lies behind a sequence is NaN."""
    need = [(n + page - 1) // page for n in lens]
    n_pages, max_pages = sum(need) + 2, max(need + [0]) + columns
    g = torch.Generator().manual_seed(seed)
    order = torch.randperm(n_pages, generator=g).int()
    bt, at = torch.full((len(lens), max_pages), int(order[-1]), dtype=torch.int32), 0
    for b, k in enumerate(need):
        bt[b, :k] = order[at:at + k]
        at += k
    pools, scales = [], []
    for i in range(2):
        pools.append([(synth.normal((n_pages, Hkv, page, dh), seed, synth.tid(7 + i, l), 1.0, "cuda") * 64).to(torch.float8_e4m3fn) for l in range(n_own)])
        scales.append([torch.randint(lo, hi, (n_pages, Hkv, page // 16), generator=g, dtype=torch.uint8).cuda() for _ in range(n_own)])
    if poison:
        used = torch.zeros(n_pages, page, dtype=torch.bool)
        for b, n in enumerate(lens):
            for i in range(need[b]):
                used[bt[b, i].long(), :min(page, n - i * page)] = True
        bad = (~used).cuda()
        for p in pools[0] + pools[1]:
            p.view(torch.uint8).transpose(1, 2)[bad] = 0x7f
        dead = (~used.view(n_pages, -1, 16).any(-1)).cuda()
        for s in scales[0] + scales[1]:
            s.transpose(1, 2)[dead] = 255
    return pools, scales, bt


def exact(q, pools, scales, bt, lens, page, scale, layer):
    """[B, Hq, dh], [B, Hq] in 64 bits, and what the kernel may be off by:
    scores: products of the tensor cores' sums of up to 128 terms, each rounded down by up to 2^-23 of the sum of magnitudes, in two
      chains: 64 * 2^-23 of sum |q k|, doubled for the factor, the difference to M and ex2 (2^-22 of scores that sum bounds);
    P: half a step of f16, 2^-11; O: fp32 sums (2^-13 covers 2^10 roundings of 2^-23); bf16: 2^-8 of the value;
    LSE: the scores' error and fp32."""
    B, Hq, dh = q.shape
    Hkv = pools[0][layer].shape[1]
    o, lse = torch.zeros(B, Hq, dh, dtype=torch.float64, device="cuda"), torch.full((B, Hq), -float("inf"), dtype=torch.float64, device="cuda")
    tol_o, tol_l = torch.zeros_like(o), torch.zeros(B, Hq, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        if n <= 0:
            continue
        pages = bt[b, :(n + page - 1) // page].long().cuda()
        kv = []
        for i in range(2):
            x = pools[i][layer][pages].double().unflatten(2, (-1, 16))
            x = x * torch.exp2(scales[i][layer][pages].double().clamp(27, 247) - 127)[..., None, None]
            kv.append(x.flatten(2, 3).transpose(0, 1).flatten(1, 2)[:, :n])
        qb = q[b].double().view(Hkv, Hq // Hkv, dh)
        x = torch.einsum("hgd,hnd->hgn", qb, kv[0]) * scale
        size = torch.einsum("hgd,hnd->hgn", qb.abs(), kv[0].abs()).amax(-1, keepdim=True) * scale
        p = torch.softmax(x, -1)
        o[b] = torch.einsum("hgn,hnd->hgd", p, kv[1]).reshape(Hq, dh)
        lse[b] = torch.logsumexp(x, -1).reshape(Hq)
        ds = 2.0 ** -16 * size
        a = torch.einsum("hgn,hnd->hgd", p, kv[1].abs())
        tol_o[b] = (a * (2.0 ** -11 + 2.0 ** -13 + 2 * ds)).reshape(Hq, dh) + 2.0 ** -8 * o[b].abs()
        tol_l[b] = ds.reshape(Hq) + 2.0 ** -20 * (1 + lse[b].abs())
    return o, lse, tol_o, tol_l


class Case:
    def __init__(self, kvp, donor, lens, Hq, Hkv, dh, page, io="bf16", splits=0, seed=81, q_gain=1.0, **cache):
        self.kvp, self.donor, self.lens, self.page = kvp, donor, lens, page
        L, B = len(donor), len(lens)
        self.own = [l for l in range(L) if donor[l] == l]
        self.pools, self.scales, self.bt = cache8(lens, len(self.own), Hkv, dh, page, seed, **cache)
        at = lambda xs: [xs[self.own.index(l)] if l in self.own else None for l in range(L)]
        self.lists = [at(self.pools[0]), at(self.pools[1]), at(self.scales[0]), at(self.scales[1])]
        self.dtype = torch.float32 if io == "f32" else torch.bfloat16
        self.desc = kvp.DecodeDesc(L, B, Hq, Hkv, dh, page, self.bt.shape[1], self.pools[0][0].shape[0], splits, kvp.F32 if io == "f32" else kvp.BF16)
        self.q = [(synth.normal((B, Hq, dh), seed, synth.tid(6, l), 1.0, "cuda") * q_gain).to(self.dtype) for l in range(L)]
        self.table, self.lengths = self.bt.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")

    def outputs(self, guard=None):
        g = guard or Guarded()
        L, B = len(self.donor), len(self.lens)
        o = [g.empty(self.q[0].shape, self.dtype, float("nan")) for _ in range(L)]
        lse = [g.empty((B, self.desc.Hq), torch.float32, float("nan")) for _ in range(L)]
        ws = g.empty((max(1, self.kvp.decode8_workspace_bytes(self.desc, self.donor)),), torch.uint8, 0xff)
        return o, lse, ws

    def run(self, scale=0.0, **kw):
        g = Guarded()
        o, lse, ws = self.outputs(g)
        self.kvp.decode8(self.desc, self.donor, self.q, *self.lists, self.table, self.lengths, o, lse, ws, scale, **kw)
        g.check()
        assert self.kvp.device_status() == self.kvp.OK
        return o, lse

    def check(self, o, lse, scale=0.0, layers=None):
        dh = self.q[0].shape[-1]
        cap = self.desc.max_pages * self.page
        lens = [min(max(n, 0), cap) for n in self.lens]
        for l in range(len(self.donor)) if layers is None else layers:
            ro, rl, to, tl = exact(self.q[l], self.pools, self.scales, self.bt, lens, self.page, scale or dh ** -0.5, self.own.index(self.donor[l]))
            some = torch.tensor(lens, device="cuda") > 0
            assert torch.isfinite(o[l]).all()
            assert ((o[l].double() - ro).abs() <= to).all(), ((o[l].double() - ro).abs() - to).max()
            assert ((lse[l].double() - rl).abs() <= tl)[some].all()
            assert (o[l][~some] == 0).all() and (lse[l][~some] == -float("inf")).all()


SHAPES = [
    ([0], [1], 1, 1, 128, 16),                                # one token
    ([0], [20000], 4, 1, 128, 128),                           # one unit over many blocks
    ([0], [9001], 16, 1, 64, 64),                             # the same at dh 64, all 16 rows
    ([0, 0], [17 + 13 * b for b in range(40)], 8, 2, 128, 16),
    ([0, 1, 2], [16] * 33, 2, 2, 64, 32),                     # whole units of one granule
    ([0, 1], [1100, 3, 900], 4, 4, 128, 16),
    ([0, 0, 0, 0], [640, 1, 333], 12, 2, 128, 48),            # 12-row passes of uneven groups
    ([0, 0, 0, 3, 3, 5], [700, 64, 15, 0, 5], 20, 4, 128, 64),   # 15 rows, 10 and 5
    ([0, 0], [0, 0, 0], 4, 2, 64, 16),                        # nothing at all
    ([0], [0] * 5 + [3000] + [0] * 30 + [1], 6, 2, 128, 128), # empty places around a long sequence
    ([0, 1], [0, 4000, 0, 0, 4000, 17, 0], 3, 1, 64, 32),
    ([0], [130, 1, 31], 9, 1, 128, 16),                       # one row in the second n-block
]


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("donor,lens,Hq,Hkv,dh,page", SHAPES)
def test_against_64_bits(kvp, donor, lens, Hq, Hkv, dh, page, io):
    c = Case(kvp, donor, lens, Hq, Hkv, dh, page, io)
    c.check(*c.run())


MANY = [
    ([0, 0], 128, 8, 8, 128, 16, 90),                         # units for single warps, several each: rows of one n-block
    ([0, 0, 2], 160, 36, 4, 64, 32, 150),                     # the same with 9 rows: two n-blocks
    ([0, 0], 80, 12, 6, 128, 64, 200),                        # two warps a unit
    ([0], 110, 72, 6, 64, 48, 130),                           # the same with 12 rows
    ([0], 35, 32, 16, 128, 128, 300),
]


@pytest.mark.parametrize("donor,B,Hq,Hkv,dh,page,most", MANY)
def test_many_short_sequences(kvp, donor, B, Hq, Hkv, dh, page, most):
    """Whole units dealt out to one, two or four warps; empty places, lengths of one and of whole blocks among them."""
    r = np.random.default_rng(B)
    lens = [int(x) for x in r.integers(0, most, B)]
    lens[::9], lens[1::11], lens[2::13] = [0] * len(lens[::9]), [1] * len(lens[1::11]), [most // 16 * 16] * len(lens[2::13])
    c = Case(kvp, donor, lens, Hq, Hkv, dh, page)
    o, lse = c.run()
    c.check(o, lse)
    again, lse2 = c.run()
    assert all(torch.equal(x, y) for x, y in zip(o + lse, again + lse2))


BY_LENGTH = [
    ([0, 1], 32, 8, 8, 128, 16, (1, 700)),                    # between one and two units a block: teams of four, two and one
    ([0, 1, 2, 3], 31, 16, 16, 64, 32, (0, 300)),             # between two and four
    ([0, 1], 128, 8, 2, 128, 48, (0, 400)),                   # the longest batch that is looked at whole
    ([0, 1, 1], 127, 4, 4, 64, 16, (10, 900)),
    ([0, 1], 129, 8, 2, 128, 16, (0, 200)),                   # and one beyond it
    ([0, 0, 0, 0], 100, 16, 4, 128, 32, (0, 500)),            # sixteen rows
    ([0, 1, 2], 50, 8, 4, 128, 16, (200, 200)),               # nobody longer than the others
    ([0, 1, 2], 50, 8, 4, 64, 16, (0, 0)),
    ([0, 1, 2, 3], 97, 4, 4, 128, 16, (1, 33)),               # one step or two
]


@pytest.mark.parametrize("columns", [1, 2000])                # with the wide table the lengths alone say that units are short
@pytest.mark.parametrize("donor,B,Hq,Hkv,dh,page,lens", BY_LENGTH)
def test_teams_go_by_the_length(kvp, donor, B, Hq, Hkv, dh, page, lens, columns):
    r = np.random.default_rng(B)
    lens = [int(x) for x in r.integers(lens[0], lens[1] + 1, B)]
    c = Case(kvp, donor, lens, Hq, Hkv, dh, page, columns=columns)
    o, lse = c.run()
    c.check(o, lse)
    again, lse2 = c.run()
    assert all(torch.equal(x, y) for x, y in zip(o + lse, again + lse2))


def test_values_that_are_not_finite(kvp):
    """NaN among the visible keys of a KV head reaches its queries' outputs and LSE and no others; among the values, its element."""
    c = Case(kvp, [0], [500, 40], 4, 2, 128, 16, poison=False)
    p = int(c.bt[0, 7])
    c.pools[0][0].view(torch.uint8)[p, 1, 3, 5] = 0x7f
    c.pools[1][0].view(torch.uint8)[int(c.bt[1, 1]), 0, 2, 9] = 0xff
    o, lse = c.run()
    ro, rl, to, tl = exact(c.q[0], c.pools, c.scales, c.bt, c.lens, 16, 128 ** -0.5, 0)
    bad = torch.zeros(2, 4, 128, dtype=torch.bool, device="cuda")
    bad[0, 2:], bad[1, :2, 9] = True, True
    assert torch.equal(torch.isnan(o[0]), bad) and ((o[0].double() - ro).abs() <= to)[~bad].all()
    assert torch.isnan(lse[0][0, 2:]).all() and torch.isfinite(lse[0][0, :2]).all() and torch.isfinite(lse[0][1]).all()
    c.q[0][1, 0, 0] = float("nan")                            # a query: its own row
    o, lse = c.run()
    assert torch.isnan(o[0][1, 0]).all() and torch.isfinite(o[0][1, 1, :9]).all() and torch.isnan(lse[0][1, 0])


def test_another_device_is_refused_and_the_current_one_serves(kvp):
    if torch.cuda.device_count() < 2:
        pytest.skip("needs a second device")
    c = Case(kvp, [0], [100], 4, 1, 64, 16)
    o, lse, ws = c.outputs()
    with torch.cuda.device(1), pytest.raises(ValueError):
        kvp.decode8(c.desc, c.donor, c.q, *c.lists, c.table, c.lengths, o, lse, ws)


@pytest.mark.parametrize("splits", [1, 3, 8, 70])
@pytest.mark.parametrize("dh", [64, 128])
def test_the_callers_splits(kvp, splits, dh):
    c = Case(kvp, [0, 0], [700, 0, 33, 1, 2049], 8, 2, dh, 32, splits=splits)
    c.check(*c.run())


def test_both_types_agree_and_runs_repeat(kvp):
    for lens in ([4000, 1, 0, 900], [100] * 20):
        a, b = (Case(kvp, [0, 0, 2], lens, 8, 2, 128, 64, io) for io in ("bf16", "f32"))
        (oa, la), (ob, lb), (oc, lc) = a.run(), b.run(), a.run()
        for l in range(3):
            assert torch.equal(oa[l].float(), ob[l]) and torch.equal(la[l], lb[l])
            assert torch.equal(oa[l], oc[l]) and torch.equal(la[l], lc[l])


@pytest.mark.parametrize("begin,end", [(0, 1), (1, 2), (1, 4), (2, 3), (0, 4)])
def test_layer_ranges(kvp, begin, end):
    c = Case(kvp, [0, 0, 2, 0], [900, 40], 8, 2, 64, 16)
    o, lse = c.run(layer_begin=begin, layer_end=end)
    c.check(o, lse, layers=range(begin, end))
    for l in set(range(4)) - set(range(begin, end)):
        assert torch.isnan(o[l]).all() and torch.isnan(lse[l]).all()


def test_more_groups_than_a_launch_takes(kvp):
    donor = list(range(70))
    c = Case(kvp, donor, [40, 0, 100], 2, 1, 64, 16)
    c.check(*c.run())
    donor = [0, 0, 0, 0, 0] + list(range(5, 14))             # more than the small parameter block's, one of them in two passes
    c = Case(kvp, donor, [500, 7], 8, 2, 128, 16)
    c.check(*c.run())


@pytest.mark.parametrize("lens", [[5, -2, 3, 100000], [16] * 40 + [-1, 1 << 30]])
def test_lengths_outside_the_table(kvp, lens):
    """Below zero: as zero.  Above the table: as much as it has."""
    c = Case(kvp, [0], [min(max(n, 0), 64) for n in lens], 4, 2, 128, 16, poison=False, columns=0)
    c.lens = lens
    c.lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    c.check(*c.run())


@pytest.mark.parametrize("scale,gain", [(0.25, 1.0), (3.0, 1.0), (0.0, 2.0 ** -100), (0.0, 40.0), (1e-30, 1e30), (0.0, 0.0)])
def test_scales_of_queries(kvp, scale, gain):
    """Queries far outside f16's range, scores of a few hundred, of nothing."""
    for dh in (64, 128):
        c = Case(kvp, [0], [1000, 77], 4, 1, dh, 16, q_gain=gain)
        c.check(*c.run(scale), scale)


@pytest.mark.parametrize("dh", [64, 128])
def test_scales_of_the_cache_over_many_powers(kvp, dh):
    """Neighbouring blocks of V with scales from 2^-100 to 2^120, their values apart by as much: the sum and the weights have
    references of their own.  K's over a few powers (scores of some hundreds)."""
    c = Case(kvp, [0], [900, 16, 1, 333], 4, 1, dh, 16)
    g = torch.Generator().manual_seed(5)
    c.scales[1][0].copy_(torch.randint(27, 228, c.scales[1][0].shape, generator=g, dtype=torch.uint8))
    c.scales[0][0].copy_(torch.randint(110, 129, c.scales[0][0].shape, generator=g, dtype=torch.uint8))
    o, lse = c.run()
    c.check(o, lse)
    c = Case(kvp, [0], [4096], 4, 1, dh, 16)                  # one block of V that matters, all others of nothing
    c.scales[1][0].fill_(27)
    c.scales[1][0][int(c.bt[0, 77])] = 160
    c.check(*c.run())


@pytest.mark.parametrize("at", [0, 15, 16, 700, 4999])
@pytest.mark.parametrize("dh", [64, 128])
def test_one_score_far_above_the_others(kvp, at, dh):
    page = 16
    c = Case(kvp, [0], [5000], 4, 1, dh, page)
    q = c.q[0]
    q[:, 1:] = q[:, :1]
    p, r = int(c.bt[0, at // page]), at % page
    c.pools[0][0][p, 0, r] = (q[0, 0].float() * 60).clamp(-448, 448).to(torch.float8_e4m3fn)
    c.scales[0][0][p] = 127
    c.check(*c.run())


def test_a_common_offset_of_v_survives(kvp):
    """All of V the same number: the output is that number, however long the sequence (the weights' roundings do not add up to a
    drift: half of a bf16 step and 2^-11)."""
    for lens in ([60000], [3, 1000]):
        c = Case(kvp, [0], lens, 4, 1, 128, 128)
        c.pools[1][0].copy_(torch.full(c.pools[1][0].shape, 96.0).to(torch.float8_e4m3fn))
        c.scales[1][0].fill_(121)
        o, _ = c.run()
        assert ((o[0].float() - 1.5).abs() <= 1.5 * (2.0 ** -8 + 2.0 ** -11)).all()


def test_pages_outside_the_pool_stay_inside(kvp):
    """Table entries that are no page are taken as the nearest one: a wrong answer for that sequence, no read out of the pool."""
    c = Case(kvp, [0], [64, 64], 4, 1, 128, 16, poison=False)
    c.table[0, 1], c.table[0, 2] = -7, 1 << 30
    o, lse = c.run()
    ro, rl, to, tl = exact(c.q[0], c.pools, c.scales, c.bt, c.lens, 16, 128 ** -0.5, 0)
    assert ((o[0].double() - ro).abs() <= to)[1].all() and torch.isfinite(o[0]).all()


@pytest.mark.parametrize("lens", [[3000, 0, 50], [20] * 40])
def test_captured_graphs_share_a_workspace(kvp, lens):
    """Two captured calls with one workspace, replayed in turn and with new lengths, and a call on another stream."""
    c, d = Case(kvp, [0, 0], lens, 8, 2, 128, 16, columns=60), Case(kvp, [0, 0], lens, 8, 2, 128, 16, seed=82, columns=60)
    s = torch.cuda.Stream()
    (oc, lc, ws), (od, ld, _) = c.outputs(), d.outputs()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        kvp.decode8(c.desc, c.donor, c.q, *c.lists, c.table, c.lengths, oc, lc, ws)
    torch.cuda.synchronize()
    c.check(oc, lc)
    graphs = []
    for x, o, l in ((c, oc, lc), (d, od, ld)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            kvp.decode8(x.desc, x.donor, x.q, *x.lists, x.table, x.lengths, o, l, ws)
        graphs.append(g)
    for n in (0, 9):
        for x in (c, d):
            x.lens = [max(y - n, 0) for y in lens]
            x.lengths.copy_(torch.tensor(x.lens, dtype=torch.int32))
        for o, l in ((oc, lc), (od, ld)):
            for t in o + l:
                t.fill_(float("nan"))
        for _ in range(3):
            for g in graphs:
                g.replay()
        torch.cuda.synchronize()
        c.check(oc, lc)
        d.check(od, ld)


def test_lengths_written_by_the_kernel_ahead(kvp):
    """The lengths are looked at before the kernels ahead have finished; what they write counts."""
    for first, second in (([20000], [777]), ([300, 5000, 0], [4000, 0, 129]), ([700] * 33, [0] + [700] * 31 + [8000])):
        longest = [max(a, b) for a, b in zip(first, second)]
        c = Case(kvp, [0], longest, 4, 1, 128, 16, poison=False)
        want = [exact(c.q[0], c.pools, c.scales, c.bt, lens, 16, 128 ** -0.5, 0) for lens in (first, second)]
        on_device = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (first, second)]
        runs = [c.outputs() for _ in range(8)]
        big = torch.zeros(64 << 20, device="cuda")
        for i, (o, lse, ws) in enumerate(runs):
            big.add_(1.0)                                     # keeps the device busy ahead of the copy
            c.lengths.copy_(on_device[i % 2])
            kvp.decode8(c.desc, c.donor, c.q, *c.lists, c.table, c.lengths, o, lse, ws)
        torch.cuda.synchronize()
        for i, (o, lse, _) in enumerate(runs):
            ro, rl, to, tl = want[i % 2]
            assert ((o[0].double() - ro).abs() <= to).all()
            some = torch.isfinite(rl)
            assert ((lse[0].double() - rl).abs() <= tl)[some].all() and (lse[0][~some] == -float("inf")).all()


@pytest.mark.parametrize("B,Hkv", [(30, 16), (100, 8)])
def test_lengths_written_ahead_of_teams(kvp, B, Hkv):
    """The same where the lengths of the whole batch say which team a unit gets."""
    r = np.random.default_rng(B)
    first, second = ([int(x) for x in r.integers(0, 350, B)] for _ in range(2))
    second[0], first[-1] = 700, 650
    c = Case(kvp, [0], [max(a, b) for a, b in zip(first, second)], Hkv, Hkv, 128, 16, poison=False)
    want = [exact(c.q[0], c.pools, c.scales, c.bt, lens, 16, 128 ** -0.5, 0) for lens in (first, second)]
    on_device = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (first, second)]
    runs = [c.outputs() for _ in range(8)]
    big = torch.zeros(64 << 20, device="cuda")
    for i, (o, lse, ws) in enumerate(runs):
        big.add_(1.0)
        c.lengths.copy_(on_device[i % 2])
        kvp.decode8(c.desc, c.donor, c.q, *c.lists, c.table, c.lengths, o, lse, ws)
    torch.cuda.synchronize()
    for i, (o, lse, _) in enumerate(runs):
        ro, rl, to, tl = want[i % 2]
        assert ((o[0].double() - ro).abs() <= to).all()
        some = torch.isfinite(rl)
        assert ((lse[0].double() - rl).abs() <= tl)[some].all() and (lse[0][~some] == -float("inf")).all()


@pytest.mark.parametrize("donor,Hkv,lens", [
    ([0, 1, 2, 3], 8, [28500 + 37 * b for b in range(8)] + [1, 0, 700]),          # one small share a block behind the large one
    ([0, 1, 2, 3], 16, [28500 + 37 * b for b in range(8)] + [1, 0, 700]),         # two
])
def test_shares_of_two_sizes(kvp, donor, Hkv, lens):
    """Lists of six and twelve shares of 160 granules a block: large ones first, and small ones behind them."""
    c = Case(kvp, donor, lens, Hkv, Hkv, 128, 128)
    o, lse = c.run()
    c.check(o, lse)
    again, lse2 = c.run()
    assert all(torch.equal(x, y) for x, y in zip(o + lse, again + lse2))


def test_beyond_32_bits(kvp):
    """A pool of more than 2^32 numbers: the last pages are found."""
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB of device memory")
    Hkv, dh, page = 8, 128, 128
    n_pages = (1 << 32) // (Hkv * dh * page) + 40
    lens = [5 * page + 3, 2 * page]
    pools = [torch.zeros(n_pages, Hkv, page, dh, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.full((n_pages, Hkv, page // 16), 120, dtype=torch.uint8, device="cuda") for _ in range(2)]
    bt = torch.tensor([[n_pages - 1 - i for i in range(6)], [n_pages - 20, 3, 0, 0, 0, 0]], dtype=torch.int32)
    T = sum(lens)
    new = [synth.normal((T, Hkv, dh), 5, i, 1.0, "cuda") for i in range(2)]
    desc = kvp.DecodeDesc(1, 2, 16, Hkv, dh, page, 6, n_pages)
    lengths, table = torch.tensor(lens, dtype=torch.int32, device="cuda"), bt.cuda()
    kvp.cache_append_tokens(desc, [0], [new[0]], [new[1]], [pools[0]], [pools[1]], table, lengths, first=torch.tensor([0, lens[0], T], dtype=torch.int32, device="cuda"),
                            theta=10000.0, k_scale=[scales[0]], v_scale=[scales[1]])
    q = synth.normal((2, 16, dh), 5, 9, 1.0, "cuda")
    o, lse = torch.empty_like(q), torch.empty(2, 16, device="cuda")
    ws = torch.empty(kvp.decode8_workspace_bytes(desc, [0]), dtype=torch.uint8, device="cuda")
    kvp.decode8(desc, [0], [q], [pools[0]], [pools[1]], [scales[0]], [scales[1]], table, lengths, [o], [lse], ws)
    codes = [[p.view(torch.float8_e4m3fn)] for p in pools]
    ro, rl, to, tl = exact(q, codes, [[s] for s in scales], bt, lens, page, dh ** -0.5, 0)
    assert ((o.double() - ro).abs() <= to).all() and ((lse.double() - rl).abs() <= tl).all()
    held = codes[1][0][n_pages - 1, :, 0].double() * torch.exp2(scales[1][n_pages - 1, :, 0].double() - 127)[:, None]
    assert ((held - new[1][0].double()).abs() <= 2.0 ** -4 * new[1][0].double().abs() + 2.0 ** -10 * torch.exp2(scales[1][n_pages - 1, :, 0].double() - 127)[:, None]).all()


def test_a_prompt_then_tokens(kvp):
    """As a serving program runs them: prompts enter the cache, then steps append a token each and attend, donors and consumers; at
    every step against attention in 64 bits over keys rotated in 64 bits and never rounded.  Rounding to e4m3 is at most 2^-4 of a
    number or half the smallest step: scores move by at most ds = 2^-4 sum |q k| scale (q and k rotated in bf16 and fp32 within that),
    outputs by (e^(2 ds) - 1) of the weights and 2^-4 of V.  The bound that is checked is the usual size: those errors are
    independent of another, so that their sums grow as roots: a tenth of the norm."""
    donor, lens, Hq, Hkv, dh, page = [0, 0, 2], [37, 16, 0, 5], 8, 2, 64, 16
    L, B, steps = 3, 4, 20
    total = [n + steps for n in lens]
    need = [(n + page - 1) // page for n in total]
    bt = torch.arange(B * max(need), dtype=torch.int32).view(B, -1).flip(0).contiguous()
    n_pages = bt.numel()
    own = [0, 2]
    new = lambda T, H, seed: [synth.normal((T, H, dh), seed, l, 1.0, "cuda") for l in range(L)]
    u8 = lambda *s: [torch.full(s, 0xff, dtype=torch.uint8, device="cuda") if l in own else None for l in range(L)]
    kc, vc, ks, vs = u8(n_pages, Hkv, page, dh), u8(n_pages, Hkv, page, dh), u8(n_pages, Hkv, 1), u8(n_pages, Hkv, 1)
    desc = kvp.DecodeDesc(L, B, Hq, Hkv, dh, page, bt.shape[1], n_pages)
    table, lengths = bt.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
    first = torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device="cuda")
    k, v = new(sum(lens), Hkv, 91), new(sum(lens), Hkv, 92)
    kvp.cache_append_tokens(desc, donor, k, v, kc, vc, table, lengths, first=first, theta=10000.0, k_scale=ks, v_scale=vs)

    def turn(x, pos):                                         # [n, H, dh]
        a = pos.double()[:, None, None] * 10000.0 ** (-torch.arange(dh // 2, device="cuda", dtype=torch.float64) * 2 / dh)
        z = torch.view_as_complex(x.double().unflatten(-1, (-1, 2))) * torch.polar(torch.ones_like(a), a)
        return torch.view_as_real(z).flatten(-2)
    at = [0] + list(np.cumsum(lens))
    span = [torch.arange(n, device="cuda") for n in lens]
    keys = {l: [turn(k[l][at[b]:at[b + 1]], span[b]) for b in range(B)] for l in own}
    values = {l: [v[l][at[b]:at[b + 1]].double() for b in range(B)] for l in own}
    ws = torch.empty(kvp.decode8_workspace_bytes(desc, donor), dtype=torch.uint8, device="cuda")
    for step in range(steps):
        lengths += 1
        q, k, v = new(B, Hq, 100 + step), new(B, Hkv, 200 + step), new(B, Hkv, 300 + step)
        q_out, o = [torch.empty_like(x) for x in q], [torch.empty_like(x) for x in q]
        lse = [torch.empty(B, Hq, device="cuda") for _ in range(L)]
        kvp.cache_append_tokens(desc, donor, k, v, kc, vc, table, lengths, theta=10000.0, q=q, q_out=q_out, k_scale=ks, v_scale=vs)
        kvp.decode8(desc, donor, q_out, kc, vc, ks, vs, table, lengths, o, lse, ws)
        for l in own:
            for b in range(B):
                pos = lengths[b:b + 1] - 1
                keys[l][b] = torch.cat([keys[l][b], turn(k[l][b:b + 1], pos)])
                values[l][b] = torch.cat([values[l][b], v[l][b:b + 1].double()])
        for l in range(L):
            want = torch.empty(B, Hq, dh, dtype=torch.float64, device="cuda")
            for b in range(B):
                x = torch.einsum("hgd,nhd->hgn", turn(q[l][b:b + 1], lengths[b:b + 1] - 1)[0].view(Hkv, Hq // Hkv, dh), keys[donor[l]][b]) * dh ** -0.5
                want[b] = torch.einsum("hgn,nhd->hgd", torch.softmax(x, -1), values[donor[l]][b]).reshape(Hq, dh)
            assert (o[l].double() - want).norm() <= 0.1 * want.norm(), (step, l)
    assert kvp.device_status() == kvp.OK


def test_drafted_tokens_as_a_batch(kvp):
    """Entries that share their pages: each token of a run sees what lies before it, as calls of their own would."""
    runs, old, Hq, Hkv, dh, page = [4, 1, 3], [30, 100, 13], 8, 2, 128, 16
    c = Case(kvp, [0, 0], [n + o for n, o in zip(runs, old)], Hq, Hkv, dh, page)
    of = [b for b, n in enumerate(runs) for _ in range(n)]
    lens = [o + 1 + i for n, o in zip(runs, old) for i in range(n)]
    d = Case(kvp, [0, 0], [1] * len(of), Hq, Hkv, dh, page)
    d.pools, d.scales, d.bt, d.lens = c.pools, c.scales, c.bt[of].contiguous(), lens
    d.lists = c.lists
    d.table, d.lengths = d.bt.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
    d.desc = kvp.DecodeDesc(2, len(of), Hq, Hkv, dh, page, d.bt.shape[1], c.desc.n_pages)
    d.check(*d.run())


def test_tensors_of_the_host_are_refused(kvp):
    c = Case(kvp, [0], [16, 3], 4, 2, 64, 16)
    o, lse, ws = c.outputs()
    for at, x in ((0, [c.q[0].cpu()]), (3, [c.lists[2][0].cpu()]), (6, c.lengths.cpu()), (9, ws.cpu())):
        args = [c.q, *c.lists, c.table, c.lengths, o, lse, ws]
        args[at] = x
        with pytest.raises(ValueError):
            kvp.decode8(c.desc, c.donor, *args)


@pytest.mark.parametrize("splits", [0, 5])
@pytest.mark.parametrize("byte", [60, 190, 230, 243, 244, 245, 246])
@pytest.mark.parametrize("dh,lens", [(64, [40, 3]), (128, [40, 1000]), (128, [20000, 33]), (64, [700] * 20)])
def test_large_values_behind_rising_scores(kvp, dh, lens, byte, splits):
    """V up to the end of bf16's range (256 * 2^119 = 2^127), scores that rise by less than the sum's reference allows (12 in the
    exponent of e, 2^17.3, in steps of at most 2^6) and many terms alike: the sum times V is far beyond fp32, the output, the value itself, is not.
    (bf16's half step, the weights' half step of 11 bits, fp32 sums.)"""
    c = Case(kvp, [0], lens, 4, 1, dh, 16, splits=splits)
    q = c.q[0]
    q[:] = q[:1, :1]
    unit = q[0, 0].float() * (dh ** 0.5 / q[0, 0].float().pow(2).sum())
    c.scales[0][0].fill_(127)
    c.pools[1][0].copy_(torch.full(c.pools[1][0].shape, 256.0).to(torch.float8_e4m3fn))
    c.scales[1][0].fill_(byte)
    for b, n in enumerate(lens):
        for i in range((n + 15) // 16):                       # 0, 4, 8, 12, 12, ... a block
            c.pools[0][0][int(c.bt[b, i])] = (unit * 4.0 * min(i, 3)).to(torch.float8_e4m3fn)
    o, lse = c.run()
    want = 256.0 * 2.0 ** (byte - 127)
    assert ((o[0].double() - want).abs() <= want * (2.0 ** -8 + 2.0 ** -11 + 2.0 ** -13)).all()
    ro, rl, to, tl = exact(q, c.pools, c.scales, c.bt, lens, 16, dh ** -0.5, 0)
    assert ((lse[0].double() - rl).abs() <= tl).all()


@pytest.mark.parametrize("splits", [0, 4])
@pytest.mark.parametrize("dh,lens", [(64, [40, 3, 0]), (128, [40, 1000]), (128, [20000]), (64, [150] * 20)])
@pytest.mark.parametrize("power", [12, 20, 27, 40, 86, 100, 110, 120])
def test_scores_far_below_zero(kvp, dh, lens, power, splits):
    """Every score of a sequence is a negative number of great magnitude, -2^power and below: its weights are as good as any others.
    All arithmetic is exact but the factor: K = -2^4 in the second half of the blocks and -2^5 in the first, one q element, a power of two.
    Blocks of V differ by powers of two as well."""
    c = Case(kvp, [0], lens, 4, 1, dh, 16, splits=splits)
    k, q = c.pools[0][0], c.q[0]
    k.zero_()
    q.zero_()
    c.scales[1][0].copy_(torch.randint(100, 150, c.scales[1][0].shape, generator=torch.Generator().manual_seed(power), dtype=torch.uint8))
    q[:, :, 5] = 2.0 ** (power // 2)
    c.scales[0][0].fill_(127 + power - power // 2)
    for b, n in enumerate(lens):
        for i in range((n + 15) // 16):
            k[int(c.bt[b, i]), :, :, 5] = -16.0 if 2 * i >= (n + 15) // 16 - 1 else -32.0
    o, lse = c.run(scale=0.25)
    assert c.kvp.device_status() == c.kvp.OK
    for b, n in enumerate(lens):
        if n == 0:
            assert (o[0][b] == 0).all() and (lse[0][b] == -float("inf")).all()
            continue
        blocks = (n + 15) // 16
        near = [i for i in range(blocks) if 2 * i >= blocks - 1]
        value = c.pools[1][0][c.bt[b, near].long().cuda(), 0].double() * torch.exp2(c.scales[1][0][c.bt[b, near].long().cuda(), 0].double() - 127)[..., None]
        value = value.flatten(0, 1)[:n - near[0] * 16]
        want, size = value.mean(0), value.abs().mean(0)
        assert ((o[0][b].double() - want).abs() <= 2.0 ** -8 * want.abs() + size * (2.0 ** -11 + 2.0 ** -13)).all()
        assert (lse[0][b].double() + 2.0 ** (power + 2) - np.log(len(value))).abs().max() <= 2.0 ** -20 * 2.0 ** (power + 2)


@pytest.mark.parametrize("dh,Hq,Hkv", [(128, 8, 2), (64, 12, 1)])
def test_fp32_queries_are_rounded_to_bf16_on_load(kvp, dh, Hq, Hkv):
    """fp32 queries between the numbers of bf16, ties to either side among them: results as from those rounded to nearest even."""
    a, b = (Case(kvp, [0, 0], [700, 1, 33], Hq, Hkv, dh, 16, io) for io in ("f32", "bf16"))
    g = torch.Generator(device="cuda").manual_seed(8)
    for x, y in zip(a.q, b.q):
        step = torch.randint(-65536, 65537, x.shape, generator=g, device="cuda")
        step[..., ::3] = torch.where(step[..., ::3] > 0, 32768, -32768)
        x.view(torch.int32).add_(torch.where(x == 0, 0, step).int())
        y.copy_(x)
        assert (x != y.float()).float().mean() > 0.9
    (oa, la), (ob, lb) = a.run(), b.run()
    b.check(ob, lb)
    for l in range(2):
        assert torch.equal(oa[l], ob[l].float()) and torch.equal(la[l], lb[l])


AHEAD = [  # lengths in turn, Hkv, dh, page, columns of the table behind the longest's
    ([20000], [777], 1, 128, 128, 1),                         # many shares, few; the merge
    ([300, 5000, 0], [4000, 0, 129], 2, 128, 16, 1),
    ([300, 5000, 1100], [4000, 200, 129], 2, 64, 16, 1),
    ([130] * 32, [130] * 31 + [9000], 2, 64, 16, 1),          # whole units, shares
    ([130, 300] * 10, [300, 130] * 10, 2, 128, 16, 1),        # whole units, fewer than blocks
    ([700] * 33, [700] * 32 + [8000], 2, 64, 16, 1),          # more lengths than a warp's lanes: behind the wait alone
    (30, 16, 128, 16, 1),                                     # teams by the length, lengths of the whole batch
    (30, 16, 128, 16, 2000),                                  # the same where the lengths alone say that units are short
    (30, 32, 64, 16, 1),
    (100, 8, 128, 16, 1),
    (128, 8, 128, 16, 1),
    (150, 16, 64, 16, 1),                                     # (more than are looked at)
]


@pytest.mark.parametrize("case", range(len(AHEAD)))
def test_lengths_that_a_kernel_of_the_library_writes(kvp, case):
    """Lengths are looked at before the kernel ahead has finished, while it is writing others: what it writes counts, in the deal, in the
    teams and in the merge."""
    if len(AHEAD[case]) == 6:
        first, second, Hkv, dh, page, columns = AHEAD[case]
    else:
        B, Hkv, dh, page, columns = AHEAD[case]
        r = np.random.default_rng(B)
        first, second = ([int(x) for x in r.integers(128, 350, B)] for _ in range(2))
        first[3], second[0], first[-1], second[-2] = 0, 700, 650, 0
    longest = [max(a, b) for a, b in zip(first, second)]
    c = Case(kvp, [0], longest, Hkv, Hkv, dh, page, poison=False, columns=columns)
    want = [exact(c.q[0], c.pools, c.scales, c.bt, lens, page, dh ** -0.5, 0) for lens in (first, second)]
    ahead = Ahead(kvp, [torch.tensor(first)], [torch.tensor(second)])
    runs = [c.outputs() for _ in range(8)]
    torch.cuda.synchronize()
    for i, (o, lse, ws) in enumerate(runs):
        ahead.write(i)
        kvp.decode8(c.desc, c.donor, c.q, *c.lists, c.table, ahead.views[0], o, lse, ws)
    assert kvp.device_status() == kvp.OK
    for i, (o, lse, _) in enumerate(runs):
        ro, rl, to, tl = want[i % 2]
        assert ((o[0].double() - ro).abs() <= to).all(), i
        some = torch.isfinite(rl)
        assert ((lse[0].double() - rl).abs() <= tl)[some].all() and (lse[0][~some] == -float("inf")).all(), i


LISTS = [  # donor, lengths, Hq, Hkv, dh, page
    # 9 to 16 rows: two blocks an SM fit at dh 128, three at dh 64
    ([0, 1, 2, 3, 4, 4, 4, 4], [16000 + 37 * b for b in range(4)] + [1, 0, 700], 32, 8, 128, 128),      # three rounds: one small share a block
    ([0, 1, 2, 3, 4, 4, 4, 4], [57000 + 37 * b for b in range(4)] + [1, 0, 700], 32, 8, 128, 128),      # twelve: two
    ([0, 0], [5000, 3, 3000, 0, 17] * 2, 64, 8, 128, 32),     # places behind the granules of a unit, fewer than three rounds
    ([0], [30000, 100, 41000, 5, 33], 128, 8, 128, 64),
    ([0, 0, 0, 0], [9000, 1, 3000, 0, 500], 32, 8, 64, 16),   # the same at dh 64: one round,
    ([0, 0, 0, 0], [70000, 80000, 7], 32, 8, 64, 64),         # two,
    ([0, 1], [100000, 120001, 130000, 60], 128, 8, 64, 128),  # five
    # up to 8 rows
    ([0], [5000, 3, 7000, 0, 17], 8, 8, 128, 32),
    ([0, 1], [60000, 100, 90000, 5], 8, 8, 128, 64),          # two rounds of shares alike
    ([0, 0], [9000, 1, 3000, 0, 500, 9000], 16, 8, 64, 16),
    ([0, 1], [60000, 100, 50000, 33], 8, 8, 64, 64),
    ([0, 1, 2], [100000, 70001, 60000, 60], 24, 8, 64, 128),
]


@pytest.mark.parametrize("case", range(len(LISTS)))
def test_long_lists(kvp, case):
    """Lists of K/V rows of every plan: rounds of shares alike, of two sizes, places that stand for a unit's merge; and the same again."""
    donor, lens, Hq, Hkv, dh, page = LISTS[case]
    c = Case(kvp, donor, lens, Hq, Hkv, dh, page)
    o, lse = c.run()
    c.check(o, lse)
    again, lse2 = c.run()
    assert all(torch.equal(x, y) for x, y in zip(o + lse, again + lse2))


@pytest.mark.parametrize("splits", [0, 4])
@pytest.mark.parametrize("dh,Hq,lens", [(64, 4, [40, 3, 0]), (128, 4, [32, 1000]), (128, 12, [20000]), (64, 16, [150] * 20), (64, 1, [300])])
@pytest.mark.parametrize("power", [10, 16, 22, 28, 34, 50, 90])
def test_scores_of_great_magnitude_that_are_rounded(kvp, dh, Hq, lens, power, splits):
    """Two keys in turn, whose scores are numbers like any others times 2^power: tokens of the larger one have one weight, the others none.
    (Every query has an element of 1 or -1 along the keys' difference: scores 2^power and more apart, far more than their errors.)"""
    c = Case(kvp, [0], lens, Hq, 1, dh, 16, splits=splits)
    g = torch.Generator(device="cuda").manual_seed(power)
    two = (torch.randn(2, dh, device="cuda", generator=g) * 64).to(torch.float8_e4m3fn)
    q, along = torch.randn(Hq, dh, device="cuda", generator=g), torch.nn.functional.normalize(two[0].float() - two[1].float(), dim=0)
    sign = torch.tensor([1.0, -1.0, -1.0] * Hq, device="cuda")[:Hq, None]
    q = (q - (q @ along)[:, None] * along + sign * along).bfloat16()
    y = q.double() @ two.double().T * 2.0 ** -6 * 0.25        # [Hq, 2]
    assert ((y[:, 0] - y[:, 1]).abs() > 1).all()
    c.q[0][:] = q * 2.0 ** (power // 2)
    c.scales[0][0].fill_(127 - 6 + power - power // 2)
    c.pools[0][0][:, :, 0::2] = two[0]
    c.pools[0][0][:, :, 1::2] = two[1]
    o, lse = c.run(scale=0.25)
    for b, n in enumerate(lens):
        if n == 0:
            assert (o[0][b] == 0).all() and (lse[0][b] == -float("inf")).all()
            continue
        pages = c.bt[b, :(n + 15) // 16].long().cuda()
        value = (c.pools[1][0][pages, 0].double() * torch.exp2(c.scales[1][0][pages, 0].double() - 127)[..., None]).flatten(0, 1)[:n]
        for h in range(Hq):
            best = int(y[h].argmax()) if n > 1 else 0
            v = value[best::2]
            want, size = v.mean(0), v.abs().mean(0)
            # beside the winners the others weigh e^-1024 at most
            assert ((o[0][b, h].double() - want).abs() <= 2.0 ** -8 * want.abs() + size * (2.0 ** -11 + 2.0 ** -13)).all(), (b, h)
            assert abs(float(lse[0][b, h]) - float(y[h, best]) * 2.0 ** power - np.log(len(v))) <= 2.0 ** -16 * float(y[h].abs().max() + 16) * 2.0 ** power
