"""Attention of new tokens over the paged cache, against attention in 64 bits over the numbers that the cache stands for."""
import random

import pytest
import torch

from guard import Guarded
from paper_2608_15943_b200 import synth

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def kvp():
    from paper_2608_15943_b200 import kvp as mod
    return mod


class Case:
    """Sequences of `lens` tokens, the last new[b] of them rows of the call.  What no row sees holds NaN: slots behind the sequence and
    in pages of no sequence; with a window the tokens before it, whose table entries are no pages either where `freed`."""

    def __init__(self, kvp, donor, lens, new, Hq, Hkv, dh, page, bits=16, window=0, sinks=0, io="bf16", seed=91, pad=0, columns=1, one_each=False, freed=True,
                 gain=1.0):
        self.kvp, self.donor, self.lens, self.new, self.page, self.window, self.sinks, self.bits = kvp, donor, lens, new, page, window, sinks, bits
        L, B = len(donor), len(lens)
        self.L, self.B, self.Hq, self.Hkv, self.dh, self.one_each = L, B, Hq, Hkv, dh, one_each
        self.dtype = torch.float32 if io == "f32" else torch.bfloat16
        self.own = [l for l in range(L) if donor[l] == l]
        need = [(n + page - 1) // page for n in lens]
        n_pages, max_pages = sum(need) + 2, max(need + [0]) + columns
        g = torch.Generator().manual_seed(seed)
        order, at = torch.randperm(n_pages, generator=g).int(), 0
        self.bt = torch.full((B, max_pages), -1, dtype=torch.int32)
        live = torch.zeros(n_pages, page, dtype=torch.bool)
        for b, k in enumerate(need):
            self.bt[b, :k] = order[at:at + k]
            at += k
            j = torch.arange(lens[b])
            seen = (j > lens[b] - new[b] - window) | (j < sinks) if window else j >= 0
            seen = seen if new[b] else torch.zeros_like(seen)
            live[self.bt[b, j // page].long(), j % page] = seen
            if freed:
                for i in range(k):
                    if not seen[i * page:(i + 1) * page].any():
                        self.bt[b, i] = (-1, n_pages, 1 << 30, -7)[i % 4]
        dead = (~live).cuda()
        self.pools, self.scales = [], []
        for i in range(2):
            ps, ss = [], []
            for l in range(len(self.own)):
                x = synth.normal((n_pages, Hkv, page, dh), seed, synth.tid(7 + i, l), 1.0, "cuda")
                if bits == 8:
                    x = (x * 64).to(E4M3)
                    x.view(torch.uint8).transpose(1, 2)[dead] = 0x7f
                    s = torch.randint(117, 124, (n_pages, Hkv, page // 16), generator=g, dtype=torch.uint8).cuda()
                    s.transpose(1, 2)[dead.view(n_pages, -1, 16).all(-1)] = 255
                    ss.append(s)
                else:
                    x.transpose(1, 2)[dead] = float("nan")
                ps.append(x)
            self.pools.append(ps)
            self.scales.append(ss)
        first = [0]
        for n in new:
            first.append(first[-1] + (1 if one_each else n))
        self.T = first[-1] + pad
        self.first_host = first
        self.first = torch.tensor(first, dtype=torch.int32, device="cuda")
        self.lengths, self.table = torch.tensor(lens, dtype=torch.int32, device="cuda"), self.bt.cuda()
        self.q = [(synth.normal((self.T, Hq, dh), seed, synth.tid(6, l), 1.0, "cuda") * gain).to(self.dtype) for l in range(L)]
        self.desc = kvp.DecodeDesc(L, B, Hq, Hkv, dh, page, max_pages, n_pages, 0, kvp.F32 if io == "f32" else kvp.BF16)
        at = lambda xs: [xs[self.own.index(l)] if l in self.own else None for l in range(L)]
        self.lists = dict(k=at(self.pools[0]), v=at(self.pools[1]))
        self.kw = dict(window=window, sinks=sinks, first=None if one_each else self.first)
        if bits == 8:
            self.kw.update(k_scale=at(self.scales[0]), v_scale=at(self.scales[1]))

    def outputs(self, guard=None):
        g = guard or Guarded()
        o = [g.empty((self.T, self.Hq, self.dh), self.dtype, float("nan")) for _ in range(self.L)]
        lse = [g.empty((self.T, self.Hq), torch.float32, float("nan")) for _ in range(self.L)]
        ws = g.empty((max(1, self.kvp.attn_chunk_workspace_bytes(self.desc, self.donor, self.T)),), torch.uint8, 0xff)
        return o, lse, ws

    def call(self, o, lse, ws, **kw):
        self.kvp.attn_chunk(self.desc, self.donor, self.q, self.lists["k"], self.lists["v"], self.table, self.lengths, o, lse, ws, **{**self.kw, **kw})

    def run(self, **kw):
        g = Guarded()
        o, lse, ws = self.outputs(g)
        self.call(o, lse, ws, **kw)
        g.check()
        assert self.kvp.device_status() == self.kvp.OK
        return o, lse

    def rows(self):
        """(row of q, sequence, position) of every row that is computed."""
        cap = self.desc.max_pages * self.page
        for b in range(self.B):
            n = self.first_host[b + 1] - self.first_host[b]
            for i in range(n):
                pos = max(self.lens[b], 0) - n + i
                if 0 <= pos < cap:
                    yield self.first_host[b] + i, b, pos

    def keys(self, b, n, layer):
        """[Hkv, n, dh] of K and V in 64 bits."""
        pages = self.bt[b, :(n + self.page - 1) // self.page].long()
        there = ((pages >= 0) & (pages < self.desc.n_pages)).cuda()
        pages = pages.clamp(0, self.desc.n_pages - 1).cuda()
        out = []
        for i in range(2):
            x = self.pools[i][layer][pages].double()
            if self.bits == 8:
                e = self.scales[i][layer][pages].double().clamp(27, 247) - 127
                x = (x.unflatten(2, (-1, 16)) * torch.exp2(e)[..., None, None]).flatten(2, 3)
            x = torch.where(there[:, None, None, None], x, 0.0)
            out.append(x.transpose(0, 1).flatten(1, 2)[:, :n])
        return out

    def exact(self, l, scale=0.0):
        """O and LSE [T, Hq, ...] in 64 bits (NaN where nothing is computed), and what the kernel may be off by:
        scores: products of up to 128 terms summed by the tensor cores, rounded down by up to 2^-23 of the sum of magnitudes each, in
          two chains: 64 * 2^-23 of sum |q k|, doubled for the factor, the difference to the maximum and ex2;
        P: half a step of bf16, 2^-8; O: fp32 sums (2^-13 covers 2^10 roundings of 2^-23); bf16: 2^-8 of the value."""
        G = self.Hq // self.Hkv
        scale = scale or self.dh ** -0.5
        nan = lambda *s: torch.full(s, float("nan"), dtype=torch.float64, device="cuda")
        o, lse, to, tl = nan(self.T, self.Hq, self.dh), nan(self.T, self.Hq), nan(self.T, self.Hq, self.dh), nan(self.T, self.Hq)
        by = {}
        for row, b, pos in self.rows():
            by.setdefault(b, []).append((row, pos))
        for b, at in by.items():
            rows, pos = torch.tensor([r for r, _ in at], device="cuda"), torch.tensor([p for _, p in at], device="cuda")
            n = int(pos[-1]) + 1
            k, v = self.keys(b, n, self.own.index(self.donor[l]))
            j = torch.arange(n, device="cuda")
            seen = j <= pos[:, None]
            if self.window:
                seen &= (j > pos[:, None] - self.window) | (j < self.sinks)
            q = self.q[l][rows].double().unflatten(1, (self.Hkv, G))
            x = torch.einsum("thgd,hnd->thgn", q, k) * scale
            x = torch.where(seen[:, None, None], x, -float("inf"))
            size = torch.einsum("thgd,hnd->thgn", q.abs(), k.abs())
            size = torch.where(seen[:, None, None], size, 0.0).amax(-1, keepdim=True) * scale
            p = torch.softmax(x, -1)
            hit = seen.any(0)                              # (0 * NaN of what nobody sees)
            v = torch.where(hit[:, None], v, 0.0)
            ob = torch.einsum("thgn,hnd->thgd", p, v)
            a = torch.einsum("thgn,hnd->thgd", p, v.abs())
            lb = torch.logsumexp(x, -1)
            ds = 2.0 ** -16 * size
            o[rows], lse[rows] = ob.flatten(1, 2), lb.flatten(1, 2)
            to[rows] = (a * (2.0 ** -8 + 2.0 ** -13 + 2 * ds) + 2.0 ** -8 * ob.abs()).flatten(1, 2)
            tl[rows] = ds.squeeze(-1).flatten(1, 2) + 2.0 ** -20 * (1 + lse[rows].abs())
        return o, lse, to, tl

    def check(self, o, lse, scale=0.0, layers=None):
        for l in range(self.L) if layers is None else layers:
            ro, rl, to, tl = self.exact(l, scale)
            some = ~torch.isnan(rl[:, 0])
            assert torch.isfinite(o[l][some]).all() and torch.isfinite(lse[l][some]).all()
            off = ((o[l].double() - ro).abs() - to)[some]
            assert (off <= 0).all(), off.max()
            off = ((lse[l].double() - rl).abs() - tl)[some]
            assert (off <= 0).all(), off.max()
            assert torch.isnan(o[l][~some]).all() and torch.isnan(lse[l][~some]).all()      # left as they were


SHAPES = [
    # donor, lengths, new tokens, Hq, Hkv, dh, page
    ([0], [1], [1], 1, 1, 128, 16),
    ([0], [5], [5], 1, 1, 64, 16),
    ([0], [64], [64], 1, 1, 128, 64),                                           # a tile of half its rows, one step
    ([0], [129], [129], 1, 1, 64, 16),                                          # the second tile has one row
    ([0], [257], [257], 2, 1, 128, 32),                                         # three tiles of two heads
    ([0, 0], [300, 17, 64], [3, 17, 1], 8, 2, 128, 16),
    ([0, 0, 2], [1000, 1, 0, 500, 128], [70, 1, 0, 128, 128], 6, 2, 64, 48),    # three heads, groups of two and one
    ([0, 0, 0, 0], [2000, 33], [9, 33], 14, 2, 128, 128),                       # 28 rows a token
    ([0, 1], [5000], [2], 16, 1, 128, 16),                                      # few rows over many shares
    ([0, 1], [5000, 3], [600, 3], 4, 4, 64, 64),
    ([0] * 8, [400, 90], [20, 40], 16, 1, 64, 32),                              # 128 rows a token
    ([0] * 9, [200], [5], 8, 1, 128, 16),                                       # a group in two
    ([0, 1, 1, 3, 4, 5, 5, 7], [700] * 3, [33, 200, 1], 8, 4, 64, 16),          # more groups than the small parameter block has
    (list(range(20)), [90, 20], [10, 20], 2, 1, 64, 16),                        # more than a launch takes
    ([0], [40] * 45, [i % 4 for i in range(45)], 4, 2, 128, 16),                # more than 32 sequences
    ([0, 0], [0, 0], [0, 0], 4, 2, 64, 16),                                     # nothing at all
    ([0, 0], [3000, 2500], [1500, 2500], 8, 2, 128, 64),
]


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("donor,lens,new,Hq,Hkv,dh,page", SHAPES)
def test_against_64_bits(kvp, donor, lens, new, Hq, Hkv, dh, page, bits):
    c = Case(kvp, donor, lens, new, Hq, Hkv, dh, page, bits, pad=3)
    c.check(*c.run())


WINDOWS = [(1, 0), (1, 5), (2, 1), (17, 0), (64, 64), (63, 65), (100, 4), (128, 130), (300, 1000), (5000, 3)]


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("window,sinks", WINDOWS)
def test_windows(kvp, window, sinks, bits):
    for donor, lens, new, Hq, Hkv, dh, page in (([0, 0], [900, 64, 65, 1, 200], [300, 64, 2, 1, 0], 8, 2, 128, 16), ([0, 1], [3000, 130], [5, 130], 3, 1, 64, 48)):
        c = Case(kvp, donor, lens, new, Hq, Hkv, dh, page, bits, window, sinks)
        c.check(*c.run())


@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (1, 3), (130, 4), (1000, 70)])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dh", [64, 128])
def test_one_token_each(kvp, dh, bits, window, sinks):
    c = Case(kvp, [0, 0, 2], [700, 1, 0, 64, 65, 2000, 17] + [90] * 30, [1, 1, 0, 1, 1, 1, 1] + [1] * 30, 8, 2, dh, 32, bits, window, sinks, one_each=True)
    c.check(*c.run())


@pytest.mark.parametrize("bits", [16, 8])
def test_fp32_tensors(kvp, bits):
    """Queries that are bf16 numbers: the results are those of the bf16 call, widened."""
    for kw in (dict(), dict(window=50, sinks=3)):
        a, b = (Case(kvp, [0, 0], [300, 20, 4000], [40, 20, 7], 6, 2, 64, 16, bits, io=io, **kw) for io in ("bf16", "f32"))
        (oa, la), (ob, lb) = a.run(), b.run()
        b.check(ob, lb)
        for l in range(2):
            some = ~torch.isnan(la[l][:, 0])
            assert torch.equal(oa[l][some].float(), ob[l][some]) and torch.equal(la[l][some], lb[l][some])


def test_fp32_queries_between_bf16_numbers(kvp):
    c = Case(kvp, [0], [200], [200], 2, 1, 128, 16, io="f32")
    c.q[0] += torch.rand(c.q[0].shape, device="cuda") * 2.0 ** -9 * c.q[0].abs()
    o, lse = c.run()
    c.q[0] = c.q[0].bfloat16().float()
    c.check(o, lse)


def test_equal_calls_give_equal_bits(kvp):
    for kw in (dict(bits=16), dict(bits=8), dict(bits=16, window=200, sinks=9)):
        c = Case(kvp, [0, 0, 2], [9000, 40, 1200], [6, 40, 700], 8, 2, 128, 64, **kw)
        (o, lse), (o2, lse2) = c.run(), c.run()
        assert all(torch.equal(x, y) for x, y in zip(o + lse, o2 + lse2))


@pytest.mark.parametrize("begin,end", [(0, 1), (1, 2), (1, 4), (2, 3), (3, 4)])
def test_layer_ranges(kvp, begin, end):
    c = Case(kvp, [0, 0, 2, 0], [900, 40], [60, 3], 8, 2, 64, 16)
    o, lse = c.run(layer_begin=begin, layer_end=end)
    c.check(o, lse, layers=range(begin, end))
    for l in set(range(4)) - set(range(begin, end)):
        assert torch.isnan(o[l]).all() and torch.isnan(lse[l]).all()


@pytest.mark.parametrize("scale,gain", [(0.25, 1.0), (3.0, 1.0), (0.0, 40.0), (0.0, 2.0 ** -100), (0.0, 0.0), (1e-30, 1e30)])
def test_scales(kvp, scale, gain):
    for dh in (64, 128):
        c = Case(kvp, [0], [1000, 77], [20, 77], 4, 1, dh, 16, gain=gain)
        c.check(*c.run(scale=scale), scale)


@pytest.mark.parametrize("bits", [16, 8])
def test_lengths_and_rows_that_do_not_fit(kvp, bits):
    """More rows than tokens, lengths below zero and above the table, rows behind T: the rows that have no place are left out."""
    c = Case(kvp, [0], [30, 40, 64, 10], [30, 5, 9, 4], 4, 2, 64, 16, bits, columns=0, freed=False)
    for x in c.pools[0] + c.pools[1]:                         # (every slot of the table may be seen)
        x.copy_(torch.randn(x.shape, device="cuda").to(x.dtype))
    for x in c.scales[0] + c.scales[1]:
        x.fill_(121)
    for lens in ([3, 70, -5, 10], [1 << 30, -(1 << 31), 66, 2], [64, 64, 0, (1 << 31) - 1]):
        c.lens = lens
        c.lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
        c.check(*c.run())
    # `first` beyond 0 .. T is taken as the end, and where it falls (which is not allowed) a sequence has no rows; here 20 .. 29 are
    # of two sequences and nothing is said of them
    c.first_host = [0, 30, 30, 39, 48]
    c.first = torch.tensor([-4, 30, 20, 39, 500], dtype=torch.int32, device="cuda")
    c.kw["first"], c.lens = c.first, [60, 64, 40, 20]
    c.lengths = torch.tensor(c.lens, dtype=torch.int32, device="cuda")
    o, lse = c.run()
    ro, rl, to, tl = c.exact(0)
    for rows in (slice(0, 20), slice(30, 48)):
        assert ((o[0].double() - ro).abs() <= to)[rows].all() and ((lse[0].double() - rl).abs() <= tl)[rows].all()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 3)])
def test_what_a_row_does_not_see_has_no_part(kvp, window, sinks, bits):
    """Infinities and NaN in K and V of later tokens, and of tokens before the window, reach the rows that see them and no others."""
    for at, what in ((199, "v"), (170, "v"), (150, "k"), (130, "v"), (64, "v"), (2, "v")):
        c = Case(kvp, [0, 0], [200, 70], [60, 70], 4, 2, 64, 16, bits, window, sinks, freed=False)
        for x in c.pools[0] + c.pools[1]:                     # nothing but the one number is not finite
            x.copy_(torch.randn(x.shape, device="cuda").to(x.dtype))
        for x in c.scales[0] + c.scales[1]:
            x.fill_(121)
        want = c.run()
        page, pool = int(c.bt[0, at // 16]), c.pools["kv".index(what)][0]
        if bits == 8:
            pool.view(torch.uint8)[page, 1, at % 16, 9] = 0x7f
        else:
            pool[page, 1, at % 16, 9] = float("inf") if what == "v" and at % 4 == 2 else float("nan")
        o, lse = c.run()
        hit = torch.zeros(c.T, dtype=torch.bool, device="cuda")
        for row, b, pos in c.rows():
            hit[row] = b == 0 and at <= pos and (not window or at > pos - window or at < sinks)
        for l in range(2):
            bad = torch.zeros(c.T, 4, 64, dtype=torch.bool, device="cuda")
            if what == "v":
                bad[hit, 2:, 9] = True
                assert torch.equal(lse[l], want[1][l])
            else:
                bad[hit, 2:] = True
                assert torch.isnan(lse[l][hit, 2:]).all() and torch.equal(lse[l][~hit], want[1][l][~hit]) and torch.equal(lse[l][:, :2], want[1][l][:, :2])
            assert torch.equal(~torch.isfinite(o[l]), bad), (at, what)
            # (the rows that the number was added to by itself have their sums in another order)
            assert ((o[l] - want[0][l]).abs()[~bad] <= 2.0 ** -7 * want[0][l].abs()[~bad] + 2.0 ** -8).all()


@pytest.mark.parametrize("bits", [16, 8])
def test_several_values_that_are_not_finite(kvp, bits):
    """In every block of a chunk, in its first and last rows, and a whole block of them."""
    c = Case(kvp, [0], [300], [300], 2, 1, 128, 16, bits, freed=False)
    bad_keys = [0, 63, 64, 100, 127, 128] + list(range(192, 256)) + [299]
    for at in bad_keys:
        x = c.pools[1][0]
        if bits == 8:
            x.view(torch.uint8)[int(c.bt[0, at // 16]), 0, at % 16, at % 128] = 0xff
        else:
            x[int(c.bt[0, at // 16]), 0, at % 16, at % 128] = -float("inf")
    o, lse = c.run()
    bad = torch.zeros(300, 2, 128, dtype=torch.bool, device="cuda")
    for at in bad_keys:
        bad[at:, :, at % 128] = True
    assert torch.equal(~torch.isfinite(o[0]), bad) and torch.isfinite(lse[0]).all()
    for at in bad_keys:
        x = c.pools[1][0]
        x.view(torch.uint8)[int(c.bt[0, at // 16]), 0, at % 16, at % 128 * (1 if bits == 8 else 2):][:1 if bits == 8 else 2] = 0
    ro, rl, to, tl = c.exact(0)
    assert ((o[0].double() - ro).abs() <= to)[~bad].all() and ((lse[0].double() - rl).abs() <= tl).all()


def test_scores_that_are_all_minus_infinity(kvp):
    c = Case(kvp, [0], [80], [4], 2, 1, 64, 16, freed=False)
    c.pools[0][0].fill_(-float("inf"))
    c.q[0].copy_(c.q[0].abs() + 0.1)
    o, lse = c.run()
    assert (o[0] == 0).all() and (lse[0] == -float("inf")).all()


@pytest.mark.parametrize("at", [0, 63, 64, 700, 2900])
def test_one_score_far_above_the_others(kvp, at):
    """References that have to move late, far and once, in every place of a share."""
    c = Case(kvp, [0], [3000], [10], 4, 1, 128, 16, freed=False)
    c.q[0][:, 1:] = c.q[0][:, :1]
    c.pools[0][0][int(c.bt[0, at // 16]), 0, at % 16] = c.q[0][0, 0] * 20
    c.check(*c.run())


def test_scale_bytes_of_any_value(kvp):
    """Scales of V from 2^-100 to 2^100 next to one another; bytes that no append writes."""
    c = Case(kvp, [0], [600, 40], [30, 40], 4, 1, 64, 16, 8, freed=False)
    g = torch.Generator().manual_seed(5)
    c.scales[1][0].copy_(torch.randint(0, 228, c.scales[1][0].shape, generator=g, dtype=torch.uint8))
    c.check(*c.run())


def test_long_cache_offsets(kvp):
    """Pages whose elements lie beyond 2^31 and bytes beyond 2^32."""
    page, Hkv, dh, n_pages = 128, 8, 128, 18000
    if torch.cuda.mem_get_info()[0] < 14e9:
        pytest.skip("needs 14 GB")
    c = Case(kvp, [0], [500, 200], [9, 200], 16, 8, dh, page, freed=False)
    far = [n_pages - 1 - 3 * i for i in range(int((c.bt >= 0).sum()))]
    table = c.bt.clone()
    table[c.bt >= 0] = torch.tensor(far, dtype=torch.int32)
    for i in range(2):
        big = torch.empty(n_pages, Hkv, page, dh, dtype=torch.bfloat16, device="cuda")
        for old, new in zip(c.bt[c.bt >= 0].tolist(), far):
            big[new] = c.pools[i][0][old]
        c.pools[i][0] = big
    c.bt, c.table, c.lists = table, table.cuda(), dict(k=[c.pools[0][0]], v=[c.pools[1][0]])
    c.desc.n_pages = n_pages
    c.check(*c.run())


def test_another_stream_and_captured_graphs(kvp):
    """Two captured calls share a workspace and are replayed in turn, with new lengths and tables; a call on another stream."""
    c, d = (Case(kvp, [0, 0], [3000, 40, 0], [20, 40, 0], 8, 2, 128, 16, seed=s, columns=60) for s in (91, 92))
    (oc, lc, ws), (od, ld, _) = c.outputs(), d.outputs()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.call(oc, lc, ws)
    torch.cuda.synchronize()
    c.check(oc, lc)
    graphs = []
    for x, o, l in ((c, oc, lc), (d, od, ld)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x.call(o, l, ws)
        graphs.append(g)
    for round in range(3):
        for x, g, o, l in ((c, graphs[0], oc, lc), (d, graphs[1], od, ld)):
            for t in o + l:
                t.fill_(float("nan"))
            x.lens = [3000 - 700 * round, 40, 0]
            x.lengths.copy_(torch.tensor(x.lens, dtype=torch.int32))
            g.replay()
        for x, o, l in ((c, oc, lc), (d, od, ld)):
            x.check(o, l)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("donor,lens,new,Hq,Hkv,dh,page,window", [
    ([0], [700, 650, 600, 900, 300, 1000, 60, 640], [600] * 4 + [300, 600, 60, 600], 32, 8, 64, 16, 0),
    ([0, 1, 1], [500 + 40 * (i % 7) for i in range(12)], [200 + 30 * (i % 5) for i in range(12)], 12, 6, 128, 48, 0),       # of two kinds
    ([0], [100 + i % 50 for i in range(130)], [1 + i % 3 for i in range(130)], 10, 5, 64, 16, 0),                           # a step or two each
    ([0, 0], [1500, 1800, 40, 2000], [1500, 1700, 40, 900], 16, 8, 64, 32, 100),
    ([0], [4000] + [200] * 20, [4000] + [200] * 20, 8, 8, 64, 64, 0),                                                       # one far longer than the others
    ([0], [6000, 9000, 100], [6000, 2000, 100], 8, 8, 64, 64, 0),
])
def test_many_units(kvp, donor, lens, new, Hq, Hkv, dh, page, window, bits):
    """Units dealt out in rounds, and the shares behind them, which even out what the rounds gave: of different sizes, some empty."""
    c = Case(kvp, donor, lens, new, Hq, Hkv, dh, page, bits, window, 5 if window else 0)
    (o, lse), (o2, lse2) = c.run(), c.run()
    c.check(o, lse)
    assert all(torch.equal(x, y) for x, y in zip(o + lse, o2 + lse2))


def test_smaller_calls_in_the_workspace_of_a_large_one(kvp):
    c = Case(kvp, [0, 1], [900, 40], [60, 3], 8, 2, 64, 16)
    ws = Guarded().empty((kvp.attn_chunk_workspace_bytes(c.desc, c.donor, 5000),), torch.uint8, 0xff)
    o, lse, _ = c.outputs()
    c.call(o, lse, ws)
    c.check(o, lse)


def test_drawn_calls(kvp):
    r = random.Random(7)
    for _ in range(30):
        B, Hkv, G, dh, page = r.randint(1, 12), r.choice((1, 2, 3)), r.choice((1, 2, 3, 4, 5, 7, 8, 16)), r.choice((64, 128)), r.choice((16, 32, 48, 64, 80, 128, 256))
        L = r.randint(1, 4)
        donor = []
        for l in range(L):
            donor.append(l if not donor or r.random() < 0.5 else donor[r.randrange(l)])
        one = r.random() < 0.3
        new = [r.choice((0, 1, 1, 3, r.randint(1, 300))) for _ in range(B)] if not one else [r.randint(0, 1) for _ in range(B)]
        lens = [n + r.choice((0, 1, r.randint(0, 100), r.randint(0, 3000))) if n or not one else 0 for n in new]
        window = r.choice((0, 0, 1, r.randint(1, 200), r.randint(1, 3000)))
        c = Case(kvp, donor, lens, new, Hkv * G, Hkv, dh, page, r.choice((16, 8)), window, r.randint(0, 200) if window else 0, r.choice(("bf16", "f32")),
                 seed=r.randint(1, 1000), pad=0 if one else r.randint(0, 5), one_each=one, freed=r.random() < 0.7)
        c.check(*c.run())
