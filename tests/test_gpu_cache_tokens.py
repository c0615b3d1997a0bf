"""Tokens into the paged cache with their rotary positions: against the oracle in 64 bits, everything else left as it was."""
import numpy as np
import pytest
import torch

from ahead import Ahead
from guard import Guarded
from oracle import cache8 as O
from test_gpu_parity import f64
from paper_2608_15943_b200 import synth

pytestmark = pytest.mark.gpu

# Rotated elements in fp32: sine and cosine within 2^-22 (two ulps of 1, and the angle's 2^-32 turns), two products and a sum of
# half an ulp each.  Together below 2^-21 of |a| + |b|; bf16 then adds half a step, 2^-8 of the value (an e4m3 code may be the
# neighbour where the border between the two is nearer than that).
FP32 = 2.0 ** -21


class Cache:
    """Pools, scattered pages, lengths; host copies of everything before the call."""

    def __init__(self, kvp, L, donor, new, old, Hq, Hkv, dh, page, bits, io="bf16", seed=61, fill=1.0, spare=2, guard=None):
        self.kvp, self.donor, self.bits, self.page, self.Hkv = kvp, donor, bits, page, Hkv
        B = len(new)
        self.own = [l for l in range(L) if donor[l] == l]
        self.lengths = [n + o for n, o in zip(new, old)]
        need = [(n + page - 1) // page for n in self.lengths]
        n_pages, max_pages = sum(need) + spare, max(need + [1]) + 1
        order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).int()
        self.table, at = torch.full((B, max_pages), int(order[-1]), dtype=torch.int32), 0
        for b, k in enumerate(need):
            self.table[b, :k] = order[at:at + k]
            at += k
        self.T = T = sum(new)
        self.first = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32)
        self.desc = kvp.DecodeDesc(L, B, Hq, Hkv, dh, page, max_pages, n_pages, 0, kvp.F32 if io == "f32" else kvp.BF16)
        rows = lambda kind, H, ls: [synth.normal((T, H, dh), seed, synth.tid(kind, l), fill, "cuda").to(torch.float32 if io == "f32" else torch.bfloat16)
                                    if l in ls else None for l in range(L)]
        self.q, self.k_new, self.v_new = rows(6, Hq, range(L)), rows(1, Hkv, self.own), rows(2, Hkv, self.own)
        self.guard = g = guard or Guarded()
        self.q_out = [g.empty(x.shape, x.dtype, 7.0) for x in self.q]
        pool = lambda kind, l: synth.normal((n_pages, Hkv, page, dh), seed, synth.tid(kind, l), 1.0, "cuda")

        def held(kind):
            out = []
            for l in range(L):
                if l not in self.own:
                    out.append(None)
                    continue
                x = g.empty((n_pages, Hkv, page, dh), torch.bfloat16 if bits == 16 else torch.float8_e4m3fn)
                x.copy_(pool(kind, l) if bits == 16 else (pool(kind, l) * 64).to(torch.float8_e4m3fn))
                out.append(x)
            return out
        self.k_cache, self.v_cache = held(7), held(8)
        self.k_scale = self.v_scale = None
        if bits == 8:
            r = np.random.default_rng(seed)

            def scales():
                out = []
                for l in range(L):
                    x = g.empty((n_pages, Hkv, page // 16), torch.uint8)
                    x.copy_(torch.from_numpy(r.integers(112, 124, x.shape).astype(np.uint8)))
                    out.append(x if l in self.own else None)
                return out
            self.k_scale, self.v_scale = scales(), scales()

    def lists(self):
        return self.k_new, self.v_new, self.k_cache, self.v_cache, self.table.cuda(), torch.tensor(self.lengths, dtype=torch.int32, device="cuda")

    def call(self, theta=10000.0, one=False, q=True, **over):
        kw = dict(first=None if one else self.first.cuda(), theta=theta, k_scale=self.k_scale, v_scale=self.v_scale)
        if q:
            kw.update(q=self.q, q_out=self.q_out)
        kw.update(over)
        self.kvp.cache_append_tokens(self.desc, self.donor, *self.lists(), **kw)

    def snapshot(self):
        host = lambda ts: [None if t is None else t.view(torch.uint8).cpu().numpy().copy() if t.element_size() == 1 else f64(t) for t in ts]
        return {n: host(getattr(self, n)) for n in ("k_cache", "v_cache", "q_out")} | (
            {n: host(getattr(self, n)) for n in ("k_scale", "v_scale")} if self.bits == 8 else {})

    def positions(self, b):
        return np.arange(self.lengths[b] - int(self.first[b + 1] - self.first[b]), self.lengths[b])

    def check(self, before, theta, q=True):
        """Everything after the call against the oracle on the state before it."""
        torch.cuda.synchronize()
        assert self.kvp.device_status() == self.kvp.OK
        after = self.snapshot()
        table = self.table.numpy()
        span = lambda b: slice(int(self.first[b]), int(self.first[b + 1]))
        for l in range(len(self.donor)):
            want, slack = before["q_out"][l].copy(), np.zeros(before["q_out"][l].shape)
            if q:
                x = f64(self.q[l])
                for b in range(len(self.lengths)):
                    want[span(b)] = O.rotate(x[span(b)], self.positions(b), theta)
                    slack[span(b)] = turn_error(x[span(b)], theta)
            assert (np.abs(after["q_out"][l] - want) <= 2.0 ** -8 * np.abs(want) * (slack >= 0) * (1 if q else 0) + slack).all()
        for name, new, turned in (("k", self.k_new, theta), ("v", self.v_new, 0.0)):
            for l in self.own:
                x = f64(new[l])
                got, want = after[name + "_cache"][l], before[name + "_cache"][l]
                if self.bits == 16:
                    slack = np.zeros(want.shape)
                    for b in range(len(self.lengths)):
                        pos, rows = self.positions(b), x[span(b)]
                        for p, r, e in zip(pos, O.rotate(rows, pos, turned), turn_error(rows, turned)):
                            want[table[b, p // self.page], :, p % self.page] = r
                            slack[table[b, p // self.page], :, p % self.page] = e + (2.0 ** -8 * np.abs(r) if turned else 0)
                    assert (np.abs(got - want) <= slack).all()
                    continue
                scale = before[name + "_scale"][l]
                near = np.zeros(want.shape, bool)           # codes whose neighbour will do
                for b in range(len(self.lengths)):
                    pos, rows = self.positions(b), x[span(b)]
                    r, err = O.rotate(rows, pos, turned), turn_error(rows, turned)
                    start = self.lengths[b] - len(rows)
                    for p, i, a, end, e in O.append8(want, scale, table[b], self.lengths[b], r):
                        lo = np.flatnonzero(table[b] == p)[0] * self.page + i * 16
                        part = slice(lo + a - start, lo + end - start)
                        power = np.exp2(-e)[None, :, None]
                        near[p, :, i * 16 + a:i * 16 + end] = (O.border_distance(r[part] * power) <= err[part] * power).transpose(1, 0, 2)
                assert np.array_equal(after[name + "_scale"][l], scale)
                off = got != want
                assert not (off & ~near).any()
                assert (np.abs(got[off].astype(int) - want[off].astype(int)) == 1).all() and off.mean() < 1e-3
        self.guard.check()


def turn_error(x, theta):
    if theta == 0:
        return np.zeros(x.shape)
    s = np.abs(x[..., 0::2]) + np.abs(x[..., 1::2])
    return FP32 * np.repeat(s, 2, -1)


@pytest.fixture(scope="module")
def kvp():
    from paper_2608_15943_b200 import kvp as mod
    return mod


CASES = [  # L, donor, new, old, Hq, Hkv, dh, page, theta
    (2, [0, 0], [1, 1, 1], [0, 15, 16], 4, 2, 128, 16, 10000.0),
    (2, [0, 1], [1] * 5, [1, 31, 7, 100, 48], 3, 1, 64, 48, 500000.0),
    (3, [0, 1, 1], [5, 0, 16, 17, 1, 40], [0, 9, 16, 3, 14, 123], 8, 2, 128, 32, 10000.0),
    (1, [0], [33, 2], [1000, 77], 5, 5, 64, 64, 10000.0),
    (1, [0], [300], [7], 16, 1, 128, 128, 0.0),
    (9, [0, 1, 2, 3, 4, 5, 6, 7, 7], [3, 4], [13, 14], 2, 1, 64, 16, 10000.0),      # more layers than the small parameter block has
]


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("L,donor,new,old,Hq,Hkv,dh,page,theta", CASES)
def test_against_the_oracle(kvp, L, donor, new, old, Hq, Hkv, dh, page, theta, bits, io):
    c = Cache(kvp, L, donor, new, old, Hq, Hkv, dh, page, bits, io)
    before = c.snapshot()
    c.call(theta)
    c.check(before, theta)
    if set(new) == {1}:                                      # the form of one token a sequence
        c = Cache(kvp, L, donor, new, old, Hq, Hkv, dh, page, bits, io)
        c.call(theta, one=True)
        c.check(before, theta)


@pytest.mark.parametrize("bits", [16, 8])
def test_many_sequences_and_layers(kvp, bits):
    """More sequences than threads of a block, more layers than one launch takes."""
    r = np.random.default_rng(4)
    new, old = [int(x) for x in r.integers(0, 4, 300)], [int(x) for x in r.integers(0, 40, 300)]
    c = Cache(kvp, 2, [0, 1], new, old, 2, 1, 64, 16, bits)
    before = c.snapshot()
    c.call()
    c.check(before, 10000.0)
    c = Cache(kvp, 70, [0] * 66 + [66] * 4, [1, 2], [3, 30], 1, 1, 64, 16, bits)
    before = c.snapshot()
    c.call()
    c.check(before, 10000.0)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dh,Hq,Hkv,page", [(64, 9, 3, 48), (128, 10, 5, 128)])
def test_long_runs(kvp, bits, dh, Hq, Hkv, page):
    """More blocks of positions than are on the device at once; heads that do not fill a group."""
    c = Cache(kvp, 2, [0, 1], [3001, 1, 2500, 4000], [0, 77, 5, 130], Hq, Hkv, dh, page, bits)
    before = c.snapshot()
    c.call()
    c.check(before, 10000.0)


@pytest.mark.parametrize("bits", [16, 8])
def test_a_prompt_among_single_tokens(kvp, bits):
    """A mixed batch: 70 sequences with a token each and one with 500, whose later blocks are looked up behind all the others."""
    new = [1] * 45 + [500] + [1] * 25
    c = Cache(kvp, 2, [0, 0], new, [i % 37 for i in range(71)], 8, 2, 128, 16, bits)
    before = c.snapshot()
    c.call()
    c.check(before, 10000.0)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("one", [False, True])
def test_without_queries_and_in_place(kvp, bits, one):
    args = (kvp, 2, [0, 0], [1, 1, 1], [4, 0, 30], 4, 2, 64, 16, bits)
    c = Cache(*args)
    before = c.snapshot()
    c.call(one=one, q=False)
    c.check(before, 10000.0, q=False)
    a, b = Cache(*args), Cache(*args)
    a.call(one=one)
    b.call(one=one, q_out=b.q)
    for x, y in zip(a.q_out, b.q):
        assert torch.equal(x, y)


@pytest.mark.parametrize("bits", [16, 8])
def test_far_positions(kvp, bits):
    """Position 130000 and beyond: the angle's error does not grow with it."""
    c = Cache(kvp, 1, [0], [3, 20], [131000, 1 << 18], 4, 1, 128, 128, bits)
    before = c.snapshot()
    c.call()
    c.check(before, 10000.0)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("one", [False, True])
def test_left_out(kvp, bits, one):
    """Lengths of zero, below and above the table, pages outside the pool, rows in front of and behind the sequences: nothing is written."""
    B = 6
    c = Cache(kvp, 1, [0], [1] * B, [20] * B, 2, 1, 64, 16, bits)
    c.lengths = [0, -3, 21, 1 << 20, 21, 21]
    c.table[4, 1], c.table[5, 1] = -1, c.desc.n_pages       # the page of position 20
    before = c.snapshot()
    c.call(one=one)
    torch.cuda.synchronize()
    after = c.snapshot()
    page = int(c.table[2, 1])
    for name in after:
        for x, y in zip(before[name], after[name]):
            if x is None:
                continue
            same = x == y
            if name == "q_out":                             # bad pages hold back K and V alone
                assert same[[0, 1, 3]].all() and not same[[2, 4, 5]].all(axis=(1, 2)).any()
            elif name.endswith("cache"):
                where = np.argwhere(~same)
                assert (where[:, 2] == 4).any() and (where[:, 0] == page).all() and (where[:, 2] >= (4 if bits == 16 else 0)).all() and (where[:, 2] <= 4).all()
            else:
                assert (np.argwhere(~same)[:, 0] == page).all()
    c.guard.check()


def test_rows_outside_the_sequences(kvp):
    """T rows of which the sequences have some: those in front, between and behind stay, whatever `first` says beyond T."""
    for bits in (16, 8):
        c = Cache(kvp, 1, [0], [4, 4, 4], [10, 10, 10], 2, 1, 64, 16, bits)
        c.first = torch.tensor([2, 5, 5, 40], dtype=torch.int32)     # rows 2..4, none, 5..39 of which there are 5..11
        c.lengths = [13, 10, 50]
        before = c.snapshot()
        c.call()
        torch.cuda.synchronize()
        after = c.snapshot()
        x = f64(c.q[0])
        got = after["q_out"][0]
        assert (got[:2] == 7).all()
        for rows, pos in ((slice(2, 5), np.arange(10, 13)), (slice(5, 12), np.arange(15, 22))):
            want = O.rotate(x[rows], pos, 10000.0)
            assert (np.abs(got[rows] - want) <= 2.0 ** -8 * np.abs(want) + turn_error(x[rows], 10000.0)).all()
        changed = {(int(p), int(s)) for p, _, s, _ in np.argwhere(before["v_cache"][0] != after["v_cache"][0])}
        table = c.table.numpy()
        new = {(int(table[b, p // 16]), p % 16) for b, ps in ((0, range(10, 13)), (2, range(15, 22))) for p in ps}
        block_of = {(p, s) for p, _ in new for s in range(16)}      # (8 bits: older numbers of a block may be rounded again)
        assert changed <= (new if bits == 16 else block_of) and {p for p, _ in changed} == {p for p, _ in new}
        c.guard.check()


def test_scale_grows_and_holds(kvp):
    """A block filled token by token with magnitudes that rise and fall over many powers of two: after each step the oracle's codes."""
    for one in (True, False):
        c = Cache(kvp, 1, [0], [1], [0], 2, 2, 64, 16, 8)
        gain = [1.0, 2.0 ** -20, 3.0, 500.0, 2.0, 2.0 ** 40, 0.0, 2.0 ** 38, 2.0 ** 41, 1.0, 2.0 ** 90, 2.0 ** 90, 7.0, 2.0 ** 100, 1.0, 0.5, 0.0, 2.0 ** -120, 2.0 ** -90, 1e-30]
        k, v = c.k_new[0].clone(), c.v_new[0].clone()
        for n, x in enumerate(gain):
            c.lengths = [n + 1]
            c.k_new[0], c.v_new[0] = k * x, v * x
            before = c.snapshot()
            c.call(theta=0.0, one=one, q=False)
            c.check(before, 0.0, q=False)


def test_a_fresh_block_forgets(kvp):
    """A block whose first token is new takes nothing from what the page held: neither scale nor numbers."""
    for one in (True, False):
        c = Cache(kvp, 1, [0], [1], [16], 1, 1, 64, 16, 8)
        p = int(c.table[0, 1])
        c.k_scale[0][p], c.v_scale[0][p] = 255, 247
        c.k_cache[0].view(torch.uint8)[p], c.v_cache[0].view(torch.uint8)[p] = 0x7f, 0xff
        before = c.snapshot()
        c.call(one=one)
        c.check(before, 10000.0)
        assert int(c.k_scale[0][p, 0, 0]) < 127 and (c.k_cache[0].view(torch.uint8)[p, 0, 1:] == 0x7f).all()


def test_not_finite(kvp):
    """Infinities and NaN become NaN in 8 bits, and the exponent goes by the rest; in bf16 they stay what they are."""
    for one in (True, False):
        c = Cache(kvp, 1, [0], [1, 1], [3, 16], 1, 1, 64, 16, 8)
        c.v_new[0][0, 0, :3] = torch.tensor([float("inf"), float("-inf"), float("nan")])
        c.v_new[0][1] = float("inf")                          # nothing finite: the least scale
        before = c.snapshot()
        c.call(theta=0.0, one=one)
        c.check(before, 0.0)
        assert int(c.v_scale[0][int(c.table[1, 1]), 0, 0]) == 27
        c = Cache(kvp, 1, [0], [1, 1], [3, 16], 1, 1, 64, 16, 16)
        c.v_new[0][0, 0, :3] = torch.tensor([float("inf"), float("-inf"), float("nan")])
        c.call(theta=0.0, one=one)
        row = c.v_cache[0][int(c.table[0, 0]), 0, 3]
        assert torch.equal(row.view(torch.int16)[:2], c.v_new[0][0, 0].view(torch.int16)[:2]) and torch.isnan(row[2]) and torch.equal(row[3:], c.v_new[0][0, 0, 3:])


def test_begun_blocks_with_foreign_scales(kvp):
    """Bytes that no append writes count as the nearest that one could have written."""
    for one in (True, False):
        for byte, e in ((0, -100), (255, 120)):
            c = Cache(kvp, 1, [0], [1], [5], 1, 1, 64, 16, 8)
            p = int(c.table[0, 0])
            c.k_scale[0][p], c.v_scale[0][p] = byte, byte
            old = O.VALUE[c.v_cache[0].view(torch.uint8)[p, 0, :5].cpu().numpy()]
            c.call(one=one, theta=0.0)
            torch.cuda.synchronize()
            got = int(c.v_scale[0][p, 0, 0]) - 127
            assert got == max(e, int(O.exponent(np.abs(f64(c.v_new[0])).max())))
            assert np.array_equal(c.v_cache[0].view(torch.uint8)[p, 0, :5].cpu().numpy(), O.round_e4m3(old * 2.0 ** max(e - got, -200)))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("one", [False, True])
def test_captured_and_on_another_stream(kvp, bits, one):
    """A captured call replayed with new lengths and rows, and a call on a side stream, give what eager calls give."""
    args = (kvp, 2, [0, 0], [1, 1, 1] if one else [4, 1, 9], [4, 0, 30], 4, 2, 64, 16, bits)
    a, b = Cache(*args, spare=4), Cache(*args, spare=4)
    k_new, v_new, k_cache, v_cache, table, lengths = b.lists()
    kw = dict(first=None if one else b.first.cuda(), theta=10000.0, q=b.q, q_out=b.q_out, k_scale=b.k_scale, v_scale=b.v_scale)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        kvp.cache_append_tokens(b.desc, b.donor, k_new, v_new, k_cache, v_cache, table, lengths, **kw)
    torch.cuda.synchronize()
    a.call(one=one)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kvp.cache_append_tokens(b.desc, b.donor, k_new, v_new, k_cache, v_cache, table, lengths, **kw)
    for step in range(1, 3):
        n = [1] * 3 if one else [4, 1, 9]
        a.lengths = [min(x - m + 1, a.desc.max_pages * 16) for x, m in zip([y + m for y, m in zip(a.lengths, [0] * 3)], [0] * 3)]
        lengths.copy_(torch.tensor(a.lengths, dtype=torch.int32))
        for x in a.k_new + a.q:
            if x is not None:
                x.mul_(1.5)
        for x in b.k_new + b.q:
            if x is not None:
                x.mul_(1.5)
        a.call(one=one)
        graph.replay()
        x, y = a.snapshot(), b.snapshot()
        for name in x:
            for u, w in zip(x[name], y[name]):
                assert u is None or np.array_equal(u, w), (step, name)


def test_lengths_of_the_step_ahead(kvp):
    """The launch does not read what the kernels ahead of it still write: appends in a row that each see the length of their own."""
    c = Cache(kvp, 1, [0], [1], [0], 1, 1, 64, 16, 8, spare=5)
    c.table[0, :] = torch.arange(c.desc.max_pages)
    k_new, v_new, k_cache, v_cache, table, lengths = c.lists()
    ref = Cache(kvp, 1, [0], [1], [0], 1, 1, 64, 16, 8, spare=5)
    ref.table[0, :] = torch.arange(c.desc.max_pages)
    lengths.zero_()
    for n in range(1, 17):
        lengths.add_(1)
        kvp.cache_append_tokens(c.desc, [0], k_new, v_new, k_cache, v_cache, table, lengths, theta=10000.0, k_scale=c.k_scale, v_scale=c.v_scale)
    for n in range(1, 17):
        ref.lengths = [n]
        ref.call(one=True, q=False)
        torch.cuda.synchronize()
    x, y = c.snapshot(), ref.snapshot()
    assert all(np.array_equal(u, w) for name in ("k_cache", "v_cache", "k_scale", "v_scale") for u, w in zip(x[name], y[name]))


@pytest.mark.parametrize("B", [3, 40])
def test_places_written_by_the_kernel_ahead(kvp, B):
    """Lengths, first rows and pages are looked at before the kernels ahead have finished; what those write counts."""
    new = [1 + i % 5 for i in range(B)]
    args = (kvp, 1, [0], new, [7 * i % 50 for i in range(B)], 4, 2, 64, 16, 8)
    c, ref = Cache(*args, spare=4), Cache(*args, spare=4)
    k_new, v_new, k_cache, v_cache, table, lengths = c.lists()
    first = c.first.cuda()
    right = (table.clone(), lengths.clone(), first.clone())
    big = torch.zeros(64 << 20, device="cuda")
    table.fill_(0), lengths.fill_(5), first.copy_(torch.arange(B + 1, dtype=torch.int32))
    torch.cuda.synchronize()
    big.add_(1.0)                                             # keeps the device busy ahead of the copies
    for x, y in zip((table, lengths, first), right):
        x.copy_(y)
    kvp.cache_append_tokens(c.desc, [0], k_new, v_new, k_cache, v_cache, table, lengths, first=first, theta=10000.0, q=c.q, q_out=c.q_out, k_scale=c.k_scale,
                            v_scale=c.v_scale)
    ref.call()
    torch.cuda.synchronize()
    x, y = c.snapshot(), ref.snapshot()
    assert all(u is None or np.array_equal(u, w) for name in x for u, w in zip(x[name], y[name]))


def test_same_as_rope_and_append(kvp):
    """One sequence position for all, bf16: kvp_rope and kvp_cache_append give the same up to a rounding."""
    B, pos = 5, 37
    c = Cache(kvp, 1, [0], [1] * B, [pos] * B, 4, 2, 128, 16, 16)
    d = Cache(kvp, 1, [0], [1] * B, [pos] * B, 4, 2, 128, 16, 16)
    c.call(one=True)
    k, q = d.k_new[0].clone().view(B, 1, 2, 128), d.q[0].clone().view(B, 1, 4, 128)
    kvp.rope(k, 10000.0, pos)
    kvp.rope(q, 10000.0, pos)
    kvp.cache_append(d.desc, [0], [k], d.v_new, d.k_cache, d.v_cache, d.table.cuda(), torch.tensor(d.lengths, dtype=torch.int32, device="cuda"))
    assert torch.equal(c.v_cache[0], d.v_cache[0])
    for x, y in ((c.k_cache[0], d.k_cache[0]), (c.q_out[0].view_as(q), q)):
        assert ((x.float() - y.float()).abs() <= 2.0 ** -7 * y.float().abs() + 1e-6).all() and (x != y).float().mean() < 1e-2


def test_host_and_foreign_tensors_are_refused(kvp):
    c = Cache(kvp, 1, [0], [1, 1], [3, 4], 2, 1, 64, 16, 8)
    k_new, v_new, k_cache, v_cache, table, lengths = c.lists()
    for over in (dict(lengths=lengths.cpu()), dict(block_table=table.cpu()), dict(k_new=[k_new[0].cpu()]), dict(v_cache=[v_cache[0].cpu()])):
        kw = dict(k_new=k_new, v_new=v_new, k_cache=k_cache, v_cache=v_cache, block_table=table, lengths=lengths, k_scale=c.k_scale, v_scale=c.v_scale) | over
        with pytest.raises(ValueError):
            kvp.cache_append_tokens(c.desc, [0], **kw)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("one", [False, True])
@pytest.mark.parametrize("theta", [0.0, 10000.0])
@pytest.mark.parametrize("dh", [64, 128])
def test_fp32_rows_are_rounded_to_bf16_on_load(kvp, bits, one, theta, dh):
    """fp32 numbers between those of bf16, ties to either side among them: cache, scales and queries as from the rows rounded to
    nearest even beforehand, bit for bit, and by the oracle of those.  One row's largest lies between 448 * 2^e and the next bf16."""
    new, old = ([1, 1, 1], [0, 15, 18]) if one else ([5, 33, 2], [0, 9, 30])
    a, b = (Cache(kvp, 2, [0, 1], new, old, 4, 2, dh, 16, bits, io) for io in ("f32", "bf16"))
    g = torch.Generator(device="cuda").manual_seed(7)
    for x, y in zip(a.q + a.k_new + a.v_new, b.q + b.k_new + b.v_new):
        step = torch.randint(-65536, 65537, x.shape, generator=g, device="cuda")
        step[..., ::3] = torch.where(step[..., ::3] > 0, 32768, -32768)          # ties
        x.view(torch.int32).add_(torch.where(x == 0, 0, step).int())
        if x.shape[1] == 2:
            x[0].clamp_(-400, 400)[0, 0] = 448.0 * 2.0 ** 3 * (1 + 2.0 ** -12)
        y.copy_(x)                                            # to nearest even
        assert (x != y.float()).float().mean() > 0.9
        bits_of = x.view(torch.int32).long() & 0xffffffff     # (torch's rounding, by the bits)
        even = (bits_of + 0x7fff + (bits_of >> 16 & 1)) >> 16
        assert torch.equal(even, y.view(torch.int16).long() & 0xffff)
    before = b.snapshot()
    a.call(theta, one=one)
    b.call(theta, one=one)
    b.check(before, theta)
    x, y = a.snapshot(), b.snapshot()
    for name in x:
        for u, w in zip(x[name], y[name]):
            assert np.array_equal(u, w), name
    a.guard.check()
    if bits == 8:
        row = int(a.table[0, old[0] // 16])
        assert int(a.v_scale[0][row, 0, old[0] % 16 // 16]) == 127 + 3 and float(a.v_cache[0][row, 0, old[0] % 16, 0]) == 448.0


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_queries_that_are_not_turned_are_the_same_numbers(kvp, bits, io):
    """theta 0, and position 0 at any theta: q_out is q, exactly, and so is K in bf16; rows of no sequence keep what q_out held."""
    for new, old, one, theta in (([5, 0, 17, 1], [0, 9, 30, 2], False, 0.0), ([1, 1, 1], [0, 15, 16], True, 0.0), ([1, 1, 1], [0, 0, 0], True, 10000.0),
                                 ([1, 1], [0, 0], False, 10000.0)):
        c = Cache(kvp, 2, [0, 0], new, old, 4, 2, 64, 16, bits, io, spare=3)
        if not one:                                           # the last rows are nobody's
            c.first = torch.cat([c.first[:-1], c.first[-1:] - 1])
            c.lengths[-1] -= 1
        rows = c.T if one else c.T - 1
        c.call(theta, one=one)
        torch.cuda.synchronize()
        for l in range(2):
            assert torch.equal(c.q_out[l][:rows], c.q[l][:rows]) and (c.q_out[l][rows:] == 7).all()
        if bits == 16:
            for b, n in enumerate(c.lengths):
                for i, p in enumerate(range(n - int(c.first[b + 1] - c.first[b]), n)):
                    row = int(c.first[b]) + i
                    page, slot = int(c.table[b, p // 16]), p % 16
                    assert torch.equal(c.k_cache[0][page, :, slot].float(), c.k_new[0][row].float()) and torch.equal(c.v_cache[0][page, :, slot].float(), c.v_new[0][row].float())
        c.guard.check()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("form,what", [("one", "lengths"), ("one", "table"), ("one", "all"), ("runs", "lengths"), ("runs", "table"), ("runs", "first"), ("runs", "all")])
@pytest.mark.parametrize("B", [2, 5])
def test_places_that_a_kernel_of_the_library_writes(kvp, form, B, what, bits):
    """Lengths, first rows and pages are looked at before the kernel ahead has finished, while it is writing others: what it writes
    counts, whichever of them it is that changes.  Each call has a cache of its own, compared with calls behind a finished kernel."""
    one = form == "one"
    r = np.random.default_rng(B)
    new = [1] * B if one else [128 + int(x) for x in r.integers(0, 40, B)]
    c = Cache(kvp, 2, [0, 0], new, [int(x) for x in r.integers(0 if not one else 130, 40 if not one else 170, B)], 4, 2, 64, 16, bits, spare=256)
    n_pages, columns = c.desc.n_pages, c.table.shape[1]
    pages = [128 + torch.from_numpy(r.permutation(n_pages - 128)[:B * columns]).int().view(B, columns) for _ in range(2)]
    lengths = [torch.tensor(c.lengths), torch.tensor([max(128, n - int(x)) for n, x in zip(c.lengths, r.integers(1, 2 if not one else 30, B))])]
    first = [c.first, torch.cat([c.first[:1], (c.first[1:] + torch.from_numpy(r.integers(-9, 0, B)).int()).clamp(min=128)])]
    if B > 2:
        lengths[1][1] = 0
    state = lambda i: [x[i if what in (name, "all") else 0] for name, x in (("lengths", lengths), ("table", pages), ("first", first)) if not one or name != "first"]
    ahead = Ahead(kvp, state(0), state(1))
    k_new, v_new = c.k_new, c.v_new
    owned = ("k_cache", "v_cache", "k_scale", "v_scale") if bits == 8 else ("k_cache", "v_cache")

    def call(out, lens, table, f=None):
        kvp.cache_append_tokens(c.desc, c.donor, k_new, v_new, out["k_cache"], out["v_cache"], table, lens, first=f, theta=10000.0, q=c.q,
                                q_out=out["q_out"], k_scale=out.get("k_scale"), v_scale=out.get("v_scale"))
    copies = lambda: {n: [None if x is None else x.clone() for x in getattr(c, n)] for n in owned + ("q_out",)}
    want, runs = [copies() for _ in range(2)], [copies() for _ in range(8)]
    for i in (0, 1):
        there = [x.cuda().int() for x in state(i)]
        torch.cuda.synchronize()
        call(want[i], *there)
        torch.cuda.synchronize()
    same = lambda x, y: all(u is None or torch.equal(u.view(torch.uint8), w.view(torch.uint8)) for n in x for u, w in zip(x[n], y[n]))
    assert not same(*want)
    for i, out in enumerate(runs):
        ahead.write(i)
        call(out, *ahead.views)
    assert kvp.device_status() == kvp.OK
    for i, out in enumerate(runs):
        assert same(out, want[i % 2]), i
