"""The cache's pages against the oracle in Python's numbers, and a serving run of everything that reads and writes them."""
import random

import pytest
import torch

from guard import Guarded
from oracle.pages import Book

pytestmark = pytest.mark.gpu
BF, I32, U8 = torch.bfloat16, torch.int32, torch.uint8
E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def kvp():
    from paper_2608_15943_b200 import kvp as mod
    return mod


class Both:
    """The device's state and the oracle's.  Numbers of the pools are random bytes; page p of the device is to have what page
    content[p] had at first."""

    def __init__(self, kvp, rows, page, max_pages, n_pages, donor=(0,), Hkv=2, dh=64, bits=16, seed=1):
        self.kvp, self.bits, self.donor = kvp, bits, list(donor)
        L = len(self.donor)
        self.guard, g = Guarded(), torch.Generator(device="cuda").manual_seed(seed)
        self.desc = kvp.DecodeDesc(L, rows, Hkv, Hkv, dh, page, max_pages, n_pages)
        self.book = Book(page, max_pages, n_pages, rows)
        new = lambda shape, dtype, fill: self.guard.empty(shape, dtype, fill)
        self.refs, self.table, self.lengths = new((n_pages,), I32, 0), new((rows, max_pages), I32, -1), new((rows,), I32, 0)
        self.lacking, self.used = new((1,), I32, 77), new((1,), I32, 77)
        self.ws = new((kvp.pages_workspace_bytes(self.desc),), U8, 0xff)

        def pool(width):
            out = []
            for l in range(L):
                x = None
                if self.donor[l] == l:
                    x = new((n_pages, width), U8, 0)
                    x.copy_(torch.randint(0, 256, x.shape, dtype=U8, device="cuda", generator=g))
                out.append(x)
            return out
        self.raw = [pool(Hkv * page * dh * bits // 8) for _ in range(2)]
        self.scales = [pool(Hkv * page // 16) for _ in range(2)] if bits == 8 else [None, None]
        self.at_first = [[x.clone() if x is not None else None for x in xs] for xs in self.raw + (self.scales if bits == 8 else [])]
        self.pools = [[x.view(E4M3 if bits == 8 else BF) if x is not None else None for x in xs] for xs in self.raw]

    def int32(self, x):
        return torch.tensor(x, dtype=I32, device="cuda")

    def copy(self, src, dst):
        self.kvp.pages_copy(self.desc, self.donor, self.int32(src), self.int32(dst), *self.pools, *self.scales)
        self.book.copy(src, dst)

    def fork(self, parent):
        self.kvp.pages_fork(self.desc, self.int32(parent), self.refs, self.table, self.lengths, self.ws)
        self.book.fork(parent)

    def resize(self, to):
        self.kvp.pages_resize(self.desc, self.donor, self.int32(to), self.refs, self.table, self.lengths, self.lacking, self.ws, *self.pools, *self.scales)
        short = self.book.resize(to)
        assert self.lacking.tolist() == [short]
        return short

    def trim(self, window, sinks):
        self.kvp.pages_trim(self.desc, window, sinks, self.refs, self.table, self.lengths)
        self.book.trim(window, sinks)

    def compact(self):
        self.kvp.pages_compact(self.desc, self.donor, self.refs, self.table, self.lengths, self.used, self.ws, *self.pools, *self.scales)
        assert self.used.tolist() == [self.book.compact()]

    def check(self):
        assert self.book.consistent()
        assert self.refs.tolist() == self.book.refs
        assert self.lengths.tolist() == self.book.lengths
        assert self.table.tolist() == self.book.table
        at = torch.tensor(self.book.content, device="cuda")
        for xs, was in zip(self.raw + (self.scales if self.bits == 8 else []), self.at_first):
            for x, w in zip(xs, was):
                assert x is None or torch.equal(x, w[at])
        self.guard.check()
        assert self.kvp.device_status() == self.kvp.OK


@pytest.mark.parametrize("rows,page,max_pages,n_pages,donor,Hkv,dh,bits", [
    (1, 16, 3, 4, (0,), 1, 64, 16),
    (5, 16, 9, 30, (0, 0), 2, 64, 8),
    (8, 48, 6, 40, (0, 1, 1, 3), 3, 128, 16),
    (7, 128, 4, 25, (0,), 8, 128, 8),
    (40, 32, 5, 150, tuple(range(10)), 1, 64, 8),             # more owners than the small parameter block has
    (3, 16, 2, 5, tuple(range(70)), 1, 64, 16),               # more than a launch takes
    (300, 16, 70, 9000, (0,), 1, 64, 16),                     # a cluster of blocks
    (1500, 16, 12, 3001, (0, 0), 1, 64, 8),                   # more rows than a block has threads
])
def test_random_runs(kvp, rows, page, max_pages, n_pages, donor, Hkv, dh, bits):
    r = random.Random(rows * 7 + page)
    s = Both(kvp, rows, page, max_pages, n_pages, donor, Hkv, dh, bits)
    cap = max_pages * page
    for step in range(25 if rows < 100 else 10):
        what = r.choice(("grow", "grow", "grow", "token", "fork", "fork", "trim", "compact", "any", "copy"))
        n = s.book.lengths
        if what == "grow":
            s.resize([min(cap, x + r.choice((0, 1, r.randint(0, 2 * page)))) if r.random() < 0.8 else x for x in n])
        elif what == "token":
            s.resize([min(cap, x + 1) for x in n])
        elif what == "any":
            s.resize([r.choice((0, x, x // 2, r.randint(0, cap))) if r.random() < 0.4 else x for x in n])
        elif what == "fork":
            s.fork([r.choice((b, b, b, -1, r.randrange(rows), r.randrange(rows), -5, rows, 1 << 30)) for b in range(rows)])
        elif what == "trim":
            s.trim(r.choice((1, page, 3 * page, 1 << 30, (1 << 31) - 1)), r.choice((0, 1, page, page + 1, (1 << 31) - 1)))
        elif what == "compact":
            s.compact()
        else:
            free = [p for p in range(n_pages) if s.book.refs[p] == 0]
            r.shuffle(free)
            held = [p for p in range(n_pages) if s.book.refs[p]]
            pairs = list(zip((r.choice(held) for _ in range(4)), free[:4])) if held else []
            if free[4:]:
                pairs += [(free[4], free[4]), (-1, free[4]), (n_pages, free[4]), (free[4], -3), (free[4], n_pages)]
            if pairs:
                s.copy([a for a, _ in pairs], [b for _, b in pairs])
        s.check()


def test_forks_of_a_shared_last_page(kvp):
    """All rows that hold it grow; all but one; one alone; a fork of forks; growth into the next page from inside a shared one."""
    s = Both(kvp, 6, 16, 4, 24)
    assert s.resize([20, 0, 0, 33, 0, 0]) == 0
    s.fork([0, 0, 0, 3, 3, 0])
    s.check()
    assert s.resize([21, 20, 22, 33, 34, 50]) == 0
    s.check()
    s.fork([5, 0, 1, 2, 3, 4])                                # every row goes on from another
    s.check()
    assert s.resize([x + 1 for x in s.book.lengths]) == 0
    s.check()
    s.fork([1, 1, 1, 1, 1, 1])
    assert s.resize([x + 17 for x in s.book.lengths]) == 0
    s.check()
    s.fork([-1] * 6)
    s.check()
    assert sum(s.book.refs) == 0


def test_a_page_that_a_shrinking_row_shares(kvp):
    """Shared at a full length, shortened into it, grown again: the other row's tokens stay."""
    s = Both(kvp, 2, 16, 4, 8)
    assert s.resize([32, 0]) == 0
    s.fork([0, 0])
    assert s.resize([30, 32]) == 0 and s.book.refs[1] == 2
    s.check()
    assert s.resize([31, 32]) == 0 and s.book.table[0][1] != s.book.table[1][1]
    s.check()


def test_too_few_pages_change_nothing(kvp):
    s = Both(kvp, 3, 16, 4, 6)
    assert s.resize([40, 20, 0]) == 0
    s.fork([0, 1, 1])
    assert s.resize([41, 21, 21]) == 0                        # one copy: the last page
    s.check()
    assert s.resize([49, 21, 21]) == 1
    s.check()
    assert s.resize([64, 64, 64]) == 1 + 2 + 2
    s.check()
    for to in ([41, -1, 21], [41, 65, 21], [(1 << 31) - 1, 21, 21], [-(1 << 31), 21, 21]):
        assert s.resize(to) == -1
        s.check()
    assert s.resize([0, 21, 21]) == 0 and s.resize([41, 21, 21]) == 0
    s.check()


def test_new_lengths_in_place(kvp):
    """The row's own lengths as the new ones: nothing changes."""
    s = Both(kvp, 3, 16, 4, 9)
    s.resize([10, 20, 30])
    kvp.pages_resize(s.desc, s.donor, s.lengths, s.refs, s.table, s.lengths, s.lacking, s.ws, *s.pools, *s.scales)
    s.check()
    assert s.lacking.tolist() == [0]


def test_places_without_a_page(kvp):
    """What a caller has put into a table beside pages is not taken for one."""
    s = Both(kvp, 2, 16, 4, 6)
    s.resize([40, 0])
    for x in (-1, -9, 6, 1 << 30):
        s.table[0, 2] = s.book.table[0][2] = x
        s.refs[2] = s.book.refs[2] = 0
        s.fork([0, 0])
        s.check()
        s.trim(3, 0)
        s.check()
        s.compact()
        s.check()
        s.resize([41, 42])
        s.check()
        s.fork([-1, -1])
        s.check()
        s.resize([40, 0])
        s.check()


def test_captured_calls(kvp):
    """A step in a graph: beams fork and grow; replayed, it goes on from what the last replay left."""
    s = Both(kvp, 6, 16, 8, 60, bits=8)
    s.resize([37] * 6)
    parents = [[0, 0, 2, 2, 4, 5], [1, 1, 0, 3, 3, 5], [5, 4, 3, 2, 1, 0]]
    parent, to = s.int32(parents[0]), s.int32([0] * 6)
    stream = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=stream):
        kvp.pages_fork(s.desc, parent, s.refs, s.table, s.lengths, s.ws)
        kvp.pages_resize(s.desc, s.donor, to, s.refs, s.table, s.lengths, s.lacking, s.ws, *s.pools, *s.scales)
        kvp.pages_compact(s.desc, s.donor, s.refs, s.table, s.lengths, s.used, s.ws, *s.pools, *s.scales)
    for i in range(6):
        parent.copy_(s.int32(parents[i % 3]))
        to.copy_(s.int32([38 + 3 * i] * 6))
        g.replay()
        s.book.fork(parents[i % 3])
        assert s.book.resize([38 + 3 * i] * 6) == 0
        s.book.compact()
        s.check()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 6)])
def test_a_serving_run(kvp, bits, window, sinks):
    """Prompts come in pieces, beams fork, drafts are taken back, pages behind the window are freed, the pool is made dense: after
    every step the new tokens' attention is that over the sequence's tokens as one piece of memory."""
    r, g = random.Random(3), torch.Generator(device="cuda").manual_seed(4)
    L, rows, Hq, Hkv, dh, page, max_pages, n_pages = 3, 5, 6, 2, 64, 16, 20, 70
    donor, owners = [0, 0, 2], [0, 2]
    desc = kvp.DecodeDesc(L, rows, Hq, Hkv, dh, page, max_pages, n_pages)
    zeros = lambda *s: torch.zeros(*s, dtype=I32, device="cuda")
    refs, table, lengths, lacking, used = zeros(n_pages), zeros(rows, max_pages) - 1, zeros(rows), zeros(1), zeros(1)
    nan = lambda: [torch.full((n_pages, Hkv, page, dh), float("nan"), device="cuda").to(E4M3 if bits == 8 else BF) if l in owners else None for l in range(L)]
    k, v = nan(), nan()
    scales = [[torch.full((n_pages, Hkv, page // 16), 255, dtype=U8, device="cuda") if l in owners else None for l in range(L)] for _ in range(2)] if bits == 8 else [None, None]
    held = dict(k_scale=scales[0], v_scale=scales[1])
    book_ws = torch.empty(kvp.pages_workspace_bytes(desc), dtype=U8, device="cuda")
    tokens = [[] for _ in range(rows)]                        # what each sequence consists of: (k, v) of the owners

    def step(new, rejected):
        """new[b] tokens join; the last rejected[b] of them are taken back afterwards."""
        old = [len(t) for t in tokens]
        kvp.pages_resize(desc, donor, torch.tensor([a + n for a, n in zip(old, new)], dtype=I32, device="cuda"), refs, table, lengths, lacking, book_ws, k, v, *scales)
        assert lacking.item() == 0
        first = [0]
        for n in new:
            first.append(first[-1] + n)
        T = first[-1]
        first = torch.tensor(first, dtype=I32, device="cuda")
        normal = lambda H: torch.randn(T, H, dh, device="cuda", dtype=BF, generator=g)
        k_new, v_new = ([normal(Hkv) if l in owners else None for l in range(L)] for _ in range(2))
        q = [normal(Hq) for _ in range(L)]
        kvp.cache_append_tokens(desc, donor, k_new, v_new, k, v, table, lengths, first=first, **held)
        o, lse = [torch.full_like(x, float("nan")) for x in q], [torch.full((T, Hq), float("nan"), device="cuda") for _ in range(L)]
        ws = torch.empty(kvp.attn_chunk_workspace_bytes(desc, donor, T), dtype=U8, device="cuda")
        kvp.attn_chunk(desc, donor, q, k, v, table, lengths, o, lse, ws, first=first, window=window, sinks=sinks, **held)
        at = 0
        for b, n in enumerate(new):
            tokens[b] += [{l: (k_new[l][at + i].double(), v_new[l][at + i].double()) for l in owners} for i in range(n)]
            for l in range(L) if n else ():
                kd, vd = (torch.stack([t[donor[l]][i] for t in tokens[b]], 1) for i in range(2))        # [Hkv, N, dh]
                pos, j = torch.arange(old[b], old[b] + n, device="cuda")[:, None], torch.arange(old[b] + n, device="cuda")
                seen = (j <= pos) & ((j > pos - window) | (j < sinks) if window else j >= 0)
                x = torch.einsum("thgd,hnd->thgn", q[l][at:at + n].double().unflatten(1, (Hkv, -1)), kd) * dh ** -0.5
                p = torch.softmax(torch.where(seen[:, None, None], x, -float("inf")), -1)
                want = torch.einsum("thgn,hnd->thgd", p, vd).flatten(1, 2)
                # 8 bits: numbers off by 2^-4 of themselves; scores by a normal sum of those, some 4 * 2^-4 of their spread
                a = torch.einsum("thgn,hnd->thgd", p, vd.abs()).flatten(1, 2)
                tol = a * 2.0 ** -7 + 2.0 ** -8 * want.abs() if bits == 16 else a * (2.0 ** -4 + 4 * 2.0 ** -4) + 2.0 ** -8
                assert ((o[l][at:at + n].double() - want).abs() <= tol).all()
            at += n
        for b, n in enumerate(rejected):
            del tokens[b][len(tokens[b]) - n:]
        kvp.pages_resize(desc, donor, torch.tensor([len(t) for t in tokens], dtype=I32, device="cuda"), refs, table, lengths, lacking, book_ws, k, v, *scales)
        if window:
            kvp.pages_trim(desc, window, sinks, refs, table, lengths)

    def fork(parent):
        kvp.pages_fork(desc, torch.tensor(parent, dtype=I32, device="cuda"), refs, table, lengths, book_ws)
        was = [list(t) for t in tokens]
        for b, p in enumerate(parent):
            tokens[b] = list(was[p]) if p >= 0 else []

    step([50, 0, 33, 0, 1], [0] * 5)
    step([20, 0, 70, 0, 1], [0] * 5)                          # the rest of the prompts
    fork([0, 0, 2, 2, 4])
    step([1, 1, 1, 1, 1], [0] * 5)
    step([5, 4, 5, 3, 1], [2, 4, 0, 3, 0])                    # drafts
    fork([1, 0, 3, 3, -1])
    step([1, 1, 1, 1, 30], [0] * 5)
    kvp.pages_compact(desc, donor, refs, table, lengths, used, book_ws, k, v, *scales)
    assert (refs[:used.item()] > 0).all() and (refs[used.item():] == 0).all()
    step([1, 1, 17, 1, 30], [0, 0, 9, 0, 0])
    fork([-1, 1, 2, 1, 1])
    for _ in range(4):
        step([r.randint(0, 12) for _ in range(rows)], [0] * 5)
        fork([r.choice((b, b, (b + 1) % rows)) for b in range(rows)])
        kvp.pages_compact(desc, donor, refs, table, lengths, used, book_ws, k, v, *scales)
    count = torch.zeros(n_pages, dtype=I32, device="cuda")
    for b, t in enumerate(tokens):
        for p in table[b, :-(-len(t) // page)].tolist():
            if p >= 0:
                count[p] += 1
    assert torch.equal(count, refs) and kvp.device_status() == kvp.OK
