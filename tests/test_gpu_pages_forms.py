"""Pages of the cache: as many rows as a call takes, large books in captured graphs, numbers that the kernel ahead is still writing."""
import random

import pytest
import torch

from ahead import Ahead
from test_gpu_pages import Both, kvp  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu
I32 = torch.int32


def test_the_most_rows(kvp):
    """All rows go on from one, and all but some of them grow inside its last page; then each gives back what it has."""
    rows = 1 << 14
    s = Both(kvp, rows, 16, 3, rows + 50, (0,), 1, 64)
    assert s.resize([20] + [0] * (rows - 1)) == 0
    s.fork([0] * rows)
    assert s.book.refs[:2] == [rows, rows]
    to = [21 if b % 1000 else 20 for b in range(rows)]
    # (the oracle's loop over all pairs of rows, without the loop: page 1 is held by more than grow, so every row that grows takes a copy)
    s.kvp.pages_resize(s.desc, s.donor, s.int32(to), s.refs, s.table, s.lengths, s.lacking, s.ws, *s.pools, *s.scales)
    page = 2
    for b in range(rows):
        if to[b] == 21:
            s.book.table[b][1], s.book.refs[page], s.book.content[page] = page, 1, 1
            page += 1
    s.book.refs[1], s.book.lengths = rows - (page - 2), to
    assert s.lacking.tolist() == [0]
    s.check()
    s.fork([-1 if b % 3 else b for b in range(rows)])
    s.check()
    s.compact()
    s.check()
    s.trim(1, 0)
    s.check()


@pytest.mark.parametrize("rows,max_pages,n_pages", [(5, 6, 40), (300, 30, 9000)])
@pytest.mark.parametrize("bits", [16, 8])
def test_two_graphs_in_turn(kvp, rows, max_pages, n_pages, bits):
    """Growth in one, forks and a dense pool in the other, on one workspace; replayed from whatever the last replay left."""
    r = random.Random(rows)
    s = Both(kvp, rows, 16, max_pages, n_pages, (0, 1, 1), 1, 64, bits)
    parent, to = s.int32([0] * rows), s.int32([0] * rows)
    torch.cuda.synchronize()
    grow, turn = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(grow):
        kvp.pages_resize(s.desc, s.donor, to, s.refs, s.table, s.lengths, s.lacking, s.ws, *s.pools, *s.scales)
        kvp.pages_trim(s.desc, 40, 3, s.refs, s.table, s.lengths)
    with torch.cuda.graph(turn):
        kvp.pages_fork(s.desc, parent, s.refs, s.table, s.lengths, s.ws)
        kvp.pages_compact(s.desc, s.donor, s.refs, s.table, s.lengths, s.used, s.ws, *s.pools, *s.scales)
    for _ in range(5):
        new = [min(16 * max_pages, max(0, n + r.randint(-20, 60))) for n in s.book.lengths]
        to.copy_(s.int32(new))
        grow.replay()
        assert s.book.resize(new) == 0
        s.book.trim(40, 3)
        s.check()
        parents = [r.choice((b, b, b, -1, r.randrange(rows))) for b in range(rows)]
        parent.copy_(s.int32(parents))
        turn.replay()
        s.book.fork(parents)
        s.book.compact()
        s.check()


@pytest.mark.parametrize("rows,max_pages,n_pages", [(130, 12, 2500), (300, 70, 9000)])
def test_numbers_that_a_kernel_of_the_library_writes(kvp, rows, max_pages, n_pages):
    """Parents and new lengths that the kernel ahead is still writing when the call comes up."""
    r = random.Random(rows)
    s = Both(kvp, rows, 16, max_pages, n_pages, (0,), 1, 64)
    number = lambda: r.choice((0, r.randint(128, 180)))       # (what the kernel ahead can write)
    state = lambda: ([number() for _ in range(rows)], [r.choice((0, 0, 128, 129 if rows > 129 else 128)) for _ in range(rows)])
    two = [state(), state()]
    ahead = Ahead(kvp, *[[torch.tensor(x, dtype=I32) for x in st] for st in two])
    torch.cuda.synchronize()
    for i in range(6):
        to, parents = two[i % 2]
        ahead.write(i)
        kvp.pages_resize(s.desc, s.donor, ahead.views[0], s.refs, s.table, s.lengths, s.lacking, s.ws, *s.pools, *s.scales)
        ahead.write(i + 1)
        ahead.write(i)
        kvp.pages_fork(s.desc, ahead.views[1], s.refs, s.table, s.lengths, s.ws)
        assert s.book.resize(to) == 0
        s.book.fork(parents)
        s.check()
