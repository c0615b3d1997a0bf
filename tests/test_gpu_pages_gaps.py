"""Rows that grow inside a place without a page (one that was freed behind a window before the row shrank into it) against the oracle."""
import random

import pytest
import torch

from test_gpu_pages import Both, kvp  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu
BF, I32 = torch.bfloat16, torch.int32


@pytest.mark.parametrize("rows,page,max_pages,n_pages", [
    (3, 16, 6, 30),
    (100, 32, 8, 900),               # kept by the threads of one block
    (300, 16, 40, 9000),             # a cluster of blocks
    (1300, 16, 10, 6000),            # more rows than a block has threads
])
@pytest.mark.parametrize("bits", [16, 8])
def test_trim_shrink_grow(kvp, rows, page, max_pages, n_pages, bits):
    r = random.Random(rows)
    s = Both(kvp, rows, page, max_pages, n_pages, (0, 0), 1, 64, bits)
    cap = max_pages * page
    some = lambda lo, hi: [r.randint(lo, hi) for _ in range(rows)]
    for step in range(6):
        s.resize([min(cap, max(x, y)) for x, y in zip(s.book.lengths, some(cap // 3, cap // 2))])
        s.check()
        s.trim(r.choice((1, 3, page + 5)), r.choice((0, 0, 1, page + 1)))
        s.check()
        s.resize([r.choice((x, r.randint(0, x))) for x in s.book.lengths])
        s.check()
        if step % 2:
            s.fork([r.choice((b, b, r.randrange(rows))) for b in range(rows)])
            s.check()
        s.resize([min(cap, x + r.choice((0, 1, 2, page, 2 * page))) for x in s.book.lengths])
        s.check()
        if step % 3 == 2:
            s.compact()
            s.check()


def test_too_few_pages_for_a_place(kvp):
    """The page of a place counts among those that are lacking; then nothing is changed."""
    s = Both(kvp, 2, 16, 4, 4)
    assert s.resize([30, 20]) == 0
    s.trim(1, 0)                                              # place 0 of both
    s.check()
    assert s.resize([10, 64]) == 0                            # row 0 gives up its second page, row 1 takes two
    s.check()
    assert sum(x == 0 for x in s.book.refs) == 1
    assert s.resize([33, 64]) == 2                            # a place, and two behind it
    s.check()
    assert s.resize([16, 64]) == 0 and s.book.table[0][0] >= 0
    s.check()


@pytest.mark.parametrize("few", [True, False])
def test_what_is_appended_there_is_kept(kvp, few):
    """A window of one token: a row's output is its own V."""
    rows, page, max_pages, n_pages = (3, 16, 4, 12) if few else (200, 16, 40, 3000)
    desc = kvp.DecodeDesc(1, rows, 1, 1, 64, page, max_pages, n_pages)
    zeros = lambda *s: torch.zeros(*s, dtype=I32, device="cuda")
    refs, table, lengths, lacking = zeros(n_pages), zeros(rows, max_pages) - 1, zeros(rows), zeros(1)
    k, v = ([torch.zeros(n_pages, 1, page, 64, dtype=BF, device="cuda")] for _ in range(2))
    ws = torch.empty(kvp.pages_workspace_bytes(desc), dtype=torch.uint8, device="cuda")

    def resize(to):
        kvp.pages_resize(desc, [0], torch.tensor(to, dtype=I32, device="cuda"), refs, table, lengths, lacking, ws, k, v)
        assert lacking.item() == 0

    resize([60] * rows)
    kvp.pages_trim(desc, 2, 0, refs, table, lengths)
    resize([20 + b % 3 for b in range(rows)])
    resize([22 + b % 3 for b in range(rows)])                 # two tokens each
    first = torch.arange(0, 2 * rows + 1, 2, dtype=I32, device="cuda")
    new = lambda: [torch.randn(2 * rows, 1, 64, dtype=BF, device="cuda")]
    k_new, v_new, q, o, lse = new(), new(), new(), new(), [torch.empty(2 * rows, 1, device="cuda")]
    kvp.cache_append_tokens(desc, [0], k_new, v_new, k, v, table, lengths, first=first)
    aws = torch.empty(kvp.attn_chunk_workspace_bytes(desc, [0], 2 * rows), dtype=torch.uint8, device="cuda")
    kvp.attn_chunk(desc, [0], q, k, v, table, lengths, o, lse, aws, first=first, window=1)
    assert torch.equal(o[0], v_new[0])
