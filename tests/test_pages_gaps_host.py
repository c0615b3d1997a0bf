"""The pages' oracle where a row grows inside a place that holds no page."""
from oracle.pages import Book


def test_a_row_that_grows_inside_a_freed_place():
    book = Book(16, 4, 8, 2)
    assert book.resize([64, 20]) == 0 and book.table == [[0, 1, 2, 3], [4, 5, -1, -1]]
    book.trim(5, 0)                                           # of 64 tokens the last 4 are seen, of 20 all behind place 0
    assert book.table == [[-1, -1, -1, 3], [-1, 5, -1, -1]]
    assert book.resize([40, 20]) == 0                         # into a freed place
    assert book.table[0] == [-1, -1, -1, -1] and book.refs == [0, 0, 0, 0, 0, 1, 0, 0]
    assert book.resize([40, 21]) == 0 and book.table[0] == [-1] * 4          # (it does not grow)
    assert book.resize([41, 21]) == 0                         # grows in it: a page there, nothing copied
    assert book.table[0] == [-1, -1, 0, -1] and book.refs[0] == 1 and book.content == list(range(8))
    assert book.resize([60, 21]) == 0 and book.table[0] == [-1, -1, 0, 1]
    assert book.consistent()


def test_order_and_lack():
    book = Book(16, 4, 6, 3)
    assert book.resize([32, 32, 20]) == 0                     # six pages
    book.trim(1, 0)
    assert book.table[2][:2] == [-1, 5] and book.refs == [0, 0, 0, 0, 0, 1]
    assert book.resize([20, 25, 20]) == 0
    book.fork([0, 1, 2])
    assert book.resize([40, 26, 64]) == 0                     # row 0 a place and one behind it, row 1 a place, row 2 two behind
    assert [t[:4] for t in book.table] == [[-1, 0, 1, -1], [-1, 2, -1, -1], [-1, 5, 3, 4]]
    book.trim(1, 0)                                           # (26 and 40 stay in their places; 64 are all freed)
    assert book.refs == [0, 1, 1, 0, 0, 0] and book.resize([40, 26, 50]) == 0
    before = [list(t) for t in book.table]
    assert book.resize([64, 64, 64]) == (1 + 2 + 1) - 4 and book.consistent()
    assert before[2] == [-1] * 4 and book.table[2] == [-1, -1, -1, 5]
    assert book.table[0] == [-1, -1, 1, 0] and book.table[1] == [-1, 2, 3, 4]
