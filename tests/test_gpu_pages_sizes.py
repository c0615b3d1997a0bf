"""Pages of the cache on both sides of the sizes at which one block, or its threads' registers, hold the whole book."""
import pytest

from test_gpu_pages import kvp, test_random_runs as random_run  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,page,max_pages,n_pages", [
    (1, 16, 1, 1),
    (2, 16, 40, 33),                 # rows of more places than a warp has lanes
    (128, 16, 32, 1500),             # as many places as are kept
    (129, 16, 32, 1500),             # and one row more, of one block still
    (32, 16, 128, 2047),
    (4, 16, 1000, 1024),
    (4, 16, 1025, 1025),
    (20, 16, 60, 8192),              # as many pages as are kept
    (20, 16, 60, 8193),
    (200, 16, 5, 800),
])
@pytest.mark.parametrize("bits", [16, 8])
def test_sizes_of_the_book(kvp, rows, page, max_pages, n_pages, bits):
    random_run(kvp, rows, page, max_pages, n_pages, (0, 0), 1, 64, bits)
