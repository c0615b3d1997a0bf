"""How the rows of attention of new tokens are counted, compiled for the host: up to the most that a call takes."""
import ctypes as C
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_15943_b200", "csrc")
MOST_TOKENS, TILE = (1 << 24) - 1, 128


@pytest.fixture(scope="module")
def rows(tmp_path_factory):
    d = tmp_path_factory.mktemp("rows")
    (d / "rows.cpp").write_text('#include "kvp_chunk_rows.h"\n'
                                'extern "C" int units(int r) { return kvp::units_of_rows(r); }\n'
                                'extern "C" int token(int n, int r) { return kvp::rows_of_token(n).token(r); }\n'
                                'extern "C" int most() { return kvp::CHUNK_MOST_TOKENS; }\n'
                                'extern "C" int tile() { return kvp::CHUNK_TILE; }\n')
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I" + CSRC, str(d / "rows.cpp"), "-o", str(d / "rows.so")], check=True)
    return C.CDLL(str(d / "rows.so"))


def test_units(rows):
    assert rows.most() == MOST_TOKENS and rows.tile() == TILE
    r = random.Random(2)
    largest = MOST_TOKENS * TILE
    for n in [0, 1, 255, 256, 257, largest, largest - 1, largest - 127, largest - 128, largest - 129, largest - 255, largest - 256] + [r.randint(0, largest) for _ in range(20000)]:
        assert rows.units(n) == -(-n // 256), n
    # every row of the last unit, those that it has not among them, is a number of 31 bits
    assert rows.units(largest) * 256 - 1 <= (1 << 31) - 1


@pytest.mark.parametrize("n", list(range(1, 129)))
def test_tokens_of_rows(rows, n):
    r = random.Random(n)
    last = rows.units(MOST_TOKENS * n) * 256 - 1
    near = [k * n + d for k in [0, 1, 2, MOST_TOKENS - 1, MOST_TOKENS] + [r.randint(0, MOST_TOKENS) for _ in range(500)] for d in (-1, 0, 1)]
    for row in [0, last] + [x for x in near if 0 <= x <= last]:
        assert rows.token(n, row) == row // n, row
