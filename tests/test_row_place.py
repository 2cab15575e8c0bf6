"""Which columns of a row a lane has, and where they lie (csrc/row_place.h), with the host's compiler, up to the longest rows there are."""
import subprocess

import pytest

from paper_2006_09791_amd import build

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "row_place.h"
using namespace gspc;

int main(int, char **a) {
    const long long cols = std::atoll(a[1]);
    const unsigned size = (unsigned)std::atoi(a[2]);
    const bool is_long = std::atoi(a[3]);
    for (int k = 4; a[k]; ++k) {
        const Place p = place_of(std::atoi(a[k]), (int)cols);
        const unsigned long long read = is_long ? column_bytes<true>(p.start, size) : column_bytes<false>(p.start, size);
        const unsigned long long written = is_long ? column_bytes<true>(p.at, size) : column_bytes<false>(p.at, size);
        std::printf("%d %llu %llu\n", p.n, read, written);
    }
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("row_place")
    (d / "row_place.cpp").write_text(PROGRAM)
    exe = str(d / "row_place")
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", build.CSRC, str(d / "row_place.cpp"), "-o", exe], check=True)
    return exe


@pytest.mark.parametrize("cols", [8, 9, 15, 24, 60, 8192, (1 << 30) - 1, 1 << 30, (1 << 30) + 1, (1 << 30) + 136, (1 << 31) - 1024, 0x7ffffff0])
@pytest.mark.parametrize("size", [2, 4])
def test_columns_lie_where_the_rows_have_them(program, cols, size):
    """Vectors at both ends and around 2^32 bytes: what is read ends with the row, what is written begins at its column."""
    last = (cols + 7) // 8 * 8
    at = sorted({v * 8 for mid in (0, last // 8, (1 << 32) // size // 8) for v in range(mid - 4, mid + 4) if 0 <= v * 8 <= last and v * 8 < 1 << 31})
    for is_long in ([True] if cols * size >= 1 << 32 else [True, False]):
        out = subprocess.run([program, str(cols), str(size), str(int(is_long)), *map(str, at)], check=True, capture_output=True, text=True).stdout.split("\n")
        for a, line in zip(at, out):
            n, read, written = map(int, line.split())
            assert n == max(0, min(8, cols - a)) and read == (min(a, cols - 8) * size if n else 0)
            assert written == a * size or n == 0            # (nothing is written there)


@pytest.mark.parametrize("name", ["rows_f8_kernels.hip", "dropout_kernels.hip"])
def test_rows_of_any_length_are_read_and_written_in_64_bits(name):
    """The kernels whose rows may be of 2^32 bytes and more take no other form."""
    with open(f"{build.CSRC}/{name}") as f:
        text = f.read()
    for call in ("fetch_some<", "store_some<"):
        assert text.count(call) == text.count(call + "ROWS, true>") > 0
    assert "beyond(" not in text
