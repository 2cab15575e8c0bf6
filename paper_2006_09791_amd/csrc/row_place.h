// Which eight columns of a dense row a lane has, and where they lie.  Host and device, without a header of HIP: a test checks the arithmetic with the
// host's compiler.
#pragma once

#include <stddef.h>

#include "divide.h"

namespace gspc {

// Eight columns of a row from `at` on, of which the first n (8, fewer at the row's end, or none) are there.  In rows of whole eights (kWhole) n is 8 or
// 0.  What is there at the end of others (kRagged) is read as the row's last eight columns, in one access, and moved to its place when it is widened;
// rows of fewer than eight columns (kThin) are read one by one.  Lanes without a column read the row's first ones: no load hangs on a branch, behind
// which a wait for older loads would have to be one for all.
enum Rows { kWhole, kRagged, kThin };
inline Rows rows_of(int cols) { return cols % 8 == 0 ? kWhole : cols > 8 ? kRagged : kThin; }
struct Place {
    unsigned at, start;         // start: of what is read
    int n, shift;
};
GSPC_HD Place place_of(int at, int cols) {
    const int left = cols - at;
    Place p;
    p.at = at;
    p.n = left < 0 ? 0 : left > 8 ? 8 : left;
    p.shift = p.n > 0 ? 8 - p.n : 0;
    p.start = p.n > 0 ? at - p.shift : 0;
    return p;
}

// Bytes from a row's first column to another one, of `size` bytes each.  LONG: in 64 bits, for rows that may be of 2^32 bytes and more (fp32 from 2^30
// columns on); else in 32, the form that needs one register of address beside a row's, where that is the same for a wave.
template <bool LONG> struct ColumnBytes { typedef unsigned type; };
template <> struct ColumnBytes<true> { typedef size_t type; };
template <bool LONG> GSPC_HD typename ColumnBytes<LONG>::type column_bytes(unsigned column, unsigned size) {
    return (typename ColumnBytes<LONG>::type)column * size;
}

}  // namespace gspc
