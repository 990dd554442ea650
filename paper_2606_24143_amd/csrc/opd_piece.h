// Where a lane reads its 16 bytes of a row.  Internal; no device code: tests compile it
// for the host.
#pragma once

#include <cstdint>

namespace opd {

// Column of the 16-byte piece `piece` (of EACH columns) of a step that begins at column d, in a
// row that ends at column `end`, 1 at least; past the end, of the last piece that begins before
// it.  d is a multiple of EACH.  So what is read lies in [0, end), rounded up to whole pieces.
template <int EACH>
constexpr int64_t piece_column(int64_t d, int piece, int64_t end) {
  const int64_t c = d + (int64_t)piece * EACH, last = (end - 1) / EACH * EACH;
  return c < last ? c : last;
}

}  // namespace opd
