// Which rows of a batch are a request's: plain code, no HIP.
#pragma once

namespace ks {

struct RowsRange { int first, n; };

// Rows of request r: row_start[r] .. row_start[r+1]-1, as far as the batch has them, whatever row_start holds: 0 <= first, 0 <= n, first + n <= n_rows for a
// range that is not empty. Both ends are brought into the batch before one is taken from the other: entries near the two ends of 32 bits would wrap into a
// range far outside.
template <typename P> constexpr RowsRange rows_of(P row_start, int r, int n_rows) {
    const int a = row_start[r], b = row_start[r + 1];
    const int first = a < 0 ? 0 : (a < n_rows ? a : n_rows), end = b < first ? first : (b < n_rows ? b : n_rows);
    return {first, end - first};
}

}  // namespace ks
