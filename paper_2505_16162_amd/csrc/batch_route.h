// Which kernel a batch over pages in bf16 goes to: plain code, no HIP.
#pragma once
#include <climits>
#include <cstdint>

namespace ks {

// Most (row, head) pairs of one kv head that a request may have for battn_few_kernel to take the batch: as many as one group holds; each further group reads the cache
// again. Whole calls, us, few rows / tiles, 32 requests at 200 to 4000 positions, bf16 queries; fp32 ones (whose tiles do three times the products):
//   40 heads of 128 over 8: 5 pairs 62 / 68; 59 / 83, 10 to 15 64 / 72; 67 / 91, 20 77 / 57; 104 / 88, 20 to 30 92 / 63; 85 / 78, 35 to 60 133 / 64; 189 / 118
//   40 over 40: 1 pair 233 / 271; 240 / 296, 16 293 / 306; 286 / 339, 20 527 / 319; 557 / 404, 60 972 / 384; 1011 / 433
//   32 heads of 64 over 8: 8 to 12 29 / 31; 34 / 52, 16 34 / 39; 40 / 54, 16 to 24 42 / 38; 51 / 57, 28 to 48 58 / 37; 70 / 64
// Two requests of 20 to 30 pairs at 100 000 positions 223 / 157; 227 / 167. The bound is the caller's most_rows, or all rows of the batch.
constexpr int FEW_PAIRS = 16;

// positions of a unit of battn_few_kernel: 8 KB of keys, 8 KB of values, which a wavefront holds in registers
constexpr int few_positions(int head_dim) { return 32 * 128 / head_dim; }

// groups of pairs of a kv head, and what battn_few_kernel has to do with them, at most: blocks of positions for every group
constexpr int64_t few_groups(int64_t n_rows, int group, int n_requests) { return (n_rows * group + FEW_PAIRS - 1) / FEW_PAIRS + n_requests; }
constexpr int64_t few_units(int64_t positions, int head_dim, int64_t groups, int n_kv_heads) {
    const int64_t blocks = (positions + few_positions(head_dim) - 1) / few_positions(head_dim);
    return blocks < INT32_MAX ? blocks * groups * n_kv_heads : INT64_MAX;
}

// Trees have many pairs from the start, but few trees over short contexts are done before a tile's first block is: whole calls, us, battn_few_kernel / tiles, one request, 40 heads of 128 over 8, bf16:
//   26 rows over 400 positions 16 / 25, 1500 21 / 24, 3000 (7600 units) 24 / 27, 6000 (15 000) 30 / 29; 60 rows 400 16 / 26, 1500 (8400) 23 / 28, 3000 (16 000) 31 / 31, 6000 44 / 33
//   40 heads over 40: 60 rows over 1500 (9900) 24 / 28; four requests of 26 rows over 1500 (15 000) 30 / 29
// The positions are those that the table can hold, the rows those of the arrays: under a table for far longer contexts the same trees take the tiles' time.
constexpr int64_t FEW_UNITS = 12288;

// positions: what a request's table can hold; most: pairs of a request and kv head, at most
constexpr bool goes_to_few(bool trees, int64_t positions, int head_dim, int64_t n_rows, int group, int n_requests, int n_kv_heads, int64_t most) {
    return most <= FEW_PAIRS || (trees && few_units(positions, head_dim, few_groups(n_rows, group, n_requests), n_kv_heads) <= FEW_UNITS);
}

}  // namespace ks
