// How the row kernels (k_quant.hip) share a session's list out to workgroups. Plain C++: no HIP
// in here.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace ikv {

constexpr int QT = 256;                    // threads per workgroup
constexpr int QU = 2;                      // places of a thread at a time
constexpr int QUANT_MOST = (1 << 24) - 1;  // rows of a session in one call: a workgroup or more each, under 2^32 threads

// Entries of a workgroup: QU places per thread, one entry at least. `per` = Hkv D / 8 places an
// entry, 8 channels of its K and of its V row each.
constexpr int quant_group(int per) { return std::max(1, QT * QU / per); }

// Workgroups that a launch has at most (or one a session and layer). The host knows the lists' room, N, not
// n_rows: past these the workgroups stride over the list and end with its rows. Launching them is what
// idle ones cost, 0.2 ns each (one row each of 64 sessions with room for 8201, 36 layers x 8 heads: 996 us
// uncapped, 33 with 2^17); striding over full lists costs balance at the end (8189 rows in 4 bits, stored and
// read back: 498 us uncapped, 498 with 2^17, 509 with 2^16, 522 with 2^15, 554 with 2^14). Rows that come
// from a pool of new rows (no src) are mostly a step's few: one session's token 18.6 us with 2^17, 10.0
// with 2^15.
constexpr int QUANT_GRID = 1 << 17, QUANT_GRID_NEW = 1 << 15;

// Bytes of the pool's rows, K and V, up to which a store's rows and codes, and a load's rows, go through the
// caches (256 MB): the decode after a store, and the one over rows read back, then find them there. Store and
// decode, load and decode, E4M3, 36 layers x 8 heads, us through the caches / past them: 500 rows (74 MB)
// 33 / 39, 36.5 / 41; 1021 (150) 59 / 64, 72 / 67; 1800 (265) 101 / 104, 114 / 113; 3000 (442) 173 / 168,
// 203 / 192; 8192 (1208) 491 / 458, 593 / 522. In 4 bits 1021: 47 / 53, 65 / 62; 2300: 105 / 102, 137 / 126.
constexpr double QUANT_STORE_KEPT = 256 << 20, QUANT_LOAD_KEPT = 128 << 20;

// Workgroups of each of `units` sessions and layers, lists of up to `longest` entries.
constexpr int quant_groups(int longest, int group, int64_t units, int most) {
  return int(std::max<int64_t>(1, std::min<int64_t>((int64_t(longest) + group - 1) / group, most / units)));
}

// Places of the workgroup whose first entry is k0, in a list of `rows`. Past the list there are
// none: the product comes after that, since a deficit of millions of entries times `per` would
// pass 32 bits and could come out positive.
constexpr int quant_places(int group, int rows, int k0, int per) {
  const int left = std::min(group, rows - k0);
  return left > 0 ? left * per : 0;
}

}  // namespace ikv
