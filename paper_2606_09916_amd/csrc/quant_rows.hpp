// How the row kernels (k_quant.hip) share a session's list out to workgroups. Plain C++: no HIP
// in here.
#pragma once

#include <algorithm>

namespace ikv {

constexpr int QT = 256;                    // threads per workgroup
constexpr int QU = 2;                      // places of a thread at a time
constexpr int QUANT_MOST = (1 << 24) - 1;  // rows of a session in one call: a workgroup or more each, under 2^32 threads

// Entries of a workgroup: QU places per thread, one entry at least. `per` = Hkv D / 8 places an
// entry, 8 channels of its K and of its V row each.
constexpr int quant_group(int per) { return std::max(1, QT * QU / per); }

// Places of the workgroup whose first entry is k0, in a list of `rows`. Past the list there are
// none: the product comes after that, since a deficit of millions of entries times `per` would
// pass 32 bits and could come out positive.
constexpr int quant_places(int group, int rows, int k0, int per) {
  const int left = std::min(group, rows - k0);
  return left > 0 ? left * per : 0;
}

}  // namespace ikv
