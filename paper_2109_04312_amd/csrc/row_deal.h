// Which rows of a [rows, E] tensor a workgroup of the elementwise passes takes.  (For the host too: a test deals the largest tensors.)
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>

namespace mate {

constexpr int kRowThreads = 256;
constexpr int kUnit = 8;   // features of a thread at a time
// A dimension of a launch has fewer than 2^32 threads (4104 wide and more, which are a row a workgroup, reach that with 2^24 rows): what is more
// than half of them goes on in the second one.
constexpr int kGroupsAcrossLog2 = 23;

struct RowDeal {
  int rows, E;
  int each;            // rows of a workgroup
  unsigned units, by;  // of a row, whole scale blocks; 2^32 / units, rounded up
};
inline RowDeal deal_rows(int rows, int E, int block /* features */) {
  RowDeal d;
  d.rows = rows;
  d.E = E;
  d.units = (unsigned)(block / kUnit) * (unsigned)((E + block - 1) / block);
  d.by = (unsigned)(((1ull << 32) + d.units - 1) / d.units);
  // four units a thread once there are enough for the chip: their loads travel together
  const size_t total = (size_t)rows * d.units;
  const unsigned want = total >= (size_t)4 * kRowThreads * 1024 ? 4 * kRowThreads : kRowThreads;
  d.each = (int)std::max(1u, want / d.units);
  return d;
}
inline dim3 groups_of(const RowDeal& d) {
  const long groups = (d.rows + (long)d.each - 1) / d.each, across = 1l << kGroupsAcrossLog2;
  return dim3((unsigned)std::min(groups, across), (unsigned)((groups + across - 1) / across));
}
// A workgroup's first row, and how many it has (none or less: it is past the last one).
__host__ __device__ inline long first_row(const RowDeal& d, unsigned x, unsigned y) { return (long)(((size_t)y << kGroupsAcrossLog2) + x) * d.each; }
__host__ __device__ inline int rows_from(const RowDeal& d, long first) { return d.rows - first < d.each ? (int)(d.rows - first) : d.each; }

}  // namespace mate
