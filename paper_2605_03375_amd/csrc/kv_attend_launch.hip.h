// Launches of the attention kernels.  A source of its own for each type of queries, pool and kind of window (kv_attend_*.hip) makes
// them: compiled side by side they take a sixth of the time.
#pragma once
#include <algorithm>

#include "kv_attend_launch.h"

namespace tutti {
namespace {

template <typename T, bool E4M3, bool SINKS, int DP, bool PAGED16, int RT>
void launch_few(const AttendArgs &a, hipStream_t stream) {
  const dim3 grid(a.max_units), wg(64 * a.abreast * a.key_waves);
  if (a.d == DP)
    hipLaunchKernelGGL((k_kv_attend<T, E4M3, DP, true, PAGED16, RT, SINKS>), grid, wg, 0, stream, a);
  else
    hipLaunchKernelGGL((k_kv_attend<T, E4M3, DP, false, PAGED16, RT, SINKS>), grid, wg, 0, stream, a);
}
template <typename T, bool E4M3, bool SINKS, int DP, int ROWS>
void launch_join(const AttendArgs &a, hipStream_t stream) {
  if (SINKS && a.most_tiles <= a.min_tiles) return;  // nothing is split
  // a sequence that is split has two parts or more to a row tile, so no more rows are to be joined than this
  const uint32_t joins = std::min(a.batch.n_rows * a.kv_heads * a.group, a.max_parts / 2 * ROWS);
  // A workgroup a row for few rows, which may have many parts (32 rows of 128 parts: one wavefront, part after part, 75 us, four
  // wavefronts 6.7, 16 wavefronts 6.2, but 1,280 rows of some parts 7.5 and 21); else a wavefront a row (1,511 queries of 20 heads in
  // two parts: 20 us, with workgroups 61), 8192 at a time (8,001 prompt tokens that are not split: 5 us, with a wavefront for each row
  // that there might be 21).
  // (SINKS, whose windows bound the parts of a row: 2,048 rows of four parts, workgroups 7.9 us, wavefronts 5.)
  if (joins <= (SINKS && a.most_tiles <= 32 * a.min_tiles ? 1024 : 4096))
    hipLaunchKernelGGL((k_kv_join<T, E4M3, DP, ROWS, 4, SINKS>), dim3(joins), dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((k_kv_join<T, E4M3, DP, ROWS, 1, SINKS>), dim3(2048), dim3(256), 0, stream, a);
}
template <typename T, bool E4M3, bool SINKS, bool PAGED16>
void launch_wide(const AttendArgs &a, hipStream_t stream) {
  const dim3 grid(a.max_units), wg(256);
  if (a.d == 128)
    hipLaunchKernelGGL((k_kv_attend_wide<T, E4M3, 128, true, PAGED16, SINKS>), grid, wg, 0, stream, a);
  else if (a.d == 112)
    hipLaunchKernelGGL((k_kv_attend_wide<T, E4M3, 112, true, PAGED16, SINKS>), grid, wg, 0, stream, a);
  else if (a.d == 96)
    hipLaunchKernelGGL((k_kv_attend_wide<T, E4M3, 96, true, PAGED16, SINKS>), grid, wg, 0, stream, a);
  else if (a.d == 80)
    hipLaunchKernelGGL((k_kv_attend_wide<T, E4M3, 80, true, PAGED16, SINKS>), grid, wg, 0, stream, a);
  else if (a.d == 64)
    hipLaunchKernelGGL((k_kv_attend_wide<T, E4M3, 64, true, PAGED16, SINKS>), grid, wg, 0, stream, a);
  else
    hipLaunchKernelGGL((k_kv_attend_wide<T, E4M3, 64, false, PAGED16, SINKS>), grid, wg, 0, stream, a);
}
template <typename T, bool E4M3, bool SINKS, int DP>
void launch_size(const AttendArgs &a, uint32_t rows, hipStream_t stream) {
  const bool paged16 = a.pool.block_tokens % 16 == 0;
  if (rows == 128) {
    paged16 ? launch_wide<T, E4M3, SINKS, true>(a, stream) : launch_wide<T, E4M3, SINKS, false>(a, stream);
    launch_join<T, E4M3, SINKS, DP, 128>(a, stream);
    return;
  }
  if (paged16)
    rows == 16 ? launch_few<T, E4M3, SINKS, DP, true, 1>(a, stream) : launch_few<T, E4M3, SINKS, DP, true, 2>(a, stream);
  else
    rows == 16 ? launch_few<T, E4M3, SINKS, DP, false, 1>(a, stream) : launch_few<T, E4M3, SINKS, DP, false, 2>(a, stream);
  rows == 16 ? launch_join<T, E4M3, SINKS, DP, 16>(a, stream) : launch_join<T, E4M3, SINKS, DP, 32>(a, stream);
}

}  // namespace

template <typename T, bool E4M3, bool SINKS>
void launch_attend(const AttendArgs &a, uint32_t rows, hipStream_t stream) {
  a.d <= 64 ? launch_size<T, E4M3, SINKS, 64>(a, rows, stream) : launch_size<T, E4M3, SINKS, 128>(a, rows, stream);
}

}  // namespace tutti
