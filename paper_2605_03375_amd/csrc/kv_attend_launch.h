// What the attention kernels' own sources give tutti_kv_attend's: one function for each type of queries, pool and kind of window.
#pragma once
#include "kv_attend.hip.h"

namespace tutti {

// rows: of queries that a workgroup takes, 16, 32 or 128
template <typename T, bool E4M3, bool SINKS>
__attribute__((visibility("hidden"))) void launch_attend(const AttendArgs &a, uint32_t rows, hipStream_t stream);

}  // namespace tutti
