// Attention kernels: bf16 queries, bf16 blocks, first keys beside a window.
#include "kv_attend_launch.hip.h"

template void tutti::launch_attend<tutti::Bf16, false, true>(const tutti::AttendArgs &, uint32_t, hipStream_t);
