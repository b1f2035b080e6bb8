// Attention kernels: fp16 queries, fp16 blocks, first keys beside a window.
#include "kv_attend_launch.hip.h"

template void tutti::launch_attend<tutti::Fp16, false, true>(const tutti::AttendArgs &, uint32_t, hipStream_t);
