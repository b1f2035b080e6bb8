// Attention kernels: fp16 queries, e4m3 blocks, first keys beside a window.
#include "kv_attend_launch.hip.h"

template void tutti::launch_attend<tutti::Fp16, true, true>(const tutti::AttendArgs &, uint32_t, hipStream_t);
