// Attention kernels: fp16 queries, fp16 blocks.
#include "kv_attend_launch.hip.h"

template void tutti::launch_attend<tutti::Fp16, false, false>(const tutti::AttendArgs &, uint32_t, hipStream_t);
