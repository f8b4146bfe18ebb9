// The attention kernels for bfloat16 queries.
#include "attend_launch.cuh"

cudaError_t covspec::attend::launch_bf16(const Call& call) { return launch<__nv_bfloat16>(call); }
