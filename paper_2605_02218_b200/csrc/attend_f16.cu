// The attention kernels for float16 queries.
#include "attend_launch.cuh"

cudaError_t covspec::attend::launch_f16(const Call& call) { return launch<__half>(call); }
