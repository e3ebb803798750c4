#include "w4.cuh"

namespace ssd {
ssd_status w4_matmul_bf16_16(int per, const W4Params& p, cudaStream_t s) { return w4_launch_group<__nv_bfloat16, 2>(per, p, s); }
}  // namespace ssd
