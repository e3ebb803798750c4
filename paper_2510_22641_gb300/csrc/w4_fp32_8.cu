#include "w4.cuh"

namespace ssd {
ssd_status w4_matmul_fp32_8(int per, const W4Params& p, cudaStream_t s) { return w4_launch_group<float, 1>(per, p, s); }
}  // namespace ssd
