#include "w4.cuh"

namespace ssd {
ssd_status w4_matmul_fp32_4(int per, const W4Params& p, cudaStream_t s) { return w4_launch_group<float, 1, true>(per, p, s); }
}  // namespace ssd
