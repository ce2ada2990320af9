// Tree attention of many rows, bf16 pools.
#include "plc_attend_many.cuh"

namespace plc {
cudaError_t launch_attend_many_bf16(const PoolDev& p, const BookDev& b, const AttendArgs& a, const AttendPlan& x, uint32_t* status, cudaStream_t st) {
    return launch_many<__nv_bfloat16>(p, b, a, x, true, status, st);
}
}  // namespace plc
