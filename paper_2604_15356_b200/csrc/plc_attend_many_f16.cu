// Tree attention of many rows, f16 pools.
#include "plc_attend_many.cuh"

namespace plc {
cudaError_t launch_attend_many_f16(const PoolDev& p, const BookDev& b, const AttendArgs& a, const AttendPlan& x, uint32_t* status, cudaStream_t st) {
    return launch_many<__half>(p, b, a, x, false, status, st);
}
}  // namespace plc
