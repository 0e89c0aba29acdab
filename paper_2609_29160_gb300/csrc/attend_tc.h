// Launcher of the tensor-memory attention kernel (attend_tc.cu).
#pragma once

#include "attend.cuh"

namespace tre {
constexpr int kTcRows = 256;      // rows that one of its CTAs takes
constexpr int kTcTokens = 128;    // positions that it takes at a time
cudaError_t launch_attend_tc(int dtype, int code, int dim, const AttendArgs& a,
                             const BatchArgs& b, const CacheArgs& c, int64_t units,
                             tre_diag* diag, cudaStream_t s);
}  // namespace tre
