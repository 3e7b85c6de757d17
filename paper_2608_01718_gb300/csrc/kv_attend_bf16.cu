// The attention kernel over a bf16 cache.
#include "kv_attend.cuh"

namespace lc {
cudaError_t launch_attend_bf16(const AttendArgs& a, int num_sms, cudaStream_t st) {
  return launch_format<LACACHE_KV_BF16>(a, num_sms, st);
}
}  // namespace lc
