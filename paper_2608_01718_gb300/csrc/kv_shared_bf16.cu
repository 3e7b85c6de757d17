// The attention kernel over a bf16 cache: the two passes over sequences that have their first positions in common.
#include "kv_attend.cuh"

namespace lc {
cudaError_t launch_common_bf16(const AttendArgs& a, int num_sms, cudaStream_t st) {
  return launch_format<LACACHE_KV_BF16, kCommon>(a, num_sms, st);
}
cudaError_t launch_own_bf16(const AttendArgs& a, int num_sms, cudaStream_t st) {
  return launch_format<LACACHE_KV_BF16, kOwn>(a, num_sms, st);
}
}  // namespace lc
