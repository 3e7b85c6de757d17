// The attention kernel over an f16 cache: the two passes over sequences that have their first positions in common.
#include "kv_attend.cuh"

namespace lc {
cudaError_t launch_common_f16(const AttendArgs& a, int num_sms, cudaStream_t st) {
  return launch_format<LACACHE_KV_F16, kCommon>(a, num_sms, st);
}
cudaError_t launch_own_f16(const AttendArgs& a, int num_sms, cudaStream_t st) {
  return launch_format<LACACHE_KV_F16, kOwn>(a, num_sms, st);
}
}  // namespace lc
