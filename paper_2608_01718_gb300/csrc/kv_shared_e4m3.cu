// The attention kernel over an e4m3 cache: the two passes over sequences that have their first positions in common.
#include "kv_attend.cuh"

namespace lc {
cudaError_t launch_common_e4m3(const AttendArgs& a, int num_sms, cudaStream_t st) {
  return launch_format<LACACHE_KV_E4M3, kCommon>(a, num_sms, st);
}
cudaError_t launch_own_e4m3(const AttendArgs& a, int num_sms, cudaStream_t st) {
  return launch_format<LACACHE_KV_E4M3, kOwn>(a, num_sms, st);
}
}  // namespace lc
