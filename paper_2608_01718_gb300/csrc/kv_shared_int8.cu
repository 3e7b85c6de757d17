// The attention kernel over an int8 cache: the two passes over sequences that have their first positions in common.
#include "kv_attend.cuh"

namespace lc {
cudaError_t launch_common_int8(const AttendArgs& a, int num_sms, cudaStream_t st) {
  return launch_format<LACACHE_KV_INT8, kCommon>(a, num_sms, st);
}
cudaError_t launch_own_int8(const AttendArgs& a, int num_sms, cudaStream_t st) {
  return launch_format<LACACHE_KV_INT8, kOwn>(a, num_sms, st);
}
}  // namespace lc
