// Attention over pages of format STEPQ_KV_F16.
#include "kv_launch.cuh"

namespace stepq {
namespace kv {

template stepq_status launch_attend<STEPQ_KV_F16>(const stepq_kv_config *, const AttendArgs &, int64_t, cudaStream_t);
template size_t attend_workspace<STEPQ_KV_F16>(const stepq_kv_config *, int, int64_t, int64_t);

}  // namespace kv
}  // namespace stepq
