#define SLICER_KV_INSTANTIATE
#include "slicer_launch_kv.hpp"
template hipError_t slicer::launch_kv_append<1>(const KvAppendArgs&, int64_t, hipStream_t);
template hipError_t slicer::launch_kv_read<1>(const KvReadArgs&, int64_t, hipStream_t);
template hipError_t slicer::launch_kv_attend<1>(const KvAttendArgs&, const KvAttendLaunch&, hipStream_t);
