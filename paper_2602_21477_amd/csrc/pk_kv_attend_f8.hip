// Attention over a cache held in e4m3.
#include "pk_kv_attend_dev.h"

namespace pk {
hipError_t launch_kv_attend_f8(const KvAttend &a, int dp, int dtype, hipStream_t s) { return run_storage<PK_F8>(a, dp, dtype, s); }
} // namespace pk
