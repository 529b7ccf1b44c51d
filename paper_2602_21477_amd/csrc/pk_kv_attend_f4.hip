// Attention over a cache held in 4 bits.
#include "pk_kv_attend_dev.h"

namespace pk {
hipError_t launch_kv_attend_f4(const KvAttend &a, int dp, int dtype, hipStream_t s) { return run_storage<PK_F4>(a, dp, dtype, s); }
} // namespace pk
