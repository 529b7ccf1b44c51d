// Attention over a cache held in bfloat16.
#include "pk_kv_attend_dev.h"

namespace pk {
hipError_t launch_kv_attend_bf16(const KvAttend &a, int dp, int dtype, hipStream_t s) { return run_storage<PK_BF16>(a, dp, dtype, s); }
} // namespace pk
