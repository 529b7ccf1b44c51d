// Attention over a key/value cache: the call's storage, and half precision's kernels.
#include "pk_kv_attend_dev.h"

namespace pk {

hipError_t launch_kv_attend_bf16(const KvAttend &a, int dp, int dtype, hipStream_t s);
hipError_t launch_kv_attend_i8(const KvAttend &a, int dp, int dtype, hipStream_t s);
hipError_t launch_kv_attend_f8(const KvAttend &a, int dp, int dtype, hipStream_t s);
hipError_t launch_kv_attend_f4(const KvAttend &a, int dp, int dtype, hipStream_t s);

hipError_t launch_kv_attend(const KvAttend &a, int storage, int dp, int dtype, hipStream_t s)
{
    switch (storage) {
    case PK_I8: return launch_kv_attend_i8(a, dp, dtype, s);
    case PK_F8: return launch_kv_attend_f8(a, dp, dtype, s);
    case PK_F4: return launch_kv_attend_f4(a, dp, dtype, s);
    case PK_F16: return run_storage<PK_F16>(a, dp, dtype, s);
    default: return launch_kv_attend_bf16(a, dp, dtype, s);
    }
}

} // namespace pk
