// Attention over the cache, heads of up to 256 values.
#include "vt_attend_kernel.h"

namespace vt {

hipError_t launch_attend_d256(const AttendArgs &a, int, bool f32, hipStream_t st) {
    return f32 ? run_attend<256, 1, true>(a, st) : run_attend<256, 1, false>(a, st);
}

}  // namespace vt
