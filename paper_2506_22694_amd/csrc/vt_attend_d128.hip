// Attention over the cache, heads of up to 128 values.
#include "vt_attend_kernel.h"

namespace vt {

hipError_t launch_attend_d128(const AttendArgs &a, int tiles, bool f32, hipStream_t st) {
    if (f32) return run_attend<128, 1, true, false>(a, st);
    if (tiles == 1) return run_attend<128, 1, false, false>(a, st);
    return run_attend<128, 2, false, false>(a, st);
}

}  // namespace vt
