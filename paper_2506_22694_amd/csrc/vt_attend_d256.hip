// Attention over the cache, heads of up to 256 values.
#include "vt_attend_kernel.h"

namespace vt {

hipError_t launch_attend_d256(const AttendArgs &a, int tiles, bool f32, hipStream_t st) {
    if (f32) return run_attend<256, 1, true>(a, st);
    if (tiles == 1) return run_attend<256, 1, false>(a, st);
    return run_attend<256, 2, false>(a, st);
}

}  // namespace vt
