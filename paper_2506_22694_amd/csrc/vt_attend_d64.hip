// Attention over the cache, heads of up to 64 values.
#include "vt_attend_kernel.h"

namespace vt {

hipError_t launch_attend_d64(const AttendArgs &a, int tiles, bool f32, hipStream_t st) {
    if (f32) return run_attend<64, 1, true, false>(a, st);
    if (tiles == 1) return run_attend<64, 1, false, false>(a, st);
    if (tiles == 2) return run_attend<64, 2, false, false>(a, st);
    return run_attend<64, 4, false, false>(a, st);
}

}  // namespace vt
