// Attention of prompts' chunks over the cache with a window and sinks: which kernel a shape gets.
#include "vt_prompt_kernel.h"

namespace vt {

hipError_t launch_prompt(const AttendArgs &a, hipStream_t st) {
    const int D = a.cache.D, tiles = a.row_tiles;
    if (D <= 64) return tiles == 1 ? run_prompt<64, 1>(a, st) : run_prompt<64, 2>(a, st);
    if (D <= 128) return tiles == 1 ? run_prompt<128, 1>(a, st) : run_prompt<128, 2>(a, st);
    return run_prompt<256, 1>(a, st);
}

}  // namespace vt
