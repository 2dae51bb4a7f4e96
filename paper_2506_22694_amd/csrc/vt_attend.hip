// Attention over the cache: which kernel a shape gets, and the join of the pieces of long requests.
#include "vt_attend_kernel.h"

namespace vt {
namespace {

constexpr int kJoinWaves = 4;

// One wave to a row and head: the pieces' sums, each brought to the maximum of all.  A piece's sum of 0 has nothing of the row.
template <bool F32Q>
__global__ __launch_bounds__(64 * kJoinWaves) void attend_join_kernel(AttendArgs a) {
    const int lane = lane_id();
    const int64_t i = (int64_t)blockIdx.x * kJoinWaves + (threadIdx.x >> 6);      // (request, row of it, head)
    const int head = (int)(i % a.hq), r = (int)(i / a.hq % a.max_rows);
    const int64_t b = i / a.hq / a.max_rows;
    if (b >= a.requests) return;
    int64_t first;
    if (r >= rows_of(a.row_start, (int)b, a.n, a.max_rows, first)) return;
    const int len = tokens_of(a.lengths[b], a.most);
    const int pieces = pieces_of(len, piece_tokens(len, a.splits, kAttendLeast));
    if (pieces == 1) return;
    const int64_t at = ((first + r) * a.hq + head) * a.splits;
    float top = kNone;
    for (int s = lane; s < pieces; s += 64) top = fmaxf(top, a.part_ms[at + s].x);
    top = wave_max(top);
    const int d = 4 * lane;
    float total = 0.0f, o[4] = {};
    for (int s0 = 0; s0 < pieces; s0 += 64) {
        const float2 ms = a.part_ms[at + min(s0 + lane, pieces - 1)];
        const float f = ms.y == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(ms.x - top);
        const float part = ms.y == 0.0f ? 0.0f : ms.y * f;
        const int here = min(64, pieces - s0);
#pragma unroll 4
        for (int s = 0; s < here; ++s) {
            const float fs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), s));
            total += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(part), s));
            float x[4] = {};
            if (d < a.cache.D) F32::load4(a.part_o + (at + s0 + s) * a.cache.D + d, x);
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] += x[j] * fs;
        }
    }
    if (d < a.cache.D) finish_row(a, first + r, head, d, o, top, total, F32Q);
}

}  // namespace

int attend_row_tiles(int rows, int D, bool f32) {
    if (f32 || rows <= 16) return 1;
    if (rows <= 32 || D > 64) return D > 128 ? 1 : 2;
    return 4;
}

hipError_t launch_attend(const AttendArgs &a, bool f32, hipStream_t st) {
    const int D = a.cache.D, tiles = attend_row_tiles(a.max_rows * a.G, D, f32);
    hipError_t e = D <= 64 ? launch_attend_d64(a, tiles, f32, st) : D <= 128 ? launch_attend_d128(a, tiles, f32, st) : launch_attend_d256(a, tiles, f32, st);
    if (e != hipSuccess || a.splits == 1) return e;
    const int64_t waves = (int64_t)a.requests * a.max_rows * a.hq;
    const unsigned grid = (unsigned)((waves + kJoinWaves - 1) / kJoinWaves);
    if (f32) attend_join_kernel<true><<<grid, 64 * kJoinWaves, 0, st>>>(a);
    else attend_join_kernel<false><<<grid, 64 * kJoinWaves, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace vt
