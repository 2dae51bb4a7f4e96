// Attention over the cache: which kernel a shape gets, and the join of what several workgroups have of a request.
#include "vt_attend_kernel.h"

namespace vt {
namespace {

constexpr int kJoinThreads = 256;
// Rows and heads from which on each has a wave instead of a workgroup
constexpr int64_t kJoinWide = 1024;

// The parts of a row and head of a request that several workgroups had: their sums, each brought to the maximum of all; a part's sum of 0
// has nothing of the row.  LV lanes read a part's row.  TEAM threads take a row and head: a workgroup, which has 256 / LV parts under way at
// a time (a wave for all of them: 18.6 us for 32 heads of 128 parts), or a wave, where rows and heads are many and parts therefore few
// (64 requests of up to 8 rows and 32 heads, both launches: 98 us with a workgroup for each, 84 with a wave; 4 requests of as many, with up
// to 33 parts: 18.3 and 19.5).
template <int LV, int TEAM, bool F32Q>
__global__ __launch_bounds__(kJoinThreads) void attend_join_kernel(AttendArgs a) {
    constexpr int GROUPS = TEAM / LV;
    __shared__ __align__(16) float sums[GROUPS][4 * LV];
    __shared__ float totals[GROUPS];
    const int member = threadIdx.x % TEAM, head = blockIdx.y * (kJoinThreads / TEAM) + (TEAM == 64 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64) : 0);
    if (TEAM == 64 && head >= a.hq) return;
    int b = blockIdx.x, r = 0;
    if (a.max_rows > 1) {
        r = b % a.max_rows;
        b /= a.max_rows;
    }
    // (every place has said what it begins; a request only if it has rows: nothing of one without is looked at)
    const int4 parts = a.part_at[b];
    if (a.by_place) b = parts.w;
    int first;
    if (r >= rows_of(a.row_start, b, a.n, a.max_rows, first) || parts.y == 1) return;
    const int h = head / a.G, rows = 16 * a.row_tiles, x = r * a.G + head - h * a.G, rb = x / rows;
    const int64_t at = ((int64_t)(rb * a.cache.heads + h) * a.places + parts.x) * 2 * rows + (x - rb * rows);
    // part i: of place parts.x + i, there the first one but for a request that begins within a share
    auto index = [&](int i) { return at + (int64_t)(2 * i + (i == 0 ? parts.z : 0)) * rows; };
    const int lane = lane_id(), group = member / LV, d = 4 * (member % LV);
    const int from = d < a.cache.D ? d : 0;
    constexpr int AHEAD = TEAM == 64 ? 2 : 4;      // parts of a group that are asked for along with the maxima
    float2 ms[AHEAD];
    float v[AHEAD][4];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
        const int64_t k = index(min(group + i * GROUPS, parts.y - 1));
        ms[i] = a.part_ms[k];
        F32::load4(a.part_o + k * a.cache.D + from, v[i]);
    }
    float top = kNone;
    for (int s = lane; s < parts.y; s += 64) top = fmaxf(top, a.part_ms[index(s)].x);
    top = wave_max(top);
    float total = 0.0f, o[4] = {};
    auto add = [&](int s, float2 part, const float *u) {
        const bool nothing = s >= parts.y || part.y == 0.0f;
        const float f = __builtin_amdgcn_exp2f(part.x - top);
        total += nothing ? 0.0f : part.y * f;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] += nothing ? 0.0f : u[j] * f;
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) add(group + i * GROUPS, ms[i], v[i]);
#pragma unroll 4
    for (int s = group + AHEAD * GROUPS; s < parts.y; s += GROUPS) {
        float u[4];
        F32::load4(a.part_o + index(s) * a.cache.D + from, u);
        add(s, a.part_ms[index(s)], u);
    }
    if constexpr (TEAM == 64) {
        if constexpr (LV < 64) {
            auto over_groups = [](float v) { return LV == 16 ? row_sum(v) : half_sum(v); };
            total = over_groups(total);
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = over_groups(o[j]);
        }
        if (group != 0 || d >= a.cache.D) return;
    } else {
        F32::store4(&sums[group][d], o);
        if (d == 0) totals[group] = total;
        __syncthreads();
        if (group != 0 || d >= a.cache.D) return;
#pragma unroll
        for (int s = 1; s < GROUPS; ++s) {
            total += totals[s];
            float v[4];
            F32::load4(&sums[s][d], v);
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] += v[j];
        }
    }
    const float inverse = total == 0.0f ? 0.0f : 1.0f / total;
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] *= inverse;
    store_values(a, (int64_t)(first + r) * a.out_stride + head * a.cache.D + d, o, F32Q);
    if (d == 0 && a.lse != nullptr) a.lse[(int64_t)(first + r) * a.hq + head] = log_sum_exp(top, total);
}

template <int LV, int TEAM>
void run_join(const AttendArgs &a, bool f32, int64_t rows, hipStream_t st) {
    constexpr int HEADS = kJoinThreads / TEAM;
    const dim3 grid((unsigned)rows, (unsigned)((a.hq + HEADS - 1) / HEADS));
    if (f32) attend_join_kernel<LV, TEAM, true><<<grid, kJoinThreads, 0, st>>>(a);
    else attend_join_kernel<LV, TEAM, false><<<grid, kJoinThreads, 0, st>>>(a);
}
template <int LV>
void run_join(const AttendArgs &a, bool f32, hipStream_t st) {
    const int64_t rows = (int64_t)(a.by_place ? a.places : a.requests) * a.max_rows;
    if (rows * a.hq <= kJoinWide) run_join<LV, kJoinThreads>(a, f32, rows, st);
    else run_join<LV, 64>(a, f32, rows, st);
}

}  // namespace

int attend_row_tiles(int rows, int D, bool f32) {
    if (f32 || rows <= 16 || D > 128) return 1;
    return rows <= 32 || D > 64 ? 2 : 4;
}

hipError_t launch_attend(const AttendArgs &a, bool f32, hipStream_t st) {
    const int D = a.cache.D, tiles = a.row_tiles;
    hipError_t e = D <= 64 ? launch_attend_d64(a, tiles, f32, st) : D <= 128 ? launch_attend_d128(a, tiles, f32, st) : launch_attend_d256(a, tiles, f32, st);
    if (e != hipSuccess || a.whole) return e;
    if (D <= 64) run_join<16>(a, f32, st);
    else if (D <= 128) run_join<32>(a, f32, st);
    else run_join<64>(a, f32, st);
    return hipGetLastError();
}

}  // namespace vt
