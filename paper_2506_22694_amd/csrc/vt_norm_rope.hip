// Norm of each head's queries and keys with the position rotation, their gradients, and the same written into a paged cache.
//
// A head row is spread over GL = 8, 16 or 32 lanes (head_dim <= 64, 128, 256), eight values each: the four pairs the lane rotates, or
// eight values past the rotated ones.  So a pair never leaves its lane, and the sum of squares is the only thing that does (three to five
// DPP steps).  A lane keeps its values in fp32 from the load to the one rounding at the store.
//
// Bound by the bytes read and written: 4096 rows of 40 heads of 128 values in bf16 (84 MB) 16.5 us, 16384 rows 68 us, 4.9 TB/s, a copy's rate
// of as much; gradients of 8192 rows (252 MB) 51 us and 4.6 for the weights' sums; 65537 rows of 8 heads read back from 8 bits (404 MB) 76 us.
#include <type_traits>

#include "vt_values.h"

namespace vt {
namespace {

constexpr int kThreads = 256;
constexpr int kNormBackwardWorkgroups = 1024;      // four on each CU

// The eight values of a lane: two runs of four.  Pairs (x[j], x[4 + j]) for halves, (x[2 j], x[2 j + 1]) for neighbours.
struct Lane {
    int o0, o1, pair;
    bool active, turns;
};
__device__ __forceinline__ Lane lane_of(int i, const NormArgs &a) {
    Lane l;
    l.pair = 4 * i;
    l.active = 8 * i < a.D;
    l.turns = a.table != nullptr && l.pair < a.rot / 2;
    const bool halves = l.turns && !a.neighbours;
    l.o0 = halves ? l.pair : 2 * l.pair;
    l.o1 = halves ? l.pair + a.rot / 2 : l.o0 + 4;
    return l;
}

template <typename T>
__device__ __forceinline__ void load8(const void *base, int64_t at, const Lane &l, float *x) {
    const typename T::store *p = static_cast<const typename T::store *>(base) + at;
    T::load4(p + l.o0, x);
    T::load4(p + l.o1, x + 4);
}
template <typename T>
__device__ __forceinline__ void store8(void *base, int64_t at, const Lane &l, const float *x) {
    typename T::store *p = static_cast<typename T::store *>(base) + at;
    T::stream4(p + l.o0, x);
    T::stream4(p + l.o1, x + 4);
}

// The same as it is stored: rows that are asked for ahead of their use
template <typename T>
struct Raw8 {
    typename T::raw4 a, b;
    __device__ __forceinline__ void load(const void *base, int64_t at, const Lane &l) {
        const typename T::store *p = static_cast<const typename T::store *>(base) + at;
        a = *reinterpret_cast<const typename T::raw4 *>(p + l.o0);
        b = *reinterpret_cast<const typename T::raw4 *>(p + l.o1);
    }
    __device__ __forceinline__ void open(float *x) const {
        T::open4(a, x);
        T::open4(b, x + 4);
    }
};

struct Angle {
    float c[4], s[4];
};
__device__ __forceinline__ Angle angle_of(const NormArgs &a, const Lane &l, int64_t row) {
    Angle t;
#pragma unroll
    for (int j = 0; j < 4; ++j) t.c[j] = 1.0f, t.s[j] = 0.0f;
    if (!l.turns) return t;
    const int64_t position = index_at(a.positions, row);
    if (position < 0 || position >= a.table_rows) {
#pragma unroll
        for (int j = 0; j < 4; ++j) t.c[j] = t.s[j] = __builtin_nanf("");
        return t;
    }
    const float *p = a.table + position * a.rot + l.pair;
    F32::load4(p, t.c);
    F32::load4(p + a.rot / 2, t.s);
    return t;
}
// x turned by +angle, or by -angle (SIGN = -1): the transpose, for gradients
template <int SIGN>
__device__ __forceinline__ void turn(float *x, const Angle &t, bool neighbours) {
    float y[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float s = SIGN < 0 ? -t.s[j] : t.s[j];
        const float a = neighbours ? x[2 * j] : x[j], b = neighbours ? x[2 * j + 1] : x[4 + j];
        const float ra = a * t.c[j] - b * s, rb = b * t.c[j] + a * s;
        y[j] = ra, y[4 + j] = rb;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (neighbours) {
            x[2 * j] = y[j], x[2 * j + 1] = y[4 + j];
        } else {
            x[j] = y[j], x[4 + j] = y[4 + j];
        }
    }
}

// One head row into the cache, values x of this lane.
template <int GL>
__device__ __forceinline__ void to_cache(const CacheArgs &c, bool is_v, int64_t cell, const Lane &l, const float *x) {
    if (c.k_scale == nullptr) {
        if (l.active && cell >= 0) store8<Bf16>(is_v ? c.v : c.k, cell * c.D, l, x);
        return;
    }
    float m = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float y = fabsf(x[j]);
        m = fmaxf(m, y < __builtin_inff() ? y : 0.0f);
    }
    m = group_max<GL>(l.active ? m : 0.0f);
    const int e = scale_exponent(__float_as_uint(m));
    if (!l.active || cell < 0) return;
    // (a value next to fp32's largest would be rounded up to 256 * 2^120, which is infinite)
    const float inverse = __uint_as_float((unsigned)(254 - e) << 23), most = e == 247 ? 240.0f : 448.0f;
    uint8_t *p = static_cast<uint8_t *>(is_v ? c.v : c.k) + cell * c.D;
    *reinterpret_cast<unsigned *>(p + l.o0) = pack_e4m3(x, inverse, most);
    *reinterpret_cast<unsigned *>(p + l.o1) = pack_e4m3(x + 4, inverse, most);
    if (l.pair == 0) (is_v ? c.v_scale : c.k_scale)[cell] = (uint8_t)e;
}

// The same in 4 bits.  The lanes exchange their values so that each has eight side by side: `row` is the group's D floats of LDS.
__device__ __forceinline__ void to_cache_of_four(const CacheArgs &c, bool is_v, int64_t cell, const Lane &l, int lane, float *row, float *x) {
    if (l.active) {
        F32::store4(row + l.o0, x);
        F32::store4(row + l.o1, x + 4);
    }
    // (a group is lanes of one wave, whose accesses to LDS are in order)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (l.active) {
        F32::load4(row + 8 * lane, x);
        F32::load4(row + 8 * lane + 4, x + 4);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    unsigned m = 0;      // bits of the largest finite size of the four lanes' values, all ones for NaN among them
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const unsigned u = __float_as_uint(x[j]) & 0x7FFFFFFFu;
        m = max(m, u < 0x7F800000u ? u : u == 0x7F800000u ? 0u : ~0u);
    }
    m = max(m, dpp_mov<0xB1>(m));
    m = max(m, dpp_mov<0x4E>(m));
    if (!l.active || cell < 0) return;
    const int e = m == ~0u ? 255 : scale_exponent_of_four(m);
    *reinterpret_cast<unsigned *>(static_cast<uint8_t *>(is_v ? c.v : c.k) + cell * (c.D / 2) + 4 * lane) = m == ~0u ? 0u : pack_e2m1(x, e);
    if (lane % 4 == 0) (is_v ? c.v_scale : c.k_scale)[scale_of_row(cell, c.D / kScaleGroup, lane / 4, c.page_shift)] = (uint8_t)e;
}

constexpr int kRowsAhead = 4;

// x^(-1/2) in 64 bits, x > 0: the instruction's first digits and a step of Newton's of the third order.  (1 / sqrt(x) of the library, correctly rounded
// twice: 8192 tokens into the cache and read back 59.5 us, 54.9 so.)
__device__ __forceinline__ double inverse_root(double x) {
    const double y = __builtin_amdgcn_rsq(x), e = fma(-x * y, y, 1.0);
    return x < __builtin_inf() ? fma(y * e, fma(0.375, e, 0.5), y) : y;      // (0 of infinity, NaN)
}

// FOUR: into a cache of 4 bits.  Its keys are computed in 64 bits up to the rounding to a code: next to a border between two codes, where fp32's last bits
// decide, the other one is up to half the value away.  (8192 tokens of 32 + 8 + 8 heads of 128 values into the cache and read back, 223 MB: 54.9 us; keys in fp32 48.)
template <typename T, int GL, bool SEVERAL, bool FOUR>
__global__ __launch_bounds__(kThreads) void norm_rope_kernel(NormArgs a) {
    constexpr int GROUPS = kThreads / GL;
    __shared__ __align__(16) float exchange[FOUR ? kThreads * 8 : 1];
    const int group = threadIdx.x / GL;
    const Lane l = lane_of(threadIdx.x % GL, a);
    const int heads = a.hq + a.hk + (a.v != nullptr ? a.hk : 0);
    // groups of a token, tokens of the workgroup (SEVERAL: more than one at a time)
    const int log2 = SEVERAL ? a.tokens_log2 : 0, per = GROUPS >> log2, own = SEVERAL ? group & (per - 1) : group;
    const bool norm = a.wq != nullptr;
    float wq[8], wk[8];
    if (norm && l.active) {
        load8<T>(a.wq, 0, l, wq);
        load8<T>(a.wk, 0, l, wk);
    }
    for (int64_t row = ((int64_t)blockIdx.x << log2) + (SEVERAL ? group / per : 0); row < a.n; row += gridDim.x << log2) {
        for (int base = own; base < heads; base += kRowsAhead * per) {
            // all of a group's rows of the token at a time: a row's 16 bytes a lane leave too little under way (8192 rows into the cache 48 us, 40 so)
            Raw8<T> raw[kRowsAhead] = {};
#pragma unroll
            for (int u = 0; u < kRowsAhead; ++u) {
                const int r = base + u * per;
                if (r >= heads || !l.active) continue;
                const bool is_q = r < a.hq, is_v = r >= a.hq + a.hk;
                const int head = is_q ? r : is_v ? r - a.hq - a.hk : r - a.hq;
                raw[u].load(is_q ? a.q : is_v ? a.v : a.k, row * (is_q ? a.q_stride : is_v ? a.v_stride : a.k_stride) + head * a.D, l);
            }
            const Angle t = angle_of(a, l, row);
            const int64_t slot = a.to_cache ? index_at(a.slots, row) : 0;
#pragma unroll
            for (int u = 0; u < kRowsAhead; ++u) {
                const int r = base + u * per;
                if (r >= heads) break;
                const bool is_q = r < a.hq, is_v = r >= a.hq + a.hk;
                const int head = is_q ? r : is_v ? r - a.hq - a.hk : r - a.hq;
                float x[8];
                raw[u].open(x);
                if constexpr (FOUR) {
                    if (!is_q) {
                        if (!is_v && (norm || a.table != nullptr)) {
                            double rms = 1.0;
                            if (norm) {
                                double ss = 0.0;
#pragma unroll
                                for (int j = 0; j < 8; ++j) ss += (double)x[j] * x[j];
                                rms = inverse_root(group_sum<GL>(ss) * a.inverse_D64 + a.eps);
                            }
                            // a pair after the other: few registers hold 64 bits at a time
                            float y[8];
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const bool nb = a.neighbours || !l.turns;
                                double p = nb ? x[2 * j] : x[j], r = nb ? x[2 * j + 1] : x[4 + j];
                                if (norm) p = p * rms * (nb ? wk[2 * j] : wk[j]), r = r * rms * (nb ? wk[2 * j + 1] : wk[4 + j]);
                                const double c = t.c[j], s = t.s[j];
                                y[j] = round_to_odd(l.turns ? p * c - r * s : p), y[4 + j] = round_to_odd(l.turns ? r * c + p * s : r);
                            }
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const bool nb = a.neighbours || !l.turns;
                                x[j] = nb ? (j % 2 ? y[4 + j / 2] : y[j / 2]) : y[j];
                                x[4 + j] = nb ? (j % 2 ? y[6 + j / 2] : y[2 + j / 2]) : y[4 + j];
                            }
                        }
                        to_cache_of_four(a.cache, is_v, row_of_slot(slot, a.cache.pages, a.cache.heads, head, a.cache.page_shift), l, threadIdx.x % GL,
                                         exchange + group * 8 * GL, x);
                        continue;
                    }
                }
                if (norm && !is_v) {
                    float ss = 0.0f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) ss += x[j] * a.inverse_D * x[j];      // (a mean all along: squares that fit do not overflow as a sum)
                    const float rms = rsqrtf(group_sum<GL>(ss) + a.eps);
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = x[j] * rms * (is_q ? wq[j] : wk[j]);
                }
                if (!is_v && l.turns) turn<1>(x, t, a.neighbours);
                if (is_q) {
                    if (l.active) store8<T>(a.q_out, row * a.q_out_stride + head * a.D, l, x);
                } else if (!a.to_cache) {
                    if (l.active) store8<T>(a.k_out, row * a.k_out_stride + head * a.D, l, x);
                } else {
                    to_cache<GL>(a.cache, is_v, row_of_slot(slot, a.cache.pages, a.cache.heads, head, a.cache.page_shift), l, x);
                }
            }
        }
    }
}

// y = x r, z = y w, out = turned z:  gz = g turned back, dw = sum gz y, gy = gz w, dx = r (gy - y mean(gy y)).
// r is found again from x, which the sums need anyway.  A workgroup takes rows blockIdx.x, + gridDim.x, ... and keeps its sums for the
// weights in registers, eight values a lane; the lanes of the same columns are added in LDS at its end, and the workgroups' sums in a
// kernel of their own, both in a fixed order.
constexpr int kBackwardAhead = kRowsAhead;

template <typename T, int GL, bool SEVERAL>
__global__ __launch_bounds__(kThreads) void norm_rope_backward_kernel(NormArgs a) {
    constexpr int GROUPS = kThreads / GL;
    __shared__ float sums[kThreads * 8];
    const int group = threadIdx.x / GL;
    const Lane l = lane_of(threadIdx.x % GL, a);
    const int heads = a.hq + a.hk;
    const int log2 = SEVERAL ? a.tokens_log2 : 0, per = GROUPS >> log2, own = SEVERAL ? group & (per - 1) : group;
    const bool norm = a.wq != nullptr;
    float wq[8], wk[8], sq[8] = {}, sk[8] = {};
    if (norm && l.active) {
        load8<T>(a.wq, 0, l, wq);
        load8<T>(a.wk, 0, l, wk);
    }
    for (int64_t row = ((int64_t)blockIdx.x << log2) + (SEVERAL ? group / per : 0); row < a.n; row += gridDim.x << log2) {
        for (int base = own; base < heads; base += kBackwardAhead * per) {
            Raw8<T> rg[kBackwardAhead] = {}, rx[kBackwardAhead] = {};
#pragma unroll
            for (int u = 0; u < kBackwardAhead; ++u) {
                const int r = base + u * per;
                if (r >= heads || !l.active) continue;
                const bool is_q = r < a.hq;
                const int head = is_q ? r : r - a.hq;
                rg[u].load(is_q ? a.gq : a.gk, row * (is_q ? a.gq_stride : a.gk_stride) + head * a.D, l);
                if (norm) rx[u].load(is_q ? a.q : a.k, row * (is_q ? a.q_stride : a.k_stride) + head * a.D, l);
            }
            const Angle t = angle_of(a, l, row);
#pragma unroll
            for (int u = 0; u < kBackwardAhead; ++u) {
                const int r = base + u * per;
                if (r >= heads) break;
                const bool is_q = r < a.hq;
                const int head = is_q ? r : r - a.hq;
                float g[8], x[8];
                rg[u].open(g);
                rx[u].open(x);
                if (l.turns) turn<-1>(g, t, a.neighbours);
                if (norm) {
                    float ss = 0.0f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) ss += x[j] * a.inverse_D * x[j];
                    const float rms = rsqrtf(group_sum<GL>(ss) + a.eps);
                    float dot = 0.0f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        x[j] *= rms;
                        const float p = g[j] * x[j];
                        sq[j] += is_q ? p : 0.0f;
                        sk[j] += is_q ? 0.0f : p;
                        g[j] *= is_q ? wq[j] : wk[j];
                        dot += l.active ? g[j] * x[j] : 0.0f;
                    }
                    dot = group_sum<GL>(dot) * a.inverse_D;
#pragma unroll
                    for (int j = 0; j < 8; ++j) g[j] = rms * (g[j] - x[j] * dot);
                }
                if (l.active) store8<T>(is_q ? a.q_out : a.k_out, row * (is_q ? a.q_out_stride : a.k_out_stride) + head * a.D, l, g);
            }
        }
    }
    if (!norm) return;
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
        if (l.active) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                sums[group * a.D + l.o0 + j] = which ? sk[j] : sq[j];
                sums[group * a.D + l.o1 + j] = which ? sk[4 + j] : sq[4 + j];
            }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < a.D; c += kThreads) {
            float s = 0.0f;
            for (int i = 0; i < kThreads / GL; ++i) s += sums[i * a.D + c];
            a.partial[((int64_t)blockIdx.x * 2 + which) * a.D + c] = s;
        }
    }
}

// Columns of [workgroups, 2 * D] added up: 8 columns and 128 shares of the workgroups to a workgroup, a share's rows all under way at a time
// (1024 rows in 16 shares, a row after the other: 20.6 us).
constexpr int kSumThreads = 1024, kSumColumns = 8;
__global__ __launch_bounds__(kSumThreads) void norm_weight_sums_kernel(NormArgs a, int workgroups) {
    constexpr int SHARES = kSumThreads / kSumColumns;
    __shared__ float sums[SHARES][kSumColumns + 1];
    const int column = threadIdx.x % kSumColumns, c = blockIdx.x * kSumColumns + column, share = threadIdx.x / kSumColumns;
    float s = 0.0f;      // (2 * D is a multiple of 16: every column exists)
    constexpr int PER = kNormBackwardWorkgroups / SHARES;
    float x[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int w = share + i * SHARES;
        x[i] = a.partial[(int64_t)min(w, workgroups - 1) * 2 * a.D + c];
        x[i] = w < workgroups ? x[i] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) s += x[i];
    sums[share][column] = s;
    __syncthreads();
    for (int half = SHARES / 2; half > 0; half /= 2) {
        if (share < half) sums[share][column] += sums[share + half][column];
        __syncthreads();
    }
    if (share == 0) (c < a.D ? a.dqw : a.dkw - a.D)[c] = sums[0][column];
}

// Rows of the cache as values: GL lanes to a head row, eight values a lane.
template <typename T, int GL>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(CacheReadArgs a) {
    const int group = threadIdx.x / GL, o = 8 * (threadIdx.x % GL);
    if (o >= a.cache.D) return;
    const int64_t all = a.n * a.cache.heads;
    for (int64_t r = (int64_t)blockIdx.x * (kThreads / GL) + group; r < all; r += (int64_t)gridDim.x * (kThreads / GL)) {      // (row, head)
        const int64_t row = r / a.cache.heads;
        const int head = (int)(r % a.cache.heads);
        const int64_t cell = row_of_slot(index_at(a.slots, row), a.cache.pages, a.cache.heads, head, a.cache.page_shift);
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const void *held = which ? a.cache.v : a.cache.k;
            float x[8] = {};
            if (cell >= 0) {
                if (a.cache.four) {
                    const unsigned u = *reinterpret_cast<const unsigned *>(static_cast<const uint8_t *>(held) + cell * (a.cache.D / 2) + o / 2);
                    const int64_t at = scale_of_row(cell, a.cache.D / kScaleGroup, o / kScaleGroup, a.cache.page_shift);
                    open_e2m1(u, (which ? a.cache.v_scale : a.cache.k_scale)[at], x);
                } else if (a.cache.k_scale == nullptr) {
                    const uint16_t *p = static_cast<const uint16_t *>(held) + cell * a.cache.D + o;
                    Bf16::load4(p, x);
                    Bf16::load4(p + 4, x + 4);
                } else {
                    const u32x2 u = *reinterpret_cast<const u32x2 *>(static_cast<const uint8_t *>(held) + cell * a.cache.D + o);
                    const unsigned e = (which ? a.cache.v_scale : a.cache.k_scale)[cell];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int w = (int)(j ? u.y : u.x);
                        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
                        x[4 * j] = scaled(lo[0], e), x[4 * j + 1] = scaled(lo[1], e), x[4 * j + 2] = scaled(hi[0], e), x[4 * j + 3] = scaled(hi[1], e);
                    }
                }
            }
            typename T::store *p = static_cast<typename T::store *>(which ? a.v_out : a.k_out) + r * a.cache.D + o;
            T::stream4(p, x);
            T::stream4(p + 4, x + 4);
        }
    }
}

// (a launch's threads are a 32-bit number)
unsigned workgroups(int64_t wanted) { return (unsigned)(wanted < (1 << 23) ? wanted : 1 << 23); }

int lanes_of(int D) { return D <= 64 ? 8 : D <= 128 ? 16 : 32; }
// Tokens that a workgroup takes at a time: as many as have all their rows under way at a time still, and leave the CUs four workgroups each:
// 8192 tokens of 10 heads of 128 values 11.9 us, 17.2 a token at a time; of 40 heads of 64 18.5 and 21.3.
int tokens_log2(int64_t n, int heads, int groups) {
    int t = 0;
    while (t < 3 && (groups >> (t + 1)) * kRowsAhead >= heads && (n >> (t + 1)) >= 1024) ++t;
    return t;
}

template <typename T>
void run_forward(NormArgs a, hipStream_t st) {
    const int GL = lanes_of(a.D);
    a.tokens_log2 = tokens_log2(a.n, a.hq + a.hk + (a.v != nullptr ? a.hk : 0), kThreads / GL);
    const dim3 grid(workgroups((a.n + ((int64_t)1 << a.tokens_log2) - 1) >> a.tokens_log2));
    auto launch = [&](auto one, auto several) { (a.tokens_log2 > 0 ? several : one)<<<grid, kThreads, 0, st>>>(a); };
    auto held = [&](auto four) {
        constexpr bool FOUR = decltype(four)::value;
        if (GL == 8) launch(norm_rope_kernel<T, 8, false, FOUR>, norm_rope_kernel<T, 8, true, FOUR>);
        else if (GL == 16) launch(norm_rope_kernel<T, 16, false, FOUR>, norm_rope_kernel<T, 16, true, FOUR>);
        else launch(norm_rope_kernel<T, 32, false, FOUR>, norm_rope_kernel<T, 32, true, FOUR>);
    };
    if (a.to_cache && a.cache.four) held(std::true_type());
    else held(std::false_type());
}
template <typename T>
void run_backward(NormArgs a, hipStream_t st) {
    const int GL = lanes_of(a.D);
    a.tokens_log2 = tokens_log2(a.n, a.hq + a.hk, kThreads / GL);
    const dim3 grid((unsigned)norm_backward_workgroups(a.n));
    auto launch = [&](auto one, auto several) { (a.tokens_log2 > 0 ? several : one)<<<grid, kThreads, 0, st>>>(a); };
    if (GL == 8) launch(norm_rope_backward_kernel<T, 8, false>, norm_rope_backward_kernel<T, 8, true>);
    else if (GL == 16) launch(norm_rope_backward_kernel<T, 16, false>, norm_rope_backward_kernel<T, 16, true>);
    else launch(norm_rope_backward_kernel<T, 32, false>, norm_rope_backward_kernel<T, 32, true>);
}
template <typename T>
void run_read(const CacheReadArgs &a, hipStream_t st) {
    const int GL = lanes_of(a.cache.D), per = kThreads / GL;
    const dim3 grid(workgroups((a.n * a.cache.heads + per - 1) / per));
    if (GL == 8) cache_read_kernel<T, 8><<<grid, kThreads, 0, st>>>(a);
    else if (GL == 16) cache_read_kernel<T, 16><<<grid, kThreads, 0, st>>>(a);
    else cache_read_kernel<T, 32><<<grid, kThreads, 0, st>>>(a);
}

}  // namespace

int norm_backward_workgroups(int64_t n) { return n < kNormBackwardWorkgroups ? (n < 1 ? 1 : (int)n) : kNormBackwardWorkgroups; }

hipError_t launch_norm_rope(const NormArgs &args, bool bf16, hipStream_t st) {
    NormArgs a = args;
    a.inverse_D = 1.0f / (float)a.D;
    a.inverse_D64 = 1.0 / a.D;
    bf16 ? run_forward<Bf16>(a, st) : run_forward<F32>(a, st);
    return hipGetLastError();
}
hipError_t launch_norm_rope_backward(const NormArgs &args, bool bf16, hipStream_t st) {
    NormArgs a = args;
    a.inverse_D = 1.0f / (float)a.D;
    bf16 ? run_backward<Bf16>(a, st) : run_backward<F32>(a, st);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.wq == nullptr) return e;
    norm_weight_sums_kernel<<<2 * a.D / kSumColumns, kSumThreads, 0, st>>>(a, norm_backward_workgroups(a.n));
    return hipGetLastError();
}
hipError_t launch_cache_read(const CacheReadArgs &a, bool bf16, hipStream_t st) {
    bf16 ? run_read<Bf16>(a, st) : run_read<F32>(a, st);
    return hipGetLastError();
}

}  // namespace vt
