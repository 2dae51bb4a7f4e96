// Attention of a draft step's rows over a paged key-value cache, on the matrix cores (v_mfma_f32_16x16x32_bf16).
//
// Bound by the one pass over the cached keys and values: a kv head's query rows (the heads that share it, times the request's new
// tokens) are one side of the products, and up to 64 of them cost the matrix cores a fraction of the time that the cache takes to
// arrive.  So what matters is that loads never stop, and a wave goes its own way: it takes 32 tokens at a time, straight from the cache
// into registers in the matrix instructions' operand layout, without LDS and without a barrier until its part of the request is done.
//
//   scores^T [token, row] = K q^T      K's operand: lane l holds values of token l % 16, which are 16 bytes side by side in memory
//   out^T [d, row] = V^T p^T           p's operand: lane l holds row l % 16 and 8 tokens -- those whose scores it has: what the
//                                      first product leaves in a lane is the second one's operand as it is
//
// The order of the tokens in the second product's sum is free, and so is that of the values of d over the lanes: lane l reads values
// E (l % 16) .. + E - 1 of each of its 8 tokens (E = head_dim / 16), whole lines of a row at a time, and is row l % 16 of E products,
// the i-th being over the values E m + i.  Only pairs of tokens within a register have to change places (one v_perm for each register).
// Softmax statistics are kept per row in a lane, which is also the row of all of the lane's sums: rescaling needs no exchange.
//
// 8-bit caches: codes become bf16 (exactly) on their way, two for each conversion; scales are powers of two and go on the scores
// and on p, where they are exact as well.  4-bit ones have a scale for 32 values, which goes into the conversion: a lane's keys of a token are then
// DP / 4 values side by side, and its values E of one token, of one group each.
//
// WINDOW: a row sees sinks and a window.  Tokens are counted without those between (Request::gap), everything goes by that number but a tile's page and what a
// row sees of it.
//
// Values of 24 bits -- the weights p, and q of fp32 rows -- are sums of three of 8, so they are three operands each, and products are exact as
// for bf16.  An infinity on the other side is still one after three products only if all three terms have the value's sign and none is
// zero: the first two are cut off from just below what they are taken of.  (p as one operand, rounded to bf16: results in bf16 off by 0.0018
// to 0.0021 of their size instead of 0.0016 to 0.0017, their own rounding; 131001 tokens as long, 64 tree levels of 8 nodes 83 instead of 84 us, over
// 8 bits 61 instead of 65, 16 nodes of 64 heads of 64 values 71 instead of 81.)
//
// 131001 tokens of one request, 8 kv heads of 128 values in bf16, 4 query heads each: 537 MB in 80 us, 6.7 TB/s, where a plain read of as much
// takes 79; 224 vector and 32 matrix instructions a tile (8 bits: 317 and 32; 48 ragged requests 541 MB in 95 us, 5.7 TB/s).  4 bits: 143 MB in 34 us,
// 48 ragged requests 292 MB in 60, 4.8 TB/s: 262 and 24 instructions a tile, which hardly overlap on a SIMD, are most of it.
#pragma once
#include "vt_values.h"

namespace vt {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4a;

__device__ __forceinline__ f32x4a mfma(u32x4 a, u32x4 b, f32x4a c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// What a cache holds: bf16, or codes of 8 or 4 bits
constexpr int kHeld16 = 0, kHeld8 = 1, kHeld4 = 2;

// bf16 pairs of two codes of 8 bits: the lower or upper two of a register
template <bool HIGH>
__device__ __forceinline__ unsigned two_codes(unsigned u) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, 1.0f, HIGH));
}
// ... of the eight codes of 4 bits of a register, times a power of two: the scale's bits 30 to 23 are its exponent + 127, all other bits count for nothing
__device__ __forceinline__ void eight_codes(unsigned u, unsigned scale, unsigned (&f)[4]) {
    const float s = __uint_as_float(scale);
    f[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, s, 0));
    f[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, s, 1));
    f[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, s, 2));
    f[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, s, 3));
}
__device__ __forceinline__ void four_codes(unsigned u, unsigned scale, unsigned (&f)[2]) {
    const float s = __uint_as_float(scale);
    f[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, s, 0));
    f[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, s, 1));
}
// Maximum and sum over the four lanes l, l ^ 16, l ^ 32, l ^ 48, which hold the same row
__device__ __forceinline__ float row_max(float v) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float row_sum(float v) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// Sum over lanes l and l ^ 32
__device__ __forceinline__ float half_sum(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// Eight fp32 values (none -0) as the sum of three operands: the leading 8 bits of what is just below the value, those of what is just below the
// rest, and the rest, which has 8.  (Below it by the last of its 24 bits; below an infinity are the largest finite ones.  0 is three zeros.)
// Two terms: the rest, of up to 2^-7 of the value, is rounded to 8 bits (2^-16 of the value at most), and is not zero either.
template <int TERMS, typename Terms>
__device__ __forceinline__ void split_terms(float (&v)[8], Terms &terms) {
#pragma unroll
    for (int i = 0; i < TERMS; ++i) {
        if (TERMS == 2 && i == 1) {
#pragma unroll
            for (int j = 0; j < 4; ++j) terms[1][j] = pack_bf16(v[2 * j], v[2 * j + 1]);
            break;
        }
        unsigned u[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            u[j] = __float_as_uint(v[j]);
            if (i == 2) continue;
            u[j] = __builtin_elementwise_sub_sat(u[j], 1u);
            v[j] -= __uint_as_float(u[j] & 0xFFFF0000u);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) terms[i][j] = __builtin_amdgcn_perm(u[2 * j + 1], u[2 * j], 0x07060302);
    }
}

constexpr float kNone = -__builtin_inff();

__device__ __forceinline__ float log_sum_exp(float top, float total) {
    return total == 0.0f ? kNone : (top + __builtin_amdgcn_logf(total)) * 0.69314718055994531f;
}
__device__ __forceinline__ void store_values(const AttendArgs &a, int64_t at, const float *o, bool f32) {
    if (f32) F32::store4(static_cast<float *>(a.out) + at, o);
    else Bf16::store4(static_cast<uint16_t *>(a.out) + at, o);
}
// y / G for y < 2048, G <= 1024
__device__ __forceinline__ int by_group(const AttendArgs &a, int y) { return a.G == 1 ? y : (int)__umulhi((unsigned)y, a.G_magic); }

// Row i of a request's rows, `row` of all
__device__ __forceinline__ int position_of(const AttendArgs &a, int64_t row, int tokens, int rows, int i) {
    return a.positions.p != nullptr ? given_position(tokens, index_at(a.positions, row)) : last_position(tokens, rows, i);
}

// Sums over the lanes up to and including each
__device__ __forceinline__ int wave_scan(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);      // row_shr:1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);      // row_bcast:15 to rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);      // row_bcast:31 to rows 2 and 3
    return v;
}
// A request: its cached tokens that are looked at, its new rows and where they begin
// With a window, tokens are counted without the `gap` of those between the sinks and the window, which no row sees.
struct Request {
    int tokens, rows, first, gap;
};
template <bool WINDOW>
__device__ __forceinline__ Request request_of(const AttendArgs &a, int b) {
    int first;
    const int rows = rows_of(a.row_start, b, a.n, a.max_rows, first), tokens = tokens_of(a.lengths[b], a.most);
    const int gap = WINDOW ? window_gap(tokens, a.positions.p != nullptr ? kTail : rows, a.window, a.sinks) : 0;
    return {tokens - gap, rows, first, gap};
}
__device__ __forceinline__ int request_steps(const Request &r) { return steps_of(r.tokens, r.rows, kAttendStep); }

// Where a workgroup's share of all requests' steps begins: request b, step `at` of it; `left` steps long (0: nothing), `per` being the
// shares' length.
struct Share {
    Request r;
    int b, at, left, per;
};
template <bool WINDOW>
__device__ __forceinline__ Share share_of(const AttendArgs &a, int place) {
    const int lane = lane_id();
    auto request = [&](int i) { return i < a.requests ? request_of<WINDOW>(a, i) : Request{0, 0, 0, 0}; };
    Request r = request(lane);
    const int mine = request_steps(r);
    int sum = mine;
#pragma unroll 4
    for (int base = 64; base < a.requests; base += 64) sum += request_steps(request(base + lane));
    const int all = a.requests <= 64 ? 0 : wave_sum_i32(sum);
    int upto = wave_scan(mine), last = __builtin_amdgcn_readlane(upto, 63);
    Share s;
    int start;
    s.left = share_steps(a.requests <= 64 ? last : __builtin_amdgcn_readfirstlane(all), a.places, place, s.per, start);
    if (s.left == 0) return s;
    int before = 0, base = 0;
    if (start >= last) {
        Request next = request(64 + lane);
        do {
            base += 64;
            if (base >= a.requests) {      // (start is below the steps of all, unless lengths are written to meanwhile)
                s.left = 0;
                return s;
            }
            before += last;
            r = next;
            next = request(base + 64 + lane);      // (under way while this block is looked at)
            upto = wave_scan(request_steps(r));
            last = __builtin_amdgcn_readlane(upto, 63);
        } while (start >= before + last);
    }
    const int at = __builtin_ctzll(__ballot(before + upto > start));
    s.b = base + at;
    s.at = start - before - (at == 0 ? 0 : __builtin_amdgcn_readlane(upto, at - 1));
    s.r = {__builtin_amdgcn_readlane(r.tokens, at), __builtin_amdgcn_readlane(r.rows, at), __builtin_amdgcn_readlane(r.first, at),
           WINDOW ? __builtin_amdgcn_readlane(r.gap, at) : 0};
    return s;
}

// Waves on a SIMD that the registers are cut to: as many as fit without scratch memory (fp32 rows of 256 values over a 16-bit cache keep
// 16 bytes of it, and read 8 of those, the tail mask, in the tiles that it applies to).  Two at least, so that there are 256 vector
// registers and no accumulation registers: copies out of those have come ahead of the matrix instructions' results here (a branch right
// behind the last product: clang 20 leaves out the wait states on its way), which the build checks there are none of.
template <int DP, int HELD, int NT, bool F32Q>
constexpr int attend_occupancy() {
    if (DP == 64) return NT == 1 ? 4 : NT == 2 ? 3 : 2;
    return 2;
}

template <int DP, int HELD, int NT, bool F32Q, bool WINDOW>
__global__ __launch_bounds__(64 * kAttendWaves, (attend_occupancy<DP, HELD, NT, F32Q>())) void attend_kernel(AttendArgs a) {
    constexpr int W = kAttendWaves, E = DP / 16, KS = DP / 32, TERMS = F32Q ? 3 : 1;      // (of q)
    constexpr bool FP8 = HELD == kHeld8, FP4 = HELD == kHeld4;
    constexpr int P_TERMS = FP4 && !F32Q ? 2 : 3;      // of the weights: over 4 bits the matrix and vector instructions are what there is too much of
    constexpr int KL = FP4 ? (DP + 127) / 128 : FP8 ? DP / 64 : DP / 32;      // loads of a token's row of K in a lane, of 16 bytes (FP4, DP = 64: of 8)
    constexpr int VR = FP4 ? (DP + 127) / 128 : FP8 ? DP / 64 : DP / 32;      // registers of a token's E values of V
    constexpr int BITS = FP4 ? 4 : FP8 ? 8 : 16;
    auto bytes = [](int values) { return values * BITS / 8; };
    constexpr int PITCH = DP + 4;
    // Rows of 256 values have no registers for a tile's keys and values at a time: values are asked for when the keys are used up, and
    // another wave's loads fill the time.
    constexpr bool LEAN = DP > 128;
    __shared__ float2 ms[W][16 * NT];
    __shared__ __align__(16) float sums[W][16 * NT][PITCH];

    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    // Workgroups go to the XCDs in turn: heads first, which have equal work, then the shares of a head's, which have too.
    const int place = blockIdx.y;
    int h = blockIdx.x, x0 = 0, x0_row = 0, x0_head = 0;      // the first of the query rows is head x0_head of the group, of new token x0_row
    if (a.row_blocks > 1) {
        x0 = h / a.cache.heads * 16 * NT;
        h %= a.cache.heads;
        x0_row = x0 / a.G, x0_head = x0 - x0_row * a.G;
    }
    const int D = a.cache.D, shift = a.cache.page_shift;
    Share share;
    if (a.whole) {
        share.b = place;
        share.at = share.per = 0;
        share.r = request_of<WINDOW>(a, place);
        share.left = request_steps(share.r);
    } else {
        share = share_of<WINDOW>(a, place);
        if (share.left == 0 && a.by_place && blockIdx.x == 0 && threadIdx.x == 0) a.part_at[place] = make_int4(place, 1, 0, 0);
    }

    // A part of a request after another, most often one or two
    for (int segment = 0; share.left > 0; ++segment) {
        // (another thread number each time to the compiler, which would keep all that follows from it in registers across the loop)
        int thread = threadIdx.x;
        asm volatile("" : "+v"(thread));
        const int lane = thread & 63, m = lane & 15, g = lane >> 4;
        const int b = share.b, at_step = share.at, len = share.r.tokens, nrows = share.r.rows, gap = share.r.gap;
        const int64_t first = share.r.first;
        const int32_t *pages = a.page_table + (int64_t)b * a.table_pages;
        int window = 0, ids = pages[min(lane, a.table_pages - 1)];
        const int steps = request_steps(share.r), take = min(share.left, steps - at_step);
        const bool complete = take == steps;
        share.left -= take;
        if (share.left > 0) {
            if (share.b + 1 >= a.requests) share.left = 0;      // (lengths that are written to meanwhile)
            else share.r = request_of<WINDOW>(a, ++share.b);
            share.at = 0;
        }
        // For the join: where the parts of each request are, or of the one request that a place may begin and not end.
        if (!a.whole && blockIdx.x == 0 && thread == 0) {
            const int4 parts = make_int4(place, complete ? 1 : 1 + (steps - take + share.per - 1) / share.per, segment != 0, b);
            const bool begins = take > 0 && at_step == 0;
            if (a.by_place) a.part_at[place] = begins ? parts : make_int4(place, 1, 0, b);
            else if (begins) a.part_at[b] = parts;
        }
        const int RG = nrows * a.G - x0;      // query rows from x0 on
        if (RG <= 0 || take <= 0) continue;
        const int t0 = at_step * kAttendStep;
        int t1 = complete ? len : min(len, t0 + take * kAttendStep);
        // WINDOW: a block of a chunk's rows ends at its last one, and leaves out what lies between the sinks and the window of its first
        int window_from = 0;
        if constexpr (WINDOW) {
            if (a.row_blocks > 1 && a.tail_mask == nullptr) {
                t1 = min(t1, last_position(len + gap, nrows, x0_row + by_group(a, x0_head + min(RG, 16 * NT) - 1)) + 1 - gap);
                window_from = last_position(len + gap, nrows, x0_row) - a.window + 1 - gap;
            }
        }
        const int64_t kept_at = (((int64_t)blockIdx.x * a.places + place) * 2 + (segment != 0)) * (16 * NT);
        float *const kept_o = a.part_o + kept_at * D;
        float2 *const kept_ms = a.part_ms + kept_at;

        // q's operand: row x0 + 16 nt + m is head h G + (x0_head + 16 nt + m) % G of new token x0_row + (x0_head + 16 nt + m) / G; the
        // values of d that the lane's K has
        u32x4 q[NT][KS * (F32Q ? 2 : 1)];
        uint64_t tail[NT];
        int from[NT], upto[NT];      // WINDOW: tokens that the row sees beside the sinks
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int x = 16 * nt + m, y = x0_head + min(x, RG - 1), up = by_group(a, y);
            const int64_t row = first + x0_row + up, at = row * a.q_stride + (h * a.G + y - up * a.G) * D;
            tail[nt] = a.tail_mask != nullptr ? a.tail_mask[row] : 0;
            if constexpr (WINDOW) {
                const int position = position_of(a, row, len + gap, nrows, x0_row + up);
                from[nt] = position - a.window + 1;
                upto[nt] = a.tail_mask != nullptr ? INT32_MAX : position;
            }
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const int d = FP4 ? DP / 4 * g + 8 * s : FP8 ? 64 * (s / 2) + 16 * g + 8 * (s % 2) : 32 * s + 8 * g;
                const bool there = x < RG && d < D;
                const int64_t from = at + (d < D ? d : 0);
#pragma unroll
                for (int i = 0; i < (F32Q ? 2 : 1); ++i) {
                    const u32x4 u = *reinterpret_cast<const u32x4 *>(static_cast<const char *>(a.q) + from * (F32Q ? 4 : 2) + 16 * i);
                    u32x4 &to = q[nt][(F32Q ? 2 : 1) * s + i];
                    to = there ? u : u32x4{0, 0, 0, 0};
                    if constexpr (F32Q) {      // (-0 is 0)
#pragma unroll
                        for (int j = 0; j < 4; ++j) to[j] = __float_as_uint(__uint_as_float(to[j]) + 0.0f);
                    }
                }
            }
        }

        // Page numbers of 64 pages, one in each lane.  (The empty asm has the wait for them where they are loaded: at the join of the branch it
        // would be for all loads under way.)
        const int last_page = max(len + gap - 1, 0) >> shift;
        // (the token that is counted as the t-th)
        const int sinks16 = WINDOW ? round16(a.sinks) : 0;
        auto real = [&](int t) { return WINDOW && t >= sinks16 ? t + gap : t; };
        if (real(t0) >> shift >= 64) {
            window = real(t0) >> shift;
            ids = pages[min(window + lane, last_page)];
        }
        asm volatile("" : "+v"(ids));
        // First row of 16 tokens (of one page: pages are multiples of 16) in the cache, or -1 where there is nothing to read.
        auto rows16 = [&](int t) -> int64_t {
            if (t >= t1) return -1;
            const int token = real(t), p = token >> shift;
            if (p >= window + 64) {
                window = p;
                ids = pages[min(p + lane, last_page)];
                asm volatile("" : "+v"(ids));
            }
            const int64_t row = row_of_page(__builtin_amdgcn_readlane(ids, p - window), a.cache.pages, a.cache.heads, h, shift);
            return row < 0 ? -1 : row + (token & ((1 << shift) - 1));
        };

        // 16 rows of the cache as a buffer: of no bytes where there are none, so that loads are issued for every tile alike, read zeros without
        // any traffic past the end, and no branch stands between a load and its wait.  A lane's offsets are within the 16 rows, or, past the
        // end of rows shorter than DP, beyond any buffer.
        constexpr int kBeyond = 1 << 30, kNt = 2;
        int k_at[KL];
#pragma unroll
        for (int s = 0; s < KL; ++s) {
            const int d = FP4 ? DP / 4 * g + 32 * s : FP8 ? 64 * s + 16 * g : 32 * s + 8 * g;
            k_at[s] = d < D ? bytes(m * D + d) : kBeyond;
        }
        const int v_at = E * m < D ? bytes(4 * g * D + E * m) : kBeyond;
        auto buffer = [&](const void *base, int64_t row, int row_bytes) {
            return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(static_cast<const char *>(base) + (row < 0 ? 0 : row) * row_bytes), 0,
                                                     row < 0 ? 0 : 16 * row_bytes, 0x00027000);
        };
        // 4 bits: scales of the 16 rows' groups, group j's `1 << shift` bytes after those of group j - 1
        auto scales_of_four = [&](const uint8_t *base, int64_t row) {
            const int groups = D / kScaleGroup;
            return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(base + (row < 0 ? 0 : scale_of_row(row, groups, 0, shift))), 0,
                                                     row < 0 ? 0 : ((groups - 1) << shift) + 16, 0x00027000);
        };
        const int v_scale_at = FP4 ? (E * m < D ? ((E * m / kScaleGroup) << shift) + 4 * g : kBeyond) : 4 * g;

        u32x4 k[2][KL];
        unsigned v[8][VR], k_scale[2][FP4 ? KL : 1] = {}, v_scale[2] = {};
        auto load_k = [&](const int64_t (&row)[2]) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const auto r = buffer(a.cache.k, row[t], bytes(D));
#pragma unroll
                for (int s = 0; s < KL; ++s) {
                    if constexpr (FP4 && DP == 64) {
                        const u32x2 u = __builtin_amdgcn_raw_buffer_load_b64(r, k_at[s], 0, kNt);
                        k[t][s].x = u.x, k[t][s].y = u.y;
                    } else {
                        k[t][s] = __builtin_amdgcn_raw_buffer_load_b128(r, k_at[s], 0, kNt);
                    }
                }
                if constexpr (FP8) k_scale[t][0] = __builtin_amdgcn_raw_buffer_load_b32(buffer(a.cache.k_scale, row[t], 1), 4 * g, 0, 0);
                if constexpr (FP4) {
#pragma unroll
                    for (int s = 0; s < KL; ++s) {
                        const int d = DP / 4 * g + 32 * s;
                        k_scale[t][s] = __builtin_amdgcn_raw_buffer_load_b8(scales_of_four(a.cache.k_scale, row[t]), d < D ? ((d / kScaleGroup) << shift) + m : kBeyond, 0, 0);
                    }
                }
            }
        };
        auto load_v = [&](const int64_t (&row)[2]) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const auto buf = buffer(a.cache.v, row[t], bytes(D));
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int at = v_at + i * bytes(D), j = 4 * t + i;
                    if constexpr (FP4 && DP == 64) {
                        v[j][0] = __builtin_amdgcn_raw_buffer_load_b16(buf, at, 0, kNt);
                    } else if constexpr (VR == 1) {
                        v[j][0] = __builtin_amdgcn_raw_buffer_load_b32(buf, at, 0, kNt);
                    } else if constexpr (VR == 2) {
                        const u32x2 u = __builtin_amdgcn_raw_buffer_load_b64(buf, at, 0, kNt);
                        v[j][0] = u.x, v[j][1] = u.y;
                    } else {
#pragma unroll
                        for (int r = 0; r < VR; r += 4) {
                            const u32x4 u = __builtin_amdgcn_raw_buffer_load_b128(buf, at + 4 * r, 0, kNt);
                            v[j][r] = u.x, v[j][r + 1] = u.y, v[j][r + 2] = u.z, v[j][r + 3] = u.w;
                        }
                    }
                }
                if constexpr (FP8) v_scale[t] = __builtin_amdgcn_raw_buffer_load_b32(buffer(a.cache.v_scale, row[t], 1), v_scale_at, 0, 0);
                if constexpr (FP4) v_scale[t] = __builtin_amdgcn_raw_buffer_load_b32(scales_of_four(a.cache.v_scale, row[t]), v_scale_at, 0, 0);
            }
        };

        f32x4a acc[NT][E];
        float top[NT], total[NT];      // of the lane's row; total over the lane's own tokens
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            top[nt] = kNone, total[nt] = 0.0f;
#pragma unroll
            for (int i = 0; i < E; ++i) acc[nt][i] = f32x4a{0, 0, 0, 0};
        }

        // Registers of V as operands of the product over its values 2 r, 2 r + 1 (16 bits) or 4 r .. 4 r + 3 (codes)
        // (4 bits: 8 r .. 8 r + 7, or 0 .. 3; their scales are in them, as `v_scale` differs from one 32 values to the next)
        constexpr int VF = FP4 ? (DP == 64 ? 4 : 8) : FP8 ? 4 : 2;
        auto operands = [&](int r, u32x4 (&f)[VF]) {
            if constexpr (FP4) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    unsigned one[VF / 2], two[VF / 2];
                    auto scale_of = [&](int i) { return i % 4 == 0 ? v_scale[i / 4] << 23 : i % 4 == 1 ? v_scale[i / 4] << 15 : i % 4 == 2 ? v_scale[i / 4] << 7 : v_scale[i / 4] >> 1; };
                    if constexpr (VF == 8) {
                        eight_codes(v[2 * j][r], scale_of(2 * j), one);
                        eight_codes(v[2 * j + 1][r], scale_of(2 * j + 1), two);
                    } else {
                        four_codes(v[2 * j][r], scale_of(2 * j), one);
                        four_codes(v[2 * j + 1][r], scale_of(2 * j + 1), two);
                    }
#pragma unroll
                    for (int i = 0; i < VF; i += 2) {
                        f[i][j] = __builtin_amdgcn_perm(two[i / 2], one[i / 2], 0x05040100);
                        f[i + 1][j] = __builtin_amdgcn_perm(two[i / 2], one[i / 2], 0x07060302);
                    }
                }
                return;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (!FP8) {
                    f[0][j] = __builtin_amdgcn_perm(v[2 * j + 1][r], v[2 * j][r], 0x05040100);
                    f[1][j] = __builtin_amdgcn_perm(v[2 * j + 1][r], v[2 * j][r], 0x07060302);
                } else {
                    // bytes: first token's value, second token's value, the next value of both
                    const unsigned lo = __builtin_amdgcn_perm(v[2 * j + 1][r], v[2 * j][r], 0x05010400);
                    const unsigned hi = __builtin_amdgcn_perm(v[2 * j + 1][r], v[2 * j][r], 0x07030602);
                    f[0][j] = two_codes<false>(lo), f[1][j] = two_codes<true>(lo);
                    f[2][j] = two_codes<false>(hi), f[3][j] = two_codes<true>(hi);
                }
            }
        };

        // NaN and infinities among values that some row does not see: 0 * inf must not reach it.  They are taken out of V, and counted in products
        // of ones for each row that sees them, whose sums become what they would have.
        unsigned p[NT][P_TERMS][4], sees[NT][4];
        auto take_out_odd = [&]() {
#pragma unroll
            for (int r = 0; r < VR; ++r) {
                u32x4 f[VF];
                operands(r, f);
#pragma unroll
                for (int i = 0; i < VF; ++i) {
                    u32x4 odd[3];      // NaN, +inf, -inf
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        odd[0][j] = odd[1][j] = odd[2][j] = 0;
#pragma unroll
                        for (int half = 0; half < 32; half += 16) {
                            const unsigned u = (f[i][j] >> half) & 0xFFFFu, one = 0x3F80u << half;
                            odd[0][j] |= (u & 0x7FFFu) > 0x7F80u ? one : 0u;
                            odd[1][j] |= u == 0x7F80u ? one : 0u;
                            odd[2][j] |= u == 0xFF80u ? one : 0u;
                        }
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const u32x4 seen = {sees[nt][0], sees[nt][1], sees[nt][2], sees[nt][3]};
                        const float add[3] = {__builtin_nanf(""), __builtin_inff(), -__builtin_inff()};
#pragma unroll
                        for (int kind = 0; kind < 3; ++kind) {
                            const f32x4a count = mfma(odd[kind], seen, f32x4a{0, 0, 0, 0});
#pragma unroll
                            for (int x = 0; x < 4; ++x) acc[nt][VF * r + i][x] += count[x] > 0.0f ? add[kind] : 0.0f;
                        }
                    }
                }
                if constexpr (FP4) continue;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    constexpr unsigned part = FP8 ? 0xFFu : 0xFFFFu, step = FP8 ? 8 : 16, odd = FP8 ? 0x7Fu : 0x7F80u;
                    unsigned clean = 0;
#pragma unroll
                    for (unsigned at = 0; at < 32; at += step) {
                        const unsigned u = (v[j][r] >> at) & part;
                        clean |= ((u & odd) == odd ? 0u : u) << at;
                    }
                    v[j][r] = clean;
                }
            }
            if constexpr (FP4) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    // the first magnitude that is infinite: 4 * 2^126, 2 * 2^127; of 255 all are NaN
                    const unsigned scale = (v_scale[j / 4] >> 8 * (j % 4)) & 0xFF, first = scale < 253 ? 8 : scale == 253 ? 6 : scale == 254 ? 4 : 0;
#pragma unroll
                    for (int r = 0; r < VR; ++r) {
                        unsigned clean = 0;
#pragma unroll
                        for (int at = 0; at < 32; at += 4) clean |= ((v[j][r] >> at) & 7) < first ? v[j][r] & (15u << at) : 0u;
                        v[j][r] = clean;
                    }
                    if (scale == 255) v_scale[j / 4] &= ~(0xFFu << 8 * (j % 4));
                }
            }
        };

        // the next tile of the wave that holds a token of the window, or of the sinks
        auto wanted = [&](int t) {
            if (WINDOW && t >= sinks16 && t + kAttendTile <= window_from) t += ((window_from - kAttendTile - t) / (kAttendTile * W) + 1) * (kAttendTile * W);
            return t;
        };
        int token = wanted(t0 + kAttendTile * wave);
        if (token < t1) {
            int64_t row[2] = {rows16(token), rows16(token + 16)};
            load_k(row);
            if constexpr (!LEAN) load_v(row);
            do {
                // scores: lane has tokens 16 t + 4 g + i of row m
                f32x4a s[NT][2];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = f32x4a{0, 0, 0, 0};
#pragma unroll
                for (int c = 0; c < KS; ++c) {
                    u32x4 terms[NT][TERMS];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        if constexpr (F32Q) asm volatile("" : "+v"(q[nt][2 * c]), "+v"(q[nt][2 * c + 1]));      // (split here, not ahead of the loop)
                        if constexpr (F32Q) {
                            float x[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(q[nt][2 * c + j / 4][j % 4]);
                            split_terms<3>(x, terms[nt]);
                        } else {
                            terms[nt][0] = q[nt][c];
                        }
                    }
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        u32x4 f;
                        if constexpr (FP4) {
                            unsigned pairs[4];
                            eight_codes(k[t][c / 4][c % 4], k_scale[t][c / 4] << 23, pairs);
                            f = u32x4{pairs[0], pairs[1], pairs[2], pairs[3]};
                        } else if constexpr (FP8) {
                            const unsigned u0 = k[t][c / 2][2 * (c % 2)], u1 = k[t][c / 2][2 * (c % 2) + 1];
                            f = u32x4{two_codes<false>(u0), two_codes<true>(u0), two_codes<false>(u1), two_codes<true>(u1)};
                        } else {
                            f = k[t][c];
                        }
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                            for (int e = TERMS - 1; e >= 0; --e) s[nt][t] = mfma(f, terms[nt][e], s[nt][t]);
                        }
                    }
                }
                float factor[2][4];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        factor[t][i] = FP8 ? scaled(a.scale_log2, (k_scale[t][0] >> 8 * i) & 0xFF) : a.scale_log2;
                }

                // the next tile's keys are asked for once this one's are used up, its values likewise below
                const int next = wanted(token + kAttendTile * W);
                int64_t next_row[2] = {rows16(next), rows16(next + 16)};
                if constexpr (!LEAN) load_k(next_row);
                else load_v(row);

                const bool ends = token + kAttendTile > t1 || row[0] < 0 || row[1] < 0;
                const int tokens[2] = {real(token), real(token + 16)};      // first ones of the two 16
                const bool tail_masked = a.tail_mask != nullptr && tokens[1] + 16 > len + gap - kTail;
                bool masked = tail_masked;
                if constexpr (WINDOW) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                        for (int t = 0; t < 2; ++t) masked |= __any((tokens[t] < from[nt] && tokens[t] + 15 >= a.sinks) || tokens[t] + 15 > upto[nt]) != 0;
                    }
                }
                // bit i: whether there is a token 16 t + 4 g + i
                unsigned there[2] = {15, 15};
                if (ends) {
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        const int left = t1 - (token + 16 * t + 4 * g);
                        there[t] = row[t] < 0 || left <= 0 ? 0u : left >= 4 ? 15u : (1u << left) - 1u;
                    }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float z[2][4];
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) z[t][i] = s[nt][t][i] * factor[t][i];
                    }
                    if (ends || masked) {
#pragma unroll
                        for (int t = 0; t < 2; ++t) {
                            unsigned seen = there[t];
                            if (tail_masked) {
                                const int bit = tokens[t] + 4 * g - (len + gap - kTail);      // of the first of the four; bits before the first: seen
                                const unsigned bits = (unsigned)(tail[nt] >> min(max(bit, 0), 63)), before = min(max(-bit, 0), 4);
                                seen &= (bit < 64 ? bits << before : 0u) | ((1u << before) - 1u);
                            }
                            if constexpr (WINDOW) {
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const int at = tokens[t] + 4 * g + i;
                                    if ((at < from[nt] && at >= a.sinks) || at > upto[nt]) seen &= ~(1u << i);
                                }
                            }
#pragma unroll
                            for (int i = 0; i < 4; ++i) z[t][i] = (seen >> i) & 1 ? z[t][i] : kNone;
                        }
                    }
                    float most = top[nt];
#pragma unroll
                    for (int t = 0; t < 2; ++t) most = fmaxf(most, fmaxf(fmaxf(z[t][0], z[t][1]), fmaxf(z[t][2], z[t][3])));
                    most = row_max(most);
                    // (a row that has seen nothing yet: exp2(-inf - 0) = 0)
                    const float base = most == kNone ? 0.0f : most;
                    const float fade = __builtin_amdgcn_exp2f(top[nt] - base);
                    if (token != t0 + kAttendTile * wave && __any(most > top[nt])) {      // (the first tile has nothing to rescale)
#pragma unroll
                        for (int i = 0; i < E; ++i) {
#pragma unroll
                            for (int r = 0; r < 4; ++r) acc[nt][i][r] *= fade;
                        }
                    }
                    top[nt] = most;
                    float w[8], sum = 0.0f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        w[j] = __builtin_amdgcn_exp2f(z[j / 4][j % 4] - base);
                        sum += w[j];
                    }
                    total[nt] = total[nt] * fade + sum;
                    if (masked) {
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            sees[nt][j] = (z[j / 2][2 * j % 4] > kNone ? 0x3F80u : 0u) | (z[j / 2][2 * j % 4 + 1] > kNone ? 0x3F800000u : 0u);
                    }
                    if constexpr (FP8) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) w[j] = scaled(w[j], (v_scale[j / 4] >> 8 * (j % 4)) & 0xFF);      // (0 stays, whatever is held)
                    }
                    split_terms<P_TERMS>(w, p[nt]);
                }
                if (ends) {
                    // what lies past the end may be anything, NaN too
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
#pragma unroll
                        for (int r = 0; r < VR; ++r) v[j][r] = (there[j / 4] >> j % 4) & 1 ? v[j][r] : 0u;
                        if constexpr (FP4) v_scale[j / 4] &= (there[j / 4] >> j % 4) & 1 ? ~0u : ~(0xFFu << 8 * (j % 4));
                    }
                }
                bool hard = false;
                if (masked) {
                    unsigned odd = 0;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
#pragma unroll
                        for (int r = 0; r < VR; ++r) {
                            if constexpr (FP4) continue;
                            else if constexpr (FP8) odd |= ((v[j][r] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
                            else odd |= ((v[j][r] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
                        }
                    }
                    if constexpr (FP4) {      // a scale of 253 or more
#pragma unroll
                        for (int t = 0; t < 2; ++t) odd |= ((v_scale[t] & 0x7F7F7F7Fu) + 0x03030303u) & v_scale[t] & 0x80808080u;
                    }
                    hard = __any(odd != 0);
                }
                if (hard) take_out_odd();
#pragma unroll
                for (int r = 0; r < VR; ++r) {
                    u32x4 f[VF];
                    operands(r, f);
#pragma unroll
                    for (int e = P_TERMS - 1; e >= 0; --e) {
#pragma unroll
                        for (int i = 0; i < VF; ++i) {
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
                                acc[nt][VF * r + i] = mfma(f[i], u32x4{p[nt][e][0], p[nt][e][1], p[nt][e][2], p[nt][e][3]}, acc[nt][VF * r + i]);
                        }
                    }
                }
                if constexpr (!LEAN) load_v(next_row);
                else load_k(next_row);
                token = next;
                row[0] = next_row[0], row[1] = next_row[1];
            } while (token < t1);
        }

        // The waves' sums joined: each brings its rows to the common maximum.  A sum of 0 is a wave without tokens for the row (one of -inf
        // scores, too): it adds nothing.  (NaN has a sum, of NaN, and no maximum.)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            total[nt] = row_sum(total[nt]);
            if (g == 0) ms[wave][16 * nt + m] = make_float2(top[nt], total[nt]);
        }
        __syncthreads();
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float2 part[W];
            float most = kNone, all = 0.0f;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                part[w] = ms[w][16 * nt + m];
                most = fmaxf(most, part[w].x);
            }
#pragma unroll
            for (int w = 0; w < W; ++w) all += part[w].y == 0.0f ? 0.0f : part[w].y * __builtin_amdgcn_exp2f(part[w].x - most);
            float fade = total[nt] == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(top[nt] - most);
            if (complete) fade = all == 0.0f ? 0.0f : fade / all;
            if (__any(total[nt] == 0.0f)) {      // (values of infinity times p = 0 may be there)
#pragma unroll
                for (int i = 0; i < E; ++i) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[nt][i][r] = total[nt] == 0.0f ? 0.0f : acc[nt][i][r];
                }
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
#pragma unroll
                for (int i = 0; i < E; i += 4) {
                    float o[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[j] = acc[nt][i + j][r] * fade;
                    F32::store4(&sums[wave][16 * nt + m][4 * E * g + E * r + i], o);
                }
            }
            if (wave == 0 && g == 0 && 16 * nt + m < RG) {
                const int y = x0_head + 16 * nt + m, up = by_group(a, y);
                if (!complete) kept_ms[16 * nt + m] = make_float2(most, all);
                else if (a.lse != nullptr) a.lse[(first + x0_row + up) * a.hq + h * a.G + y - up * a.G] = log_sum_exp(most, all);
            }
        }
        __syncthreads();
        constexpr int PER = 64 * W / (DP / 4);      // rows that the workgroup takes at a time
        const int d = 4 * (thread % (DP / 4));
#pragma unroll
        for (int c = 0; c < 16 * NT; c += PER) {
            const int x = c + thread / (DP / 4);
            if (x >= RG || d >= D) continue;
            float o[4] = {};
#pragma unroll
            for (int w = 0; w < W; ++w) {
                float u[4];
                F32::load4(&sums[w][x][d], u);
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] += u[i];
            }
            if (!complete) {
                F32::store4(kept_o + (x * D + d), o);
                continue;
            }
            const int y = x0_head + x, up = by_group(a, y);
            store_values(a, (first + x0_row + up) * a.out_stride + (h * a.G + y - up * a.G) * D + d, o, F32Q);
        }
        if (share.left > 0) __syncthreads();
    }
}

template <int DP, int HELD, int NT, bool F32Q, bool WINDOW>
hipError_t run_attend(const AttendArgs &a, hipStream_t st) {
    const dim3 grid((unsigned)(a.cache.heads * a.row_blocks), (unsigned)a.places);
    attend_kernel<DP, HELD, NT, F32Q, WINDOW><<<grid, 64 * kAttendWaves, 0, st>>>(a);
    return hipGetLastError();
}
template <int DP, int NT, bool F32Q, bool WINDOW>
hipError_t run_attend(const AttendArgs &a, hipStream_t st) {
    if (a.cache.four) return run_attend<DP, kHeld4, NT, F32Q, WINDOW>(a, st);
    return a.cache.k_scale != nullptr ? run_attend<DP, kHeld8, NT, F32Q, WINDOW>(a, st) : run_attend<DP, kHeld16, NT, F32Q, WINDOW>(a, st);
}

}  // namespace vt
