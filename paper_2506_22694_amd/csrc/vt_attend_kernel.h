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
// and on p, where they are exact as well.
//
// Values of 24 bits -- the weights p, and q of fp32 rows -- are sums of three of 8, so they are three operands each, and products are exact as
// for bf16.  An infinity on the other side is still one after three products only if all three terms have the value's sign and none is
// zero: the first two are cut off from just below what they are taken of.  (p as one operand, rounded to bf16: results in bf16 off by 0.0018
// to 0.0021 of their size instead of 0.0016 to 0.0017, their own rounding; 131001 tokens as long, 64 tree levels of 8 nodes 83 instead of 84 us, over
// 8 bits 61 instead of 65, 16 nodes of 64 heads of 64 values 71 instead of 81.)
//
// 131001 tokens of one request, 8 kv heads of 128 values in bf16, 4 query heads each: 537 MB in 80 us, 6.7 TB/s, where a plain read of as much
// takes 79; 224 vector and 32 matrix instructions a tile (8 bits: 317 and 32; 48 ragged requests 541 MB in 95 us, 5.7 TB/s).
#pragma once
#include "vt_values.h"

namespace vt {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4a;

__device__ __forceinline__ f32x4a mfma(u32x4 a, u32x4 b, f32x4a c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// bf16 pairs of two codes: the lower or upper two of a register
template <bool HIGH>
__device__ __forceinline__ unsigned two_codes(unsigned u) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, 1.0f, HIGH));
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
template <typename Terms>
__device__ __forceinline__ void split_terms(float (&v)[8], Terms &terms) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
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
struct Request {
    int tokens, rows, first;
};
__device__ __forceinline__ Request request_of(const AttendArgs &a, int b) {
    int first;
    const int rows = rows_of(a.row_start, b, a.n, a.max_rows, first);
    return {tokens_of(a.lengths[b], a.most), rows, first};
}
__device__ __forceinline__ int request_steps(const Request &r) { return steps_of(r.tokens, r.rows, kAttendStep); }

// Where a workgroup's share of all requests' steps begins: request b, step `at` of it; `left` steps long (0: nothing), `per` being the
// shares' length.
struct Share {
    Request r;
    int b, at, left, per;
};
__device__ __forceinline__ Share share_of(const AttendArgs &a, int place) {
    const int lane = lane_id();
    auto request = [&](int i) { return i < a.requests ? request_of(a, i) : Request{0, 0, 0}; };
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
    s.r = {__builtin_amdgcn_readlane(r.tokens, at), __builtin_amdgcn_readlane(r.rows, at), __builtin_amdgcn_readlane(r.first, at)};
    return s;
}

// Waves on a SIMD that the registers are cut to: as many as fit without scratch memory (fp32 rows of 256 values over a 16-bit cache keep
// 16 bytes of it, and read 8 of those, the tail mask, in the tiles that it applies to).  Two at least, so that there are 256 vector
// registers and no accumulation registers: copies out of those have come ahead of the matrix instructions' results here (a branch right
// behind the last product: clang 20 leaves out the wait states on its way), which the build checks there are none of.
template <int DP, bool FP8, int NT, bool F32Q>
constexpr int attend_occupancy() {
    if (DP == 64) return NT == 1 ? 4 : NT == 2 ? 3 : 2;
    return 2;
}

template <int DP, bool FP8, int NT, bool F32Q>
__global__ __launch_bounds__(64 * kAttendWaves, (attend_occupancy<DP, FP8, NT, F32Q>())) void attend_kernel(AttendArgs a) {
    constexpr int W = kAttendWaves, E = DP / 16, KS = DP / 32, TERMS = F32Q ? 3 : 1;      // (of q)
    constexpr int KL = FP8 ? DP / 64 : DP / 32;       // 16-byte loads of a token's row of K in a lane
    constexpr int VR = FP8 ? DP / 64 : DP / 32;       // registers of a token's E values of V
    constexpr int SZ = FP8 ? 1 : 2;
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
        share.r = request_of(a, place);
        share.left = request_steps(share.r);
    } else {
        share = share_of(a, place);
        if (share.left == 0 && a.by_place && blockIdx.x == 0 && threadIdx.x == 0) a.part_at[place] = make_int4(place, 1, 0, 0);
    }

    // A part of a request after another, most often one or two
    for (int segment = 0; share.left > 0; ++segment) {
        // (another thread number each time to the compiler, which would keep all that follows from it in registers across the loop)
        int thread = threadIdx.x;
        asm volatile("" : "+v"(thread));
        const int lane = thread & 63, m = lane & 15, g = lane >> 4;
        const int b = share.b, at_step = share.at, len = share.r.tokens, nrows = share.r.rows;
        const int64_t first = share.r.first;
        const int32_t *pages = a.page_table + (int64_t)b * a.table_pages;
        int window = 0, ids = pages[min(lane, a.table_pages - 1)];
        const int steps = request_steps(share.r), take = min(share.left, steps - at_step);
        const bool complete = take == steps;
        share.left -= take;
        if (share.left > 0) {
            if (share.b + 1 >= a.requests) share.left = 0;      // (lengths that are written to meanwhile)
            else share.r = request_of(a, ++share.b);
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
        const int t0 = at_step * kAttendStep, t1 = complete ? len : min(len, t0 + take * kAttendStep);
        const int64_t kept_at = (((int64_t)blockIdx.x * a.places + place) * 2 + (segment != 0)) * (16 * NT);
        float *const kept_o = a.part_o + kept_at * D;
        float2 *const kept_ms = a.part_ms + kept_at;

        // q's operand: row x0 + 16 nt + m is head h G + (x0_head + 16 nt + m) % G of new token x0_row + (x0_head + 16 nt + m) / G; the
        // values of d that the lane's K has
        u32x4 q[NT][KS * (F32Q ? 2 : 1)];
        uint64_t tail[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int x = 16 * nt + m, y = x0_head + min(x, RG - 1), up = by_group(a, y);
            const int64_t row = first + x0_row + up, at = row * a.q_stride + (h * a.G + y - up * a.G) * D;
            tail[nt] = a.tail_mask != nullptr ? a.tail_mask[row] : 0;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const int d = FP8 ? 64 * (s / 2) + 16 * g + 8 * (s % 2) : 32 * s + 8 * g;
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
        const int last_page = max(len - 1, 0) >> shift;
        if (t0 >> shift >= 64) {
            window = t0 >> shift;
            ids = pages[min(window + lane, last_page)];
        }
        asm volatile("" : "+v"(ids));
        // First row of 16 tokens (of one page: pages are multiples of 16) in the cache, or -1 where there is nothing to read.
        auto rows16 = [&](int token) -> int64_t {
            if (token >= t1) return -1;
            const int p = token >> shift;
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
            const int d = FP8 ? 64 * s + 16 * g : 32 * s + 8 * g;
            k_at[s] = d < D ? (m * D + d) * SZ : kBeyond;
        }
        const int v_at = E * m < D ? (4 * g * D + E * m) * SZ : kBeyond;
        auto buffer = [&](const void *base, int64_t row, int row_bytes) {
            return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(static_cast<const char *>(base) + (row < 0 ? 0 : row) * row_bytes), 0,
                                                     row < 0 ? 0 : 16 * row_bytes, 0x00027000);
        };

        u32x4 k[2][KL];
        unsigned v[8][VR], k_scale[2] = {}, v_scale[2] = {};
        auto load_k = [&](const int64_t (&row)[2]) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const auto r = buffer(a.cache.k, row[t], D * SZ);
#pragma unroll
                for (int s = 0; s < KL; ++s) k[t][s] = __builtin_amdgcn_raw_buffer_load_b128(r, k_at[s], 0, kNt);
                if constexpr (FP8) k_scale[t] = __builtin_amdgcn_raw_buffer_load_b32(buffer(a.cache.k_scale, row[t], 1), 4 * g, 0, 0);
            }
        };
        auto load_v = [&](const int64_t (&row)[2]) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const auto buf = buffer(a.cache.v, row[t], D * SZ);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int at = v_at + i * D * SZ, j = 4 * t + i;
                    if constexpr (VR == 1) {
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
                if constexpr (FP8) v_scale[t] = __builtin_amdgcn_raw_buffer_load_b32(buffer(a.cache.v_scale, row[t], 1), 4 * g, 0, 0);
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
        constexpr int VF = FP8 ? 4 : 2;
        auto operands = [&](int r, u32x4 (&f)[VF]) {
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
        unsigned p[NT][3][4], sees[NT][4];
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
        };

        int token = t0 + kAttendTile * wave;
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
                            split_terms(x, terms[nt]);
                        } else {
                            terms[nt][0] = q[nt][c];
                        }
                    }
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        u32x4 f;
                        if constexpr (FP8) {
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
                        factor[t][i] = FP8 ? scaled(a.scale_log2, (k_scale[t] >> 8 * i) & 0xFF) : a.scale_log2;
                }

                // the next tile's keys are asked for once this one's are used up, its values likewise below
                const int next = token + kAttendTile * W;
                int64_t next_row[2] = {rows16(next), rows16(next + 16)};
                if constexpr (!LEAN) load_k(next_row);
                else load_v(row);

                const bool ends = token + kAttendTile > t1 || row[0] < 0 || row[1] < 0;
                const bool masked = a.tail_mask != nullptr && token + kAttendTile > len - 64;
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
                            if (masked) {
                                const int bit = token + 16 * t + 4 * g - (len - 64);      // of the first of the four; bits before the first: seen
                                const unsigned bits = (unsigned)(tail[nt] >> min(max(bit, 0), 63)), before = min(max(-bit, 0), 4);
                                seen &= (bit < 64 ? bits << before : 0u) | ((1u << before) - 1u);
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
                    split_terms(w, p[nt]);
                }
                if (ends) {
                    // what lies past the end may be anything, NaN too
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
#pragma unroll
                        for (int r = 0; r < VR; ++r) v[j][r] = (there[j / 4] >> j % 4) & 1 ? v[j][r] : 0u;
                    }
                }
                bool hard = false;
                if (masked) {
                    unsigned odd = 0;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
#pragma unroll
                        for (int r = 0; r < VR; ++r) {
                            if constexpr (FP8) odd |= ((v[j][r] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
                            else odd |= ((v[j][r] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
                        }
                    }
                    hard = __any(odd != 0);
                }
                if (hard) take_out_odd();
#pragma unroll
                for (int r = 0; r < VR; ++r) {
                    u32x4 f[VF];
                    operands(r, f);
#pragma unroll
                    for (int e = 2; e >= 0; --e) {
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

template <int DP, bool FP8, int NT, bool F32Q>
hipError_t run_attend(const AttendArgs &a, hipStream_t st) {
    const dim3 grid((unsigned)(a.cache.heads * a.row_blocks), (unsigned)a.places);
    attend_kernel<DP, FP8, NT, F32Q><<<grid, 64 * kAttendWaves, 0, st>>>(a);
    return hipGetLastError();
}
template <int DP, int NT, bool F32Q>
hipError_t run_attend(const AttendArgs &a, hipStream_t st) {
    return a.cache.k_scale != nullptr ? run_attend<DP, true, NT, F32Q>(a, st) : run_attend<DP, false, NT, F32Q>(a, st);
}

}  // namespace vt
