// Attention of many rows of a request at a time -- a prompt's chunk -- over the cache with a sliding window and sinks, on the matrix cores.
//
// Bound by the products: a row of q meets every token of its window, and a workgroup's 64 NT query rows share what is read, so that the cache's
// bytes are few beside them.  Tiles of TN tokens go through LDS, as bf16 whatever the cache holds, twice: one is computed on while the next one's
// loads are under way.  Each of the four waves has 16 NT query rows (the heads that share a kv head, times new tokens) of its own:
//
//   scores^T [token, row] = K q^T      K's operand: a token's 16 bytes in a lane, from LDS; q stays in registers
//   out^T [d, row] = V^T p^T           V's operand: four tokens of one column in a lane, by the transposing read of LDS; p's operand is what the
//                                      first product leaves in a lane, so the running maxima and sums are a lane's own
//
// 16 bytes c of token t lie at place c ^ key(t) of the token's row in LDS, so that the sixteen lanes that read sixteen rows of K use all of its 64 banks.  (The transposing reads
// of V meet in banks: 24 % of LDS's cycles are conflicts, 38 % with 64-value heads.)
//
// A weight p goes into the product as two bf16 terms, 16 bits of it, off by 2^-16 at most (one term, 8 bits, would be as large an error as the result's own rounding,
// 2^-8; the third, which attention of few rows has, is 2^-8 of an error that the rounding of bf16 results hides already).
//
// 8192 rows of 32 heads of 128 values over 8, a window of 4096 in bf16: 575 to 595 us, 695 to 718 TFLOP/s, once the card's clock has settled (the first some fifty calls after other
// work 660 to 810); a tile of a wave is 96 matrix instructions and some 310 others, which hardly overlap on a SIMD (a wave of products beside one of multiply-adds: 95 % of the sum
// of both) and take 90 % of its cycles.  64 query rows a workgroup where 128 are too few of them (one chunk of 256 rows, split as well).
#pragma once
#include "vt_attend_kernel.h"

namespace vt {

// Where the partial results of share z of the workgroup's rows begin, in blocks of its rows
__device__ __forceinline__ int64_t prompt_part(const AttendArgs &a, int z) { return ((int64_t)z * a.requests + blockIdx.y) * (a.cache.heads * a.row_blocks) + blockIdx.x; }

template <int DP, int HELD, int NT>
__global__ __launch_bounds__(256, 2) void prompt_kernel(AttendArgs a) {
    constexpr int W = 4, E = DP / 16, KS = DP / 32, CH = DP / 8;      // CH: 16-byte places of a row in LDS
    constexpr int TN = DP <= 128 ? 64 : 32, PIECES = TN / 16;
    constexpr int PER = HELD == kHeld16 ? 8 : HELD == kHeld8 ? 16 : 32;      // values of a 16-byte load
    constexpr int COLS = DP / PER, LOADS = (16 * COLS + 63) / 64;            // loads of a row; of a lane for 16 rows
    constexpr int UNITS = 2 * PIECES / W;                                    // 16 rows of K or V that a wave brings
    __shared__ __align__(512) u32x4 held[2][2][TN][CH];
    auto key = [](int t) { return CH >= 16 ? t & 15 : t >> 1 & 7; };
    __shared__ __align__(16) int flags[2][4];      // of the pieces.  1: a page outside the cache, 2: NaN or infinities among the values

    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const int h = blockIdx.x % a.cache.heads, block = a.row_blocks - 1 - blockIdx.x / a.cache.heads, b = blockIdx.y;      // (the longest first)
    const int D = a.cache.D, shift = a.cache.page_shift;
    int first;
    const int rows = rows_of(a.row_start, b, a.n, a.max_rows, first), len = tokens_of(a.lengths[b], a.most);
    const int x0 = block * 16 * NT * W, all = rows * a.G;
    if (x0 >= all) return;
    // tokens that any of the workgroup's rows sees: `end` and those before it but for the gap
    const int x0_row = x0 / a.G, x0_head = x0 - x0_row * a.G;
    const int lowest = last_position(len, rows, x0_row), highest = last_position(len, rows, (min(x0 + 16 * NT * W, all) - 1) / a.G);
    const int end = max(highest + 1, 0), sinks16 = min(round16(a.sinks), round16(end));
    const int gap = max((max(lowest - a.window + 1, 0) & ~15) - sinks16, 0), count = end - gap;
    auto real = [&](int t) { return t >= sinks16 ? t + gap : t; };
    // of those the workgroup's share, one of gridDim.z
    const int share = (count + TN * (int)gridDim.z - 1) / (TN * (int)gridDim.z) * TN, begin = min((int)blockIdx.z * share, max(count, 0)), stop = min(begin + share, count);

    // q's operand (its sign that of the scale, so that the largest score stays the largest when it is scaled), and what the lane's rows see
    const float by = fabsf(a.scale_log2);
    const unsigned turn = a.scale_log2 < 0.0f ? 0x80008000u : 0u;
    u32x4 q[NT][KS];
    int from[NT], upto[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int x = 16 * (NT * wave + nt) + m, y = x0_head + min(x, all - x0 - 1), up = by_group(a, y);
        const int64_t at = (first + (int64_t)x0_row + up) * a.q_stride + (h * a.G + y - up * a.G) * D;
        upto[nt] = last_position(len, rows, x0_row + up);
        from[nt] = upto[nt] - a.window + 1;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int d = 32 * s + 8 * g;
            const u32x4 u = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(a.q) + at + (d < D ? d : 0));
            q[nt][s] = d < D && by != 0.0f ? u ^ turn : u32x4{0, 0, 0, 0};
        }
    }

    // Page numbers of 64 pages, one in each lane
    const int32_t *pages = a.page_table + (int64_t)b * a.table_pages;
    const int last_page = max(end - 1, 0) >> shift;
    int window = real(begin) >> shift, ids = pages[min(window + lane, last_page)];
    auto rows16 = [&](int t) -> int64_t {      // of the cache, or -1
        if (t >= count) return -1;
        const int token = real(t), p = token >> shift;
        if (p >= window + 64) {
            window = p;
            ids = pages[min(p + lane, last_page)];
        }
        const int64_t row = row_of_page(__builtin_amdgcn_readlane(ids, p - window), a.cache.pages, a.cache.heads, h, shift);
        return row < 0 ? -1 : row + (token & ((1 << shift) - 1));
    };

    // What the wave brings of a tile: unit u is piece (W u + wave) % PIECES of K (the first PIECES of the 2 PIECES) or V
    constexpr int kBeyond = 1 << 30, BITS = HELD == kHeld16 ? 16 : HELD == kHeld8 ? 8 : 4;
    struct Raw {
        u32x4 raw[LOADS];
        unsigned scale[LOADS];
    } next;
    int64_t row = -1;      // of the wave's piece (the same one of K and V where it brings both)
    auto bring = [&](int u, int t0, Raw &x) __attribute__((always_inline)) {
        const int unit = W * u + wave, piece = unit % PIECES;
        const bool is_v = unit >= PIECES;
        if (u == 0) row = rows16(t0 + 16 * piece);
        const int row_bytes = D * BITS / 8;
        const auto buffer = __builtin_amdgcn_make_buffer_rsrc(static_cast<char *>(is_v ? a.cache.v : a.cache.k) + (row < 0 ? 0 : row) * row_bytes, 0,
                                                              row < 0 ? 0 : 16 * row_bytes, 0x00027000);
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int id = 64 * j + lane, r = id / COLS, c = id % COLS;
            const bool inside = r < 16 && c * PER < D;
            x.raw[j] = __builtin_amdgcn_raw_buffer_load_b128(buffer, inside ? r * row_bytes + 16 * c : kBeyond, 0, 0);
            if constexpr (HELD != kHeld16) {
                const int groups = HELD == kHeld4 ? D / kScaleGroup : 1;
                const uint8_t *const scales = is_v ? a.cache.v_scale : a.cache.k_scale;
                const auto of = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(scales + (row < 0 ? 0 : scale_of_row(row, groups, 0, shift))), 0,
                                                                  row < 0 ? 0 : ((groups - 1) << shift) + 16, 0x00027000);
                x.scale[j] = __builtin_amdgcn_raw_buffer_load_b8(of, inside ? (HELD == kHeld4 ? c << shift : 0) + r : kBeyond, 0, 0);
            }
        }
    };
    // ... into LDS.  `edge`: some row does not see some token of the tile
    auto keep = [&](int u, int buf, int t0, bool edge, const Raw &x) __attribute__((always_inline)) {
        const int unit = W * u + wave, piece = unit % PIECES;
        const int is_v = unit >= PIECES;
        unsigned odd = 0;
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int id = 64 * j + lane, r = id / COLS, c = id % COLS;
            if (16 * COLS % 64 != 0 && r >= 16) continue;
            u32x4 out[PER / 8];
            const unsigned s = HELD == kHeld16 ? 0 : x.scale[j] << 23;
            if constexpr (HELD == kHeld16) {
                out[0] = x.raw[j];
            } else if constexpr (HELD == kHeld8) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const unsigned w = x.raw[j][i];
                    out[i / 2][2 * (i % 2)] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, __uint_as_float(s), false));
                    out[i / 2][2 * (i % 2) + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, __uint_as_float(s), true));
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    unsigned f[4];
                    eight_codes(x.raw[j][i], s, f);
                    out[i] = u32x4{f[0], f[1], f[2], f[3]};
                }
            }
#pragma unroll
            for (int i = 0; i < PER / 8; ++i) {
                if (edge && is_v) {
                    if (t0 + 16 * piece + r >= count) out[i] = u32x4{0, 0, 0, 0};      // (past the end there may be anything)
#pragma unroll
                    for (int k = 0; k < 4; ++k) odd |= ((out[i][k] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
                }
                held[buf][is_v][16 * piece + r][(c * (PER / 8) + i) ^ key(r)] = out[i];
            }
        }
        if (is_v) {
            const int bits = (row >= 0 || t0 + 16 * piece >= count ? 0 : 1) | (__any(odd != 0) ? 2 : 0);
            if (lane == 0) flags[buf][piece] = bits;
        }
    };
    auto edge_of = [&](int t0) {
        return t0 < highest - a.window + 1 - gap || t0 + TN > lowest + 1 - gap;
    };

    f32x4a acc[NT][E];
    float top[NT], total[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        top[nt] = kNone, total[nt] = 0.0f;
#pragma unroll
        for (int i = 0; i < E; ++i) acc[nt][i] = f32x4a{0, 0, 0, 0};
    }

    const float scale_by = by != 0.0f ? by : 1.0f;      // (then q is zeros)
    typedef __attribute__((ext_vector_type(4))) short s16x4;
    typedef __attribute__((address_space(3))) char Lds;
    typedef __attribute__((address_space(3))) u32x4 LdsVector;
    typedef __attribute__((address_space(3))) s16x4 LdsFour;
    // where a lane reads: of K places 4 c + g of row m, of V column pairs 2 i + (m % 4) / 2 of row 4 g + m / 4.  Rows are aligned to their size, so that c
    // and i are exclusive ors of a constant, and all else is a constant to add.
    const unsigned lds = (unsigned)(size_t)(Lds *)&held[0][0][0][0];
    const unsigned k_at = lds + 16 * (m * CH + (g ^ key(m))), v_at = lds + 16 * ((4 * g + m / 4) * CH + ((m % 4 / 2) ^ key(4 * g + m / 4))) + 8 * (m % 2);
    // NaN and infinities among values that some row sees and another one does not: added to those that see them (at scores above -inf, as attend_kernel does), and
    // taken out, as 0 * inf must not reach the others.  (Out of line, a token after the other: what no sound cache holds.)
    auto take_out_odd = [&](int buf, const f32x4a (&z)[NT][PIECES]) __attribute__((always_inline)) {
        unsigned sees[NT] = {};      // bit 4 t + i: of token 16 t + 4 g + i
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int j = 4 * PIECES - 1; j >= 0; --j) sees[nt] = 2 * sees[nt] + (z[nt][j / 4][j % 4] > kNone ? 1u : 0u);
        }
#pragma unroll 1
        for (int t = 0; t < TN; ++t) {
            bool seen[NT];      // by the lane's row
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
                seen[nt] = ((unsigned)__builtin_amdgcn_ds_bpermute(4 * ((t & 12) * 4 + m), (int)sees[nt]) >> (4 * (t >> 4) + (t & 3)) & 1) != 0;
            const char *const row = reinterpret_cast<const char *>(held[buf][1][t]);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const u32x2 u = *reinterpret_cast<const u32x2 *>(row + 16 * ((2 * i + g / 2) ^ key(t)) + 8 * (g % 2));
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const unsigned bits = r % 2 ? u[r / 2] & 0xFFFF0000u : u[r / 2] << 16;
                    const float odd = (bits & 0x7F800000u) == 0x7F800000u ? __uint_as_float(bits) : 0.0f;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) acc[nt][i][r] += seen[nt] ? odd : 0.0f;
                }
            }
        }
        __syncthreads();
        for (int at = threadIdx.x; at < TN * CH; at += 256) {
            u32x4 &u = held[buf][1][at / CH][at % CH];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if ((u[k] & 0x7F80u) == 0x7F80u) u[k] &= 0xFFFF0000u;
                if ((u[k] & 0x7F800000u) == 0x7F800000u) u[k] &= 0x0000FFFFu;
            }
        }
        __syncthreads();
    };
    // `middle` is between the products
    auto tile = [&](int buf, int t0, bool edge, auto middle) __attribute__((always_inline)) {
        const int shifted = buf * (2 * TN * CH * 16);
        f32x4a s[NT][PIECES];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int t = 0; t < PIECES; ++t) s[nt][t] = f32x4a{0, 0, 0, 0};
        }
#pragma unroll
        for (int c = 0; c < KS; ++c) {
#pragma unroll
            for (int t = 0; t < PIECES; ++t) {
                const u32x4 f = *reinterpret_cast<const LdsVector *>((Lds *)(size_t)((k_at + shifted) ^ 64u * c) + 16 * 16 * t * CH);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) s[nt][t] = mfma(f, q[nt][c], s[nt][t]);
            }
        }
        const int4 said = *reinterpret_cast<const int4 *>(flags[buf]);
        int bits = said.x | said.y << 2;
        if constexpr (PIECES == 4) bits |= said.z << 4 | said.w << 6;
        bits = __builtin_amdgcn_readfirstlane(bits);
        constexpr int kOdd = 0xAA;
        float base[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            f32x4a (&z)[PIECES] = s[nt];
            if (edge || bits != 0) {
#pragma unroll
                for (int j = 0; j < 4 * PIECES; ++j) {
                    const int token = real(t0 + 16 * (j / 4)) + 4 * g + j % 4;
                    const bool seen = (token >= from[nt] || token < a.sinks) && token <= upto[nt] && (bits >> 2 * (j / 4) & 1) == 0;
                    z[j / 4][j % 4] = seen ? z[j / 4][j % 4] : kNone;
                }
            }
            // (the base is 2^kAhead above the maximum where it is set, and stays as long as no score passes it: little is rescaled, and no weight is above 1, which
            // would make infinities of the largest values)
            constexpr float kAhead = 8.0f;
            float most = kNone;
#pragma unroll
            for (int j = 0; j < 4 * PIECES; ++j) most = fmaxf(most, z[j / 4][j % 4]);
            most = row_max(most) * scale_by;
            if (__any(most > top[nt])) {
                const float now = fmaxf(top[nt], most + kAhead), fade = top[nt] == kNone ? 0.0f : __builtin_amdgcn_exp2f(top[nt] - now);
#pragma unroll
                for (int i = 0; i < E; ++i) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[nt][i][r] *= fade;
                }
                top[nt] = now;
                total[nt] *= fade;
            }
            base[nt] = top[nt] == kNone ? 0.0f : top[nt];
        }
        middle();
        // (here and unlikely, for the order that the products' code gets: 8192 rows 588 us and chunks of 64-value heads 134.6, ahead of `middle` 608 and 145)
        if (__builtin_expect((bits & kOdd) != 0, 0)) take_out_odd(buf, s);
#pragma unroll
        for (int t = 0; t < PIECES; t += 2) {
            u32x4 p[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const f32x4a z = s[nt][t + j / 2];
                    const float w0 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[2 * j % 4], scale_by, -base[nt]));
                    const float w1 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[2 * j % 4 + 1], scale_by, -base[nt]));
                    total[nt] += w0 + w1;
                    const unsigned u0 = __float_as_uint(w0), u1 = __float_as_uint(w1);
                    p[nt][0][j] = __builtin_amdgcn_perm(u1, u0, 0x07060302);
                    // (the rest is counted from 2^-24 of the first term below it, so that no term of a weight is zero: an infinite value times 0 is NaN.  Cut off
                    // from just below the weight, as split_terms does: 8192 rows 600 us for 594, chunks of 64-value heads 142 for 136)
                    constexpr float kBelow = 0x1p-24f - 1.0f;
                    p[nt][1][j] = pack_bf16(__builtin_fmaf(__uint_as_float(u0 & 0xFFFF0000u), kBelow, w0), __builtin_fmaf(__uint_as_float(u1 & 0xFFFF0000u), kBelow, w1));
                }
            }
#pragma unroll
            for (int i = 0; i < E; ++i) {
                u32x4 f;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        reinterpret_cast<LdsFour *>((Lds *)(size_t)((v_at + shifted) ^ 32u * i) + 16 * (TN + 16 * (t + k)) * CH));
                    const u32x2 u = __builtin_bit_cast(u32x2, v);
                    f[2 * k] = u.x, f[2 * k + 1] = u.y;
                }
#pragma unroll
                for (int e = 1; e >= 0; --e) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) acc[nt][i] = mfma(f, p[nt][e], acc[nt][i]);
                }
            }
        }
    };

    if (begin < stop) {
        Raw first_k;
        bring(0, begin, first_k);
        if (UNITS > 1) bring(1, begin, next);
        keep(0, 0, begin, edge_of(begin), first_k);
        if (UNITS > 1) keep(1, 0, begin, edge_of(begin), next);
        __syncthreads();
        for (int t0 = begin, buf = 0; t0 < stop; t0 += TN, buf ^= 1) {
            const bool more = t0 + TN < stop, next_edge = edge_of(t0 + TN);
            if (more) bring(0, t0 + TN, next);
            tile(buf, t0, edge_of(t0), [&]() {
                if (UNITS > 1 && more) {
                    keep(0, buf ^ 1, t0 + TN, next_edge, next);
                    bring(1, t0 + TN, next);
                }
            });
            if (more) keep(UNITS - 1, buf ^ 1, t0 + TN, next_edge, next);
            __syncthreads();
        }
    }

#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int x = 16 * (NT * wave + nt) + m;
        const float sum = row_sum(total[nt]), inverse = sum == 0.0f ? 0.0f : 1.0f / sum;
        if (x >= all - x0) continue;
        if (gridDim.z > 1) {
            const int64_t part = prompt_part(a, blockIdx.z) * (16 * NT * W) + x;
            if (g == 0) a.part_ms[part] = make_float2(top[nt], sum);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                if (16 * i >= D) break;
                const float o[4] = {acc[nt][i][0], acc[nt][i][1], acc[nt][i][2], acc[nt][i][3]};
                F32::store4(a.part_o + part * D + 16 * i + 4 * g, o);
            }
            continue;
        }
        const int y = x0_head + x, up = by_group(a, y);
        const int64_t row = first + (int64_t)x0_row + up;
        const int head = h * a.G + y - up * a.G;
        if (g == 0 && a.lse != nullptr) a.lse[row * a.hq + head] = log_sum_exp(top[nt], sum);
        uint16_t *const out = static_cast<uint16_t *>(a.out) + row * a.out_stride + head * D + 4 * g;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if (16 * i >= D) break;
            float o[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] = sum == 0.0f ? 0.0f : acc[nt][i][r] * inverse;
            Bf16::store4(out + 16 * i, o);
        }
    }
}

// The shares of a row joined: each brought to the maximum of all; a share's sum of 0 has nothing of the row.  LV lanes take a row, a workgroup 256 / LV of
// a block's ROWS (a block to a workgroup: 256 rows of 32 heads in eight shares 94 us, 50.5 so).
template <int LV, int ROWS>
__global__ __launch_bounds__(256) void prompt_join_kernel(AttendArgs a) {
    constexpr int PER = 256 / LV, PARTS = ROWS / PER;
    const int grid = a.cache.heads * a.row_blocks, block = blockIdx.x / PARTS, x_block = block % grid, b = block / grid;
    const int h = x_block % a.cache.heads, x = blockIdx.x % PARTS * PER + threadIdx.x / LV, at = (a.row_blocks - 1 - x_block / a.cache.heads) * ROWS + x;
    const int D = a.cache.D, d = 4 * (threadIdx.x % LV);
    int first;
    if (at >= rows_of(a.row_start, b, a.n, a.max_rows, first) * a.G) return;
    auto index = [&](int z) { return (((int64_t)z * a.requests + b) * grid + x_block) * ROWS + x; };
    float top = kNone, total = 0.0f, o[4] = {};
#pragma unroll 8
    for (int z = 0; z < a.places; ++z) {
        const float2 part = a.part_ms[index(z)];
        top = part.y == 0.0f ? top : fmaxf(top, part.x);
    }
#pragma unroll 8
    for (int z = 0; z < a.places; ++z) {
        const float2 part = a.part_ms[index(z)];
        float u[4];
        F32::load4(a.part_o + index(z) * D + (d < D ? d : 0), u);
        const bool nothing = part.y == 0.0f;
        const float f = __builtin_amdgcn_exp2f(part.x - top);
        total += nothing ? 0.0f : part.y * f;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] += nothing ? 0.0f : u[j] * f;
    }
    if (d >= D) return;
    const float inverse = total == 0.0f ? 0.0f : 1.0f / total;
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] *= inverse;
    const int row = first + at / a.G, head = h * a.G + at % a.G;
    Bf16::store4(static_cast<uint16_t *>(a.out) + (int64_t)row * a.out_stride + head * D + d, o);
    if (d == 0 && a.lse != nullptr) a.lse[(int64_t)row * a.hq + head] = log_sum_exp(top, total);
}

template <int DP, int NT>
hipError_t run_prompt(const AttendArgs &a, hipStream_t st) {
    const dim3 grid((unsigned)(a.cache.heads * a.row_blocks), (unsigned)a.requests, (unsigned)a.places);
    if (a.cache.four) prompt_kernel<DP, kHeld4, NT><<<grid, 256, 0, st>>>(a);
    else if (a.cache.k_scale != nullptr) prompt_kernel<DP, kHeld8, NT><<<grid, 256, 0, st>>>(a);
    else prompt_kernel<DP, kHeld16, NT><<<grid, 256, 0, st>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.places == 1) return e;
    prompt_join_kernel<DP / 4, 64 * NT><<<grid.x * grid.y * (64 * NT / (1024 / DP)), 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace vt
