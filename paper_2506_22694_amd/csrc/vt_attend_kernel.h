// Attention of a draft step's rows over a paged key-value cache, on the matrix cores (v_mfma_f32_16x16x32_bf16).
//
// Bound by the one pass over the cached keys and values: a kv head's query rows (the heads that share it, times the request's new
// tokens) are one side of the products, and up to 64 of them cost the matrix cores a fraction of the time that the cache takes to
// arrive.  So what matters is that loads never stop, and a wave goes its own way: it takes 32 tokens at a time, straight from the cache
// into registers in the matrix instructions' operand layout, without LDS and without a barrier until its piece of the request is done.
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
// fp32 rows: a value of 24 bits is the sum of three of 8, so q and p are three operands each, and products are exact as for bf16.
#pragma once
#include <type_traits>

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
// What is left of a value after its leading 8 bits
__device__ __forceinline__ float less_bf16(float x, float &leading) {
    leading = (float)(__bf16)x;
    return x - leading;
}

constexpr float kNone = -__builtin_inff();

// Four values of a row from their sums over all tokens, relative to the row's maximum (log 2), and its log-sum-exp.
__device__ __forceinline__ void finish_row(const AttendArgs &a, int64_t row, int head, int d, const float *sums, float top, float total, bool f32) {
    float o[4];
    const float inverse = total == 0.0f ? 0.0f : 1.0f / total;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = sums[i] * inverse;
    const int64_t to = row * a.out_stride + (int64_t)head * a.cache.D + d;
    if (f32) F32::store4(static_cast<float *>(a.out) + to, o);
    else Bf16::store4(static_cast<uint16_t *>(a.out) + to, o);
    if (d == 0 && a.lse != nullptr) a.lse[row * a.hq + head] = total == 0.0f ? kNone : (top + __builtin_amdgcn_logf(total)) * 0.69314718055994531f;
}

template <int DP, bool FP8, int NT, bool F32Q>
__global__ __launch_bounds__(64 * kAttendWaves) void attend_kernel(AttendArgs a) {
    constexpr int W = kAttendWaves, E = DP / 16, KS = DP / 32, TERMS = F32Q ? 3 : 1;
    constexpr int KL = FP8 ? DP / 64 : DP / 32;       // 16-byte loads of a token's row of K in a lane
    constexpr int VR = FP8 ? DP / 64 : DP / 32;       // registers of a token's E values of V
    constexpr int SZ = FP8 ? 1 : 2;
    constexpr int PITCH = DP + 4;
    __shared__ float ms[2][W][16 * NT];
    __shared__ __align__(16) float sums[W][16][PITCH];

    const int lane = lane_id(), m = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int unit = blockIdx.x, split = blockIdx.y;
    const int rb = unit % a.row_blocks, h = (unit / a.row_blocks) % a.cache.heads, b = unit / a.row_blocks / a.cache.heads;

    int64_t first;
    const int nrows = rows_of(a.row_start, b, a.n, a.max_rows, first);
    const int RG = nrows * a.G, x0 = rb * 16 * NT;
    const int len = tokens_of(a.lengths[b], a.most);
    const int piece = piece_tokens(len, a.splits, kAttendLeast), pieces = pieces_of(len, piece);
    if (x0 >= RG || split >= pieces) return;
    const int t0 = split * piece, t1 = min(len, t0 + piece);
    const int D = a.cache.D;

    // q's operand: row x = x0 + 16 nt + m is new token x / G, head h G + x % G; the values of d that the lane's K has
    u32x4 q[NT][TERMS][KS];
    uint64_t tail[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int x = x0 + 16 * nt + m;
        const int64_t row = first + min(x, RG - 1) / a.G;
        const int64_t at = row * a.q_stride + (int64_t)(h * a.G + min(x, RG - 1) % a.G) * D;
        tail[nt] = a.tail_mask != nullptr ? a.tail_mask[row] : 0;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int d = FP8 ? 64 * (s / 2) + 16 * g + 8 * (s % 2) : 32 * s + 8 * g;
            const bool there = x < RG && d < D;
            if constexpr (!F32Q) {
                q[nt][0][s] = there ? *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(a.q) + at + d) : u32x4{0, 0, 0, 0};
            } else {
                float v[8] = {}, lead[8];
                if (there) {
                    F32::load4(static_cast<const float *>(a.q) + at + d, v);
                    F32::load4(static_cast<const float *>(a.q) + at + d + 4, v + 4);
                }
#pragma unroll
                for (int i = 0; i < TERMS; ++i) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = less_bf16(v[j], lead[j]);
                    q[nt][i][s] = u32x4{pack_bf16(lead[0], lead[1]), pack_bf16(lead[2], lead[3]), pack_bf16(lead[4], lead[5]),
                                        pack_bf16(lead[6], lead[7])};
                }
            }
        }
    }

    // Page numbers of 64 pages, one in each lane
    const int32_t *pages = a.page_table + (int64_t)b * a.table_pages;
    const int shift = a.cache.page_shift, last_page = (len - 1) >> shift;
    int window = 0, ids = 0;
    bool none_read = true;
    // First row of 16 tokens (of one page: pages are multiples of 16) in the cache; row 0 where there is nothing to read.
    auto rows16 = [&](int token, bool &there) -> int64_t {
        int64_t row = -1;
        if (token < t1) {
            const int p = token >> shift;
            if (none_read || p >= window + 64) {
                window = p;
                none_read = false;
                ids = pages[min(p + lane, last_page)];
            }
            row = row_of_page(__builtin_amdgcn_readlane(ids, p - window), a.cache.pages, a.cache.heads, h, shift);
        }
        there = row >= 0;
        return there ? row + (token & ((1 << shift) - 1)) : 0;
    };

    // Offsets of a lane's loads from the first row; past the end of rows shorter than DP: the row's first values again (K: dropped below,
    // V: in sums that nobody asks for).
    int k_at[KL];
#pragma unroll
    for (int s = 0; s < KL; ++s) {
        const int d = FP8 ? 64 * s + 16 * g : 32 * s + 8 * g;
        k_at[s] = (m * D + (d < D ? d : 0)) * SZ;
    }
    const int v_at = (4 * g * D + (E * m < D ? E * m : 0)) * SZ;

    u32x4 k[2][KL];
    unsigned v[8][VR], k_scale[2] = {}, v_scale[2] = {};
    auto load_k = [&](const int64_t (&row)[2]) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const char *p = static_cast<const char *>(a.cache.k) + row[t] * D * SZ;
#pragma unroll
            for (int s = 0; s < KL; ++s) k[t][s] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p + k_at[s]));
            if constexpr (FP8) k_scale[t] = *reinterpret_cast<const unsigned *>(a.cache.k_scale + row[t] + 4 * g);
        }
    };
    auto load_v = [&](const int64_t (&row)[2]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const char *p = static_cast<const char *>(a.cache.v) + (row[j / 4] + j % 4) * D * SZ + v_at;
            if constexpr (VR == 1) {
                v[j][0] = __builtin_nontemporal_load(reinterpret_cast<const unsigned *>(p));
            } else if constexpr (VR == 2) {
                const u32x2 u = __builtin_nontemporal_load(reinterpret_cast<const u32x2 *>(p));
                v[j][0] = u.x, v[j][1] = u.y;
            } else {
#pragma unroll
                for (int i = 0; i < VR / 4; ++i) {
                    const u32x4 u = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p) + i);
                    v[j][4 * i] = u.x, v[j][4 * i + 1] = u.y, v[j][4 * i + 2] = u.z, v[j][4 * i + 3] = u.w;
                }
            }
        }
        if constexpr (FP8) {
#pragma unroll
            for (int t = 0; t < 2; ++t) v_scale[t] = *reinterpret_cast<const unsigned *>(a.cache.v_scale + row[t] + 4 * g);
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

    // acc += V^T p^T.  HARD: some row does not see a token that holds NaN or infinities, and 0 * inf must not reach it.  Those values are
    // left out of the product, and counted in products of ones: where a row sees one, its sum is what it would have been.
    unsigned p[NT][TERMS][4], sees[NT][4];
    auto add_values = [&](auto hard) {
        constexpr bool HARD = decltype(hard)::value;
        auto one = [&](int i, u32x4 f) {
            if constexpr (!HARD) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                    for (int e = TERMS - 1; e >= 0; --e) acc[nt][i] = mfma(f, u32x4{p[nt][e][0], p[nt][e][1], p[nt][e][2], p[nt][e][3]}, acc[nt][i]);
                }
            } else {
                u32x4 finite = f, nan, plus, minus;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    unsigned out[4] = {0, 0, 0, 0};
#pragma unroll
                    for (int s = 0; s < 32; s += 16) {
                        const unsigned u = (f[r] >> s) & 0xFFFFu;
                        const bool odd = (u & 0x7F80u) == 0x7F80u, is_nan = (u & 0x7FFFu) > 0x7F80u;
                        out[0] |= (odd ? 0u : u) << s;
                        out[1] |= (is_nan ? 0x3F80u : 0u) << s;
                        out[2] |= (u == 0x7F80u ? 0x3F80u : 0u) << s;
                        out[3] |= (u == 0xFF80u ? 0x3F80u : 0u) << s;
                    }
                    finite[r] = out[0], nan[r] = out[1], plus[r] = out[2], minus[r] = out[3];
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const u32x4 seen = {sees[nt][0], sees[nt][1], sees[nt][2], sees[nt][3]};
                    const f32x4a z = {0, 0, 0, 0};
                    const f32x4a n0 = mfma(nan, seen, z), n1 = mfma(plus, seen, z), n2 = mfma(minus, seen, z);
#pragma unroll
                    for (int e = TERMS - 1; e >= 0; --e) acc[nt][i] = mfma(finite, u32x4{p[nt][e][0], p[nt][e][1], p[nt][e][2], p[nt][e][3]}, acc[nt][i]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        if (n0[r] > 0) acc[nt][i][r] = __builtin_nanf("");
                        if (n1[r] > 0) acc[nt][i][r] += __builtin_inff();
                        if (n2[r] > 0) acc[nt][i][r] -= __builtin_inff();
                    }
                }
            }
        };
#pragma unroll
        for (int r = 0; r < VR; ++r) {
            if constexpr (!FP8) {
                u32x4 lo, hi;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    lo[j] = __builtin_amdgcn_perm(v[2 * j + 1][r], v[2 * j][r], 0x05040100);
                    hi[j] = __builtin_amdgcn_perm(v[2 * j + 1][r], v[2 * j][r], 0x07060302);
                }
                one(2 * r, lo);
                one(2 * r + 1, hi);
            } else {
                u32x4 f[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    // bytes: first token's value, second token's value, the next value of both
                    const unsigned lo = __builtin_amdgcn_perm(v[2 * j + 1][r], v[2 * j][r], 0x05010400);
                    const unsigned hi = __builtin_amdgcn_perm(v[2 * j + 1][r], v[2 * j][r], 0x07030602);
                    f[0][j] = two_codes<false>(lo), f[1][j] = two_codes<true>(lo);
                    f[2][j] = two_codes<false>(hi), f[3][j] = two_codes<true>(hi);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) one(4 * r + i, f[i]);
            }
        }
    };

    int token = t0 + kAttendTile * wave;
    if (token < t1) {
        bool there[2];
        int64_t row[2];
        row[0] = rows16(token, there[0]);
        row[1] = rows16(token + 16, there[1]);
        load_k(row);
        load_v(row);
        for (;;) {
            // scores: lane has tokens 16 t + 4 g + i of row m
            f32x4a s[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = f32x4a{0, 0, 0, 0};
#pragma unroll
            for (int t = 0; t < 2; ++t) {
#pragma unroll
                for (int c = 0; c < KS; ++c) {
                    u32x4 f;
                    if constexpr (FP8) {
                        const unsigned u0 = k[t][c / 2][2 * (c % 2)], u1 = k[t][c / 2][2 * (c % 2) + 1];
                        f = u32x4{two_codes<false>(u0), two_codes<true>(u0), two_codes<false>(u1), two_codes<true>(u1)};
                    } else {
                        f = k[t][c];
                    }
                    if (D != DP && (FP8 ? 64 * (c / 2) + 16 * g : 32 * c + 8 * g) >= D) f = u32x4{0, 0, 0, 0};
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                        for (int e = TERMS - 1; e >= 0; --e) s[nt][t] = mfma(f, q[nt][e][c], s[nt][t]);
                    }
                }
            }
            float factor[2][4];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    factor[t][i] = FP8 ? scale_of((k_scale[t] >> 8 * i) & 0xFF) * a.scale_log2 : a.scale_log2;
            }

            // the next tile's keys are asked for once this one's are used up, its values likewise below
            const int next = token + kAttendTile * W;
            bool next_there[2];
            int64_t next_row[2];
            next_row[0] = rows16(next, next_there[0]);
            next_row[1] = rows16(next + 16, next_there[1]);
            load_k(next_row);

            const bool ends = token + kAttendTile > t1 || !there[0] || !there[1];
            const bool masked = a.tail_mask != nullptr && token + kAttendTile > len - 64;
            if constexpr (FP8) {
                if (ends) {      // (a scale of what lies past the end may be infinite, and p = 0 there)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const bool seen = token + 16 * (j / 4) + 4 * g + j % 4 < t1 && there[j / 4];
                        v_scale[j / 4] &= seen ? ~0u : ~(0xFFu << 8 * (j % 4));
                    }
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
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int at = token + 16 * t + 4 * g + i, bit = at - (len - 64);
                            bool seen = at < t1 && there[t];
                            if (masked && bit >= 0) seen = seen && ((tail[nt] >> (bit & 63)) & 1) != 0;
                            if (!seen) z[t][i] = kNone;
                        }
                    }
                }
                float most = top[nt];
#pragma unroll
                for (int t = 0; t < 2; ++t) most = fmaxf(most, fmaxf(fmaxf(z[t][0], z[t][1]), fmaxf(z[t][2], z[t][3])));
                most = row_max(most);
                // (a row that has seen nothing yet: exp2(-inf - 0) = 0)
                const float base = most == kNone ? 0.0f : most;
                const float fade = __builtin_amdgcn_exp2f(top[nt] - base);
                if (__any(most > top[nt])) {
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
                    for (int j = 0; j < 8; ++j) w[j] *= scale_of((v_scale[j / 4] >> 8 * (j % 4)) & 0xFF);
                }
#pragma unroll
                for (int e = 0; e < TERMS; ++e) {
                    float lead[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if constexpr (TERMS > 1) w[j] = less_bf16(w[j], lead[j]);
                        else lead[j] = w[j];
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) p[nt][e][j] = pack_bf16(lead[2 * j], lead[2 * j + 1]);
                }
            }
            if (ends) {
                // what lies past the end may be anything, NaN too
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool seen = token + 16 * (j / 4) + 4 * g + j % 4 < t1 && there[j / 4];
#pragma unroll
                    for (int r = 0; r < VR; ++r) v[j][r] = seen ? v[j][r] : 0u;
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
            if (hard) add_values(std::integral_constant<bool, true>{});
            else add_values(std::integral_constant<bool, false>{});
            if (next >= t1) break;
            load_v(next_row);
            token = next;
            there[0] = next_there[0], there[1] = next_there[1];
        }
    }

    // The waves' sums joined: each brings its rows to the common maximum.  A sum of 0 is a wave without tokens for the row (one of -inf
    // scores, too): it adds nothing.  (NaN has a sum, of NaN, and no maximum.)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        total[nt] = row_sum(total[nt]);
        if (g == 0) ms[0][wave][16 * nt + m] = top[nt], ms[1][wave][16 * nt + m] = total[nt];
    }
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        float most = kNone;
#pragma unroll
        for (int w = 0; w < W; ++w) most = fmaxf(most, ms[0][w][16 * nt + m]);
        const float fade = __builtin_amdgcn_exp2f(top[nt] - most);
        if (nt != 0) __syncthreads();
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float *to = &sums[wave][m][4 * E * g + E * r];
#pragma unroll
            for (int i = 0; i < E; ++i) to[i] = total[nt] == 0.0f ? 0.0f : acc[nt][i][r] * fade;
        }
        __syncthreads();
        for (int c = threadIdx.x; c < 4 * DP; c += 64 * W) {
            const int xr = c / (DP / 4), d = 4 * (c % (DP / 4)), x = x0 + 16 * nt + xr;
            if (x >= RG || d >= D) continue;
            float top_row = kNone, sum_row = 0.0f;
#pragma unroll
            for (int w = 0; w < W; ++w) top_row = fmaxf(top_row, ms[0][w][16 * nt + xr]);
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float part = ms[1][w][16 * nt + xr];
                sum_row += part == 0.0f ? 0.0f : part * __builtin_amdgcn_exp2f(ms[0][w][16 * nt + xr] - top_row);
            }
            float o[4] = {};
#pragma unroll
            for (int w = 0; w < W; ++w) {
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] += sums[w][xr][d + i];
            }
            const int64_t row = first + x / a.G;
            const int head = h * a.G + x % a.G;
            const int64_t at = row * a.hq + head;
            if (pieces > 1) {
                F32::store4(a.part_o + (at * a.splits + split) * D + d, o);
                if (d == 0) a.part_ms[at * a.splits + split] = make_float2(top_row, sum_row);
                continue;
            }
            finish_row(a, row, head, d, o, top_row, sum_row, F32Q);
        }
    }
}

template <int DP, bool FP8, int NT, bool F32Q>
hipError_t run_attend(const AttendArgs &a, hipStream_t st) {
    const dim3 grid((unsigned)(a.requests * a.cache.heads * a.row_blocks), (unsigned)a.splits);
    attend_kernel<DP, FP8, NT, F32Q><<<grid, 64 * kAttendWaves, 0, st>>>(a);
    return hipGetLastError();
}
template <int DP, int NT, bool F32Q>
hipError_t run_attend(const AttendArgs &a, hipStream_t st) {
    return a.cache.k_scale != nullptr ? run_attend<DP, true, NT, F32Q>(a, st) : run_attend<DP, false, NT, F32Q>(a, st);
}

}  // namespace vt
