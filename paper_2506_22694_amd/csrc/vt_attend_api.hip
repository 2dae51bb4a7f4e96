// C ABI of include/vocabtrim_attention.h: argument checks, how the work is cut up, kernel dispatch.  Every entry point only enqueues
// work on the caller's stream.
#include "vocabtrim_attention.h"

#include <cmath>

#include "vt_attn.h"

namespace {

constexpr int64_t kMaxRows = (int64_t)1 << 31, kMaxLength = (int64_t)1 << 30;
// Workgroups and threads of a launch are 32-bit numbers.
constexpr int64_t kMaxGrid = (int64_t)1 << 23;

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline bool element(int type) { return type == VT_F32 || type == VT_BF16; }
inline bool index_type(int type) { return type == VT_I32 || type == VT_I64; }
inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

inline vt::IndexArgs indexes(const void *p, int type) { return {p, type == VT_I64}; }
inline bool index_aligned(const void *p, int type) { return aligned(p, type == VT_I64 ? 8 : 4); }

// A tensor of heads that is there: VT_OK, or what is wrong with it.
int heads_status(const void *p, int64_t stride, int heads, int D) {
    if (p == nullptr) return VT_ERR_NULL;
    if (stride < (int64_t)heads * D) return VT_ERR_SHAPE;
    return aligned(p, 16) && stride % 8 == 0 ? VT_OK : VT_ERR_ALIGN;
}

int norm_status(int type, int64_t n, int q_heads, int k_heads, int D, const void *q_weight, const void *k_weight, float eps, const float *table,
                int64_t table_rows, int rot, int style, const void *positions, int pos_type) {
    if (!element(type) || (table != nullptr && !index_type(pos_type))) return VT_ERR_DTYPE;
    if (n < 0 || n >= kMaxRows || q_heads < 0 || k_heads < 0 || q_heads + (int64_t)k_heads < 1 || q_heads + (int64_t)k_heads > VT_MAX_ATTENTION_HEADS ||
        D < 8 || D > VT_MAX_HEAD_DIM)
        return VT_ERR_SHAPE;
    if ((q_weight == nullptr) != (k_weight == nullptr)) return VT_ERR_NULL;
    if (q_weight != nullptr && !(eps > 0.0f && std::isfinite(eps))) return VT_ERR_SHAPE;
    if (table != nullptr) {
        if (rot < 8 || rot > D || table_rows < 1 || (style != VT_ROPE_HALVES && style != VT_ROPE_NEIGHBOURS)) return VT_ERR_SHAPE;
        if (n > 0 && positions == nullptr) return VT_ERR_NULL;
        if (rot % 8 != 0 || !aligned(table, 16) || !index_aligned(positions, pos_type)) return VT_ERR_ALIGN;
    }
    return D % 8 == 0 && aligned(q_weight, 16) && aligned(k_weight, 16) ? VT_OK : VT_ERR_ALIGN;
}

int cache_status(const vt_kv_cache *c) {
    if (c == nullptr) return VT_ERR_NULL;
    if (c->type != VT_BF16 && c->type != VT_E4M3) return VT_ERR_DTYPE;
    if (c->pages < 1 || c->pages > kMaxRows || c->heads < 1 || c->heads > VT_MAX_ATTENTION_HEADS || c->head_dim < 16 || c->head_dim > VT_MAX_HEAD_DIM ||
        c->page_size < 16 || c->page_size > 65536 || (c->page_size & (c->page_size - 1)) != 0)
        return VT_ERR_SHAPE;
    if (c->k == nullptr || c->v == nullptr) return VT_ERR_NULL;
    if (c->type == VT_E4M3 && (c->k_scale == nullptr || c->v_scale == nullptr)) return VT_ERR_NULL;
    if (c->head_dim % 16 != 0 || !aligned(c->k, 16) || !aligned(c->v, 16)) return VT_ERR_ALIGN;
    return c->type != VT_E4M3 || (aligned(c->k_scale, 4) && aligned(c->v_scale, 4)) ? VT_OK : VT_ERR_ALIGN;
}
vt::CacheArgs cache_args(const vt_kv_cache &c) {
    const bool coded = c.type == VT_E4M3;
    return {c.k, c.v, coded ? c.k_scale : nullptr, coded ? c.v_scale : nullptr, c.pages, c.heads, __builtin_ctz((unsigned)c.page_size), c.head_dim};
}

// How attention is cut up: blocks of a kv head's query rows, and shares of all requests' tokens.
struct Split {
    bool ok = false, whole = true;
    int row_blocks = 1, row_tiles = 1, places = 1;
    size_t entries = 0, bytes = 0, most_bytes = 0;       // rows of partial results; bytes of this call; of any call of up to these sizes
};

// Shares that all requests' tokens are cut into: two workgroups' on each of the 256 CUs, all there at a time, the one reading while the other
// begins or ends a request (48 ragged requests in 8 bits 104 us, with one on each CU 107, with four 106).  One request has one beginning,
// and the workgroups of a CU take each other's time: 16384 tokens 17.2 us with one on each CU, 18.5 with two; 131001 tokens 88.0 and 88.8.
// (Levels of a few short requests have no more steps than places: there it is one step to a workgroup and one tile to a wave, whose loads have
// nothing to hide behind.  Longer shares were not measured on them.)
constexpr int64_t kAttendWorkgroups = 512, kAttendWorkgroupsOfOne = 256;
// Up to here a workgroup takes a request whole, without the second launch: 300 tokens of one request 6.6 us whole, 7.9 in shares, 512 tokens
// 8.9 and 8.0.  Where there are many requests the workgroups are enough: of two requests' worth of tokens for each workgroup and no more
// than kAttendWholeOfMany (8-bit cache, 64 requests of up to 1000 tokens, 512 workgroups: 19.5 us whole, 26.0 in shares; 16 requests, 128
// workgroups: 13.2 and 11.2; 64 requests of up to 4000: 60.5 and 46.0).
constexpr int64_t kAttendWhole = 384, kAttendWholeOfMany = 1536;

Split split_of(int64_t n, int q_heads, int kv_heads, int D, int requests, int max_rows, int64_t max_length, bool f32) {
    Split s;
    if (n < 0 || n >= kMaxRows || q_heads < 1 || q_heads > VT_MAX_ATTENTION_HEADS || kv_heads < 1 || q_heads % kv_heads != 0 || D < 16 || D > VT_MAX_HEAD_DIM ||
        requests < 0 || requests > VT_MAX_REQUESTS || max_rows < 1 || n > (int64_t)requests * max_rows || max_length < 0 || max_length > kMaxLength)
        return s;
    const int64_t rows = (int64_t)max_rows * (q_heads / kv_heads);
    const int64_t steps = (max_length + vt::kAttendStep - 1) / vt::kAttendStep;
    // (workgroups and threads of a launch, and all requests' steps, are 32-bit numbers)
    if (rows > kMaxGrid || (int64_t)requests * max_rows * q_heads > kMaxGrid || (steps + 1) * requests > kMaxLength) return s;
    s.row_tiles = vt::attend_row_tiles((int)rows, D, f32);
    const int64_t per = 16 * s.row_tiles, blocks = (rows + per - 1) / per, units = kv_heads * blocks;
    const int64_t few = 2 * units * requests < kAttendWholeOfMany ? 2 * units * requests : kAttendWholeOfMany;
    s.whole = max_length <= (few > kAttendWhole ? few : kAttendWhole);
    int64_t places = requests;
    if (!s.whole) {
        places = ((requests == 1 ? kAttendWorkgroupsOfOne : kAttendWorkgroups) + units - 1) / units;
        if (places > steps * requests) places = steps * requests;
    }
    if (places * units > kMaxGrid || places > 65535) return s;
    s.ok = true;
    s.row_blocks = (int)blocks;
    s.places = (int)places;
    const size_t entry = (D + 2) * sizeof(float);
    // Any call of up to these sizes: units * places are below workgroups + units, units * per below kv_heads * (rows + per), and per is no
    // larger with fewer rows.  (Fewer requests of the same lengths may be taken in shares where these are taken whole.)
    const size_t most = 2 * (size_t)(kAttendWorkgroups * per + kv_heads * (rows + per));
    s.most_bytes = max_length <= kAttendWhole ? 0 : round_up(most * entry + requests * sizeof(int4), 256);
    if (s.whole) return s;
    s.entries = (size_t)units * places * 2 * per;
    s.bytes = s.entries * entry + requests * sizeof(int4);
    return s;
}

}  // namespace

extern "C" {

int vt_qk_norm_rope(const void *q, int64_t q_stride, const void *k, int64_t k_stride, int type, int64_t n, int32_t q_heads, int32_t k_heads,
                    int32_t head_dim, const void *q_weight, const void *k_weight, float eps, const float *table, int64_t table_rows,
                    int32_t rotary_dim, int style, const void *positions, int pos_type, void *q_out, int64_t q_out_stride, void *k_out,
                    int64_t k_out_stride, void *stream) {
    int s = norm_status(type, n, q_heads, k_heads, head_dim, q_weight, k_weight, eps, table, table_rows, rotary_dim, style, positions, pos_type);
    if (s != VT_OK) return s;
    if (n == 0) return VT_OK;
    if (q_heads > 0) {
        if ((s = heads_status(q, q_stride, q_heads, head_dim)) != VT_OK) return s;
        if ((s = heads_status(q_out, q_out_stride, q_heads, head_dim)) != VT_OK) return s;
    }
    if (k_heads > 0) {
        if ((s = heads_status(k, k_stride, k_heads, head_dim)) != VT_OK) return s;
        if ((s = heads_status(k_out, k_out_stride, k_heads, head_dim)) != VT_OK) return s;
    }
    vt::NormArgs a{};
    a.q = q, a.k = k, a.q_stride = q_stride, a.k_stride = k_stride;
    a.n = n, a.hq = q_heads, a.hk = k_heads, a.D = head_dim, a.rot = rotary_dim, a.neighbours = style == VT_ROPE_NEIGHBOURS;
    a.wq = q_weight, a.wk = k_weight, a.eps = eps;
    a.table = table, a.table_rows = table_rows, a.positions = indexes(positions, pos_type);
    a.q_out = q_out, a.k_out = k_out, a.q_out_stride = q_out_stride, a.k_out_stride = k_out_stride;
    return vt::status_of_hip(vt::launch_norm_rope(a, type == VT_BF16, static_cast<hipStream_t>(stream)));
}

size_t vt_qk_norm_rope_backward_ws_bytes(int64_t n, int32_t head_dim) {
    if (n < 0 || n >= kMaxRows || head_dim < 8 || head_dim > VT_MAX_HEAD_DIM) return 0;
    return round_up((size_t)vt::norm_backward_workgroups(n) * 2 * head_dim * sizeof(float), 256);
}

int vt_qk_norm_rope_backward(const void *gq, int64_t gq_stride, const void *gk, int64_t gk_stride, const void *q, int64_t q_stride, const void *k,
                             int64_t k_stride, int type, int64_t n, int32_t q_heads, int32_t k_heads, int32_t head_dim, const void *q_weight,
                             const void *k_weight, float eps, const float *table, int64_t table_rows, int32_t rotary_dim, int style,
                             const void *positions, int pos_type, void *dq, int64_t dq_stride, void *dk, int64_t dk_stride, float *dqw,
                             float *dkw, void *ws, size_t ws_bytes, void *stream) {
    int s = norm_status(type, n, q_heads, k_heads, head_dim, q_weight, k_weight, eps, table, table_rows, rotary_dim, style, positions, pos_type);
    if (s != VT_OK) return s;
    const bool norm = q_weight != nullptr;
    if (n > 0 && q_heads > 0) {
        if ((s = heads_status(gq, gq_stride, q_heads, head_dim)) != VT_OK) return s;
        if (norm && (s = heads_status(q, q_stride, q_heads, head_dim)) != VT_OK) return s;
        if ((s = heads_status(dq, dq_stride, q_heads, head_dim)) != VT_OK) return s;
    }
    if (n > 0 && k_heads > 0) {
        if ((s = heads_status(gk, gk_stride, k_heads, head_dim)) != VT_OK) return s;
        if (norm && (s = heads_status(k, k_stride, k_heads, head_dim)) != VT_OK) return s;
        if ((s = heads_status(dk, dk_stride, k_heads, head_dim)) != VT_OK) return s;
    }
    if (norm) {
        if (dqw == nullptr || dkw == nullptr) return VT_ERR_NULL;
        if (!aligned(dqw, 4) || !aligned(dkw, 4)) return VT_ERR_ALIGN;
        if (ws == nullptr || !aligned(ws, 256) || ws_bytes < vt_qk_norm_rope_backward_ws_bytes(n, head_dim)) return VT_ERR_WORKSPACE;
    } else if (n == 0) {
        return VT_OK;
    }
    vt::NormArgs a{};
    a.gq = gq, a.gk = gk, a.gq_stride = gq_stride, a.gk_stride = gk_stride;
    a.q = q, a.k = k, a.q_stride = q_stride, a.k_stride = k_stride;
    a.n = n, a.hq = q_heads, a.hk = k_heads, a.D = head_dim, a.rot = rotary_dim, a.neighbours = style == VT_ROPE_NEIGHBOURS;
    a.wq = q_weight, a.wk = k_weight, a.eps = eps;
    a.table = table, a.table_rows = table_rows, a.positions = indexes(positions, pos_type);
    a.q_out = dq, a.k_out = dk, a.q_out_stride = dq_stride, a.k_out_stride = dk_stride;
    a.partial = static_cast<float *>(ws), a.dqw = dqw, a.dkw = dkw;
    return vt::status_of_hip(vt::launch_norm_rope_backward(a, type == VT_BF16, static_cast<hipStream_t>(stream)));
}

int vt_qkv_to_cache(const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride, int type, int64_t n,
                    int32_t q_heads, const void *q_weight, const void *k_weight, float eps, const float *table, int64_t table_rows,
                    int32_t rotary_dim, int style, const void *positions, int pos_type, void *q_out, int64_t q_out_stride,
                    const vt_kv_cache *cache, const void *slots, int slot_type, void *stream) {
    int s = cache_status(cache);
    if (s != VT_OK) return s;
    const int heads = cache->heads, D = cache->head_dim;
    if (!index_type(slot_type)) return VT_ERR_DTYPE;
    if ((s = norm_status(type, n, q_heads, heads, D, q_weight, k_weight, eps, table, table_rows, rotary_dim, style, positions, pos_type)) != VT_OK) return s;
    if (n == 0) return VT_OK;
    if (slots == nullptr) return VT_ERR_NULL;
    if (!index_aligned(slots, slot_type)) return VT_ERR_ALIGN;
    if (q_heads > 0) {
        if ((s = heads_status(q, q_stride, q_heads, D)) != VT_OK) return s;
        if ((s = heads_status(q_out, q_out_stride, q_heads, D)) != VT_OK) return s;
    }
    if ((s = heads_status(k, k_stride, heads, D)) != VT_OK) return s;
    if ((s = heads_status(v, v_stride, heads, D)) != VT_OK) return s;
    vt::NormArgs a{};
    a.q = q, a.k = k, a.v = v, a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride;
    a.n = n, a.hq = q_heads, a.hk = heads, a.D = D, a.rot = rotary_dim, a.neighbours = style == VT_ROPE_NEIGHBOURS;
    a.wq = q_weight, a.wk = k_weight, a.eps = eps;
    a.table = table, a.table_rows = table_rows, a.positions = indexes(positions, pos_type);
    a.q_out = q_out, a.q_out_stride = q_out_stride;
    a.to_cache = 1, a.cache = cache_args(*cache), a.slots = indexes(slots, slot_type);
    return vt::status_of_hip(vt::launch_norm_rope(a, type == VT_BF16, static_cast<hipStream_t>(stream)));
}

int vt_kv_cache_read(const vt_kv_cache *cache, const void *slots, int slot_type, int64_t n, void *k_out, void *v_out, int out_type, void *stream) {
    const int s = cache_status(cache);
    if (s != VT_OK) return s;
    if (!element(out_type) || !index_type(slot_type)) return VT_ERR_DTYPE;
    if (n < 0 || n >= kMaxRows) return VT_ERR_SHAPE;
    if (n == 0) return VT_OK;
    if (slots == nullptr || k_out == nullptr || v_out == nullptr) return VT_ERR_NULL;
    if (!index_aligned(slots, slot_type) || !aligned(k_out, 16) || !aligned(v_out, 16)) return VT_ERR_ALIGN;
    vt::CacheReadArgs a{cache_args(*cache), indexes(slots, slot_type), n, k_out, v_out};
    return vt::status_of_hip(vt::launch_cache_read(a, out_type == VT_BF16, static_cast<hipStream_t>(stream)));
}

size_t vt_paged_attention_ws_bytes(int64_t n, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int32_t n_requests, int32_t max_rows,
                                   int64_t max_length) {
    return split_of(n, q_heads, kv_heads, head_dim, n_requests, max_rows, max_length, false).most_bytes;
}

int vt_paged_attention(const void *q, int64_t q_stride, int type, int64_t n, int32_t q_heads, const vt_kv_cache *cache, const int32_t *page_table,
                       int32_t table_pages, const int32_t *lengths, int32_t n_requests, const int32_t *row_start, int32_t max_rows,
                       const uint64_t *tail_mask, int64_t max_length, float scale, void *out, int64_t out_stride, float *out_lse, void *ws,
                       size_t ws_bytes, void *stream) {
    int s = cache_status(cache);
    if (s != VT_OK) return s;
    if (!element(type)) return VT_ERR_DTYPE;
    const bool f32 = type == VT_F32;
    const Split split = split_of(n, q_heads, cache->heads, cache->head_dim, n_requests, max_rows, max_length, f32);
    if (!split.ok || table_pages < 1 || !std::isfinite(scale)) return VT_ERR_SHAPE;
    if (row_start == nullptr && (n != n_requests || max_rows != 1)) return VT_ERR_SHAPE;
    if (n == 0 || n_requests == 0) return VT_OK;
    if (page_table == nullptr || lengths == nullptr) return VT_ERR_NULL;
    if ((s = heads_status(q, q_stride, q_heads, cache->head_dim)) != VT_OK) return s;
    if ((s = heads_status(out, out_stride, q_heads, cache->head_dim)) != VT_OK) return s;
    if (!aligned(page_table, 4) || !aligned(lengths, 4) || !aligned(row_start, 4) || !aligned(tail_mask, 8)) return VT_ERR_ALIGN;
    if (split.bytes > 0 && (ws == nullptr || !aligned(ws, 256) || ws_bytes < split.bytes)) return VT_ERR_WORKSPACE;
    if (!aligned(out_lse, 4)) return VT_ERR_ALIGN;
    vt::AttendArgs a{};
    a.q = q, a.q_stride = q_stride, a.n = (int)n, a.hq = q_heads, a.G = q_heads / cache->heads;
    a.cache = cache_args(*cache);
    a.page_table = page_table, a.table_pages = table_pages, a.lengths = lengths, a.requests = n_requests;
    a.row_start = row_start, a.max_rows = max_rows, a.tail_mask = tail_mask;
    const int64_t held = (int64_t)table_pages * cache->page_size;
    a.most = (int)(max_length < held ? max_length : held);
    a.scale_log2 = scale * 1.4426950408889634f;
    a.out = out, a.out_stride = out_stride, a.lse = out_lse;
    a.whole = split.whole, a.places = split.places, a.row_blocks = split.row_blocks, a.row_tiles = split.row_tiles;
    a.G_magic = (unsigned)(((uint64_t)1 << 32) / a.G) + 1u;
    a.by_place = n_requests > split.places;
    a.part_o = static_cast<float *>(ws);
    a.part_ms = reinterpret_cast<float2 *>(a.part_o + split.entries * cache->head_dim);
    a.part_at = reinterpret_cast<int4 *>(a.part_ms + split.entries);
    return vt::status_of_hip(vt::launch_attend(a, f32, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
