// Internal interface of the attention kernels: norm and rotation with its gradients, the paged cache, attention over it.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace vt {

struct CacheArgs {
    void *k, *v;
    uint8_t *k_scale, *v_scale;      // null: held in bf16
    int64_t pages;
    int heads, page_shift, D;
    int four;                        // codes of 4 bits, two to a byte; scales of 32 values (else of a row)
};

// One row of positions or slots, of either index type.
struct IndexArgs {
    const void *p;
    int wide;      // int64
};

struct NormArgs {
    const void *q, *k, *v;      // forward; v with a cache only
    int64_t q_stride, k_stride, v_stride;
    const void *gq, *gk;        // backward
    int64_t gq_stride, gk_stride;
    int64_t n;
    int hq, hk, D, rot, neighbours;
    const void *wq, *wk;        // null: no norm
    float eps;
    float inverse_D;            // (set by the launch, this and the next two: 1 / D; tokens that a workgroup takes at a time)
    int tokens_log2;
    double inverse_D64;
    const float *table;         // null: no rotation
    int64_t table_rows;
    IndexArgs positions;
    void *q_out, *k_out;        // (backward: dq, dk)
    int64_t q_out_stride, k_out_stride;
    int to_cache;
    CacheArgs cache;
    IndexArgs slots;
    float *partial, *dqw, *dkw;      // backward with weights
};
hipError_t launch_norm_rope(const NormArgs &a, bool bf16, hipStream_t st);
hipError_t launch_norm_rope_backward(const NormArgs &a, bool bf16, hipStream_t st);
int norm_backward_workgroups(int64_t n);

struct CacheReadArgs {
    CacheArgs cache;
    IndexArgs slots;
    int64_t n;
    void *k_out, *v_out;
};
hipError_t launch_cache_read(const CacheReadArgs &a, bool bf16, hipStream_t st);

struct AttendArgs {
    const void *q;
    int64_t q_stride;
    int n, hq, G;      // query heads, and how many share a kv head
    CacheArgs cache;
    const int32_t *page_table;
    int table_pages;
    const int32_t *lengths;
    int requests;
    const int32_t *row_start;
    int max_rows;
    const uint64_t *tail_mask;
    int window, sinks;       // 0: no window
    IndexArgs positions;     // of rows with a tail mask and a window; null: a request's rows are its last tokens
    int most;          // tokens of a request that are looked at
    float scale_log2;
    void *out;
    int64_t out_stride;
    float *lse;
    int row_blocks, row_tiles;      // blocks of 16 row_tiles query rows
    int whole;                      // a workgroup to each request, kv head and row block
    int places;                     // ... or this many to all requests together, of each kv head and row block
    unsigned G_magic;               // floor(2^32 / G) + 1, G > 1
    float *part_o;                  // [row_blocks, heads, places, 2, 16 row_tiles, D], the same of (max, sum),
    float2 *part_ms;
    int by_place;                   // requests are more than places
    int4 *part_at;                  // [requests or places]: first place of a request's parts, how many, the first one's number there, request
};
// 16-row tiles of queries that one workgroup takes
int attend_row_tiles(int rows, int D, bool f32);
hipError_t launch_attend(const AttendArgs &a, bool f32, hipStream_t st);
// Rows that are a request's last tokens, with a window: row_blocks blocks of 64 row_tiles query rows (csrc/vt_prompt.hip)
hipError_t launch_prompt(const AttendArgs &a, hipStream_t st);

constexpr int kAttendWaves = 4;
constexpr int kAttendTile = 32;                                   // cached tokens that a wave takes at a time
constexpr int kAttendStep = kAttendWaves * kAttendTile;          // ... and a workgroup: the steps that requests are cut up by

// csrc/vt_attend_d*.hip
hipError_t launch_attend_d64(const AttendArgs &a, int tiles, bool f32, hipStream_t st);
hipError_t launch_attend_d128(const AttendArgs &a, int tiles, bool f32, hipStream_t st);
hipError_t launch_attend_d256(const AttendArgs &a, int tiles, bool f32, hipStream_t st);
// csrc/vt_attend_window_d*.hip
hipError_t launch_attend_window_d64(const AttendArgs &a, int tiles, bool f32, hipStream_t st);
hipError_t launch_attend_window_d128(const AttendArgs &a, int tiles, bool f32, hipStream_t st);
hipError_t launch_attend_window_d256(const AttendArgs &a, int tiles, bool f32, hipStream_t st);

// The status of a HIP call's result, remembered for vt_last_device_error (csrc/vt_api.hip)
int status_of_hip(hipError_t e);

}  // namespace vt
