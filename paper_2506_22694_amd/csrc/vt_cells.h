// Where a paged cache's rows lie, for the kernels that write and read them.  No HIP in here: what arrives in device memory (slots,
// page numbers, lengths) is checked by these functions alone, and the tests run them on the host.
#pragma once
#include <stdint.h>

#ifdef __HIPCC__
#define VT_BOTH __host__ __device__ __forceinline__
#else
#define VT_BOTH inline
#endif

namespace vt {

// Index of a head's row in [pages, heads, page_size], or -1 for a slot outside the cache.
VT_BOTH int64_t row_of_slot(int64_t slot, int64_t pages, int heads, int head, int page_shift) {
    if (slot < 0 || (slot >> page_shift) >= pages) return -1;
    const int64_t place = slot & (((int64_t)1 << page_shift) - 1);
    return ((((slot >> page_shift) * heads) + head) << page_shift) + place;
}
// Index of a head's first row in a page, or -1 for a page outside the cache.
VT_BOTH int64_t row_of_page(int page, int64_t pages, int heads, int head, int page_shift) {
    if (page < 0 || page >= pages) return -1;
    return ((int64_t)page * heads + head) << page_shift;
}
// Cached tokens of a request that are looked at.
VT_BOTH int tokens_of(int length, int most) { return length < 0 ? 0 : length > most ? most : length; }

// New rows of request b: the first one in `first`; none where row_start is out of order or past the n rows there are.
VT_BOTH int rows_of(const int32_t *row_start, int b, int n, int max_rows, int &first) {
    if (row_start == nullptr) {
        first = b;
        return 1;
    }
    first = row_start[b];
    int end = row_start[b + 1];
    if (end > n) end = n;
    if (first < 0 || end <= first) return 0;
    return end - first > max_rows ? max_rows : end - first;
}

// Requests are taken in steps of `step` tokens; one without tokens has one too, for its rows' results.
VT_BOTH int steps_of(int tokens, int rows, int step) {
    return rows <= 0 ? 0 : tokens <= step ? 1 : (int)((unsigned)(tokens - 1) / (unsigned)step) + 1;
}
// All requests' steps, one after the other, in shares of `per`: the start of share `place`, and its length (0: there is none).
VT_BOTH int share_steps(int all, int places, int place, int &per, int &start) {
    per = all <= places ? 1 : (int)((unsigned)(all - 1) / (unsigned)places) + 1;
    const int64_t from = (int64_t)place * per;
    start = from < all ? (int)from : all;
    return all - start < per ? all - start : per;
}

// Exponent (biased by 127) of the smallest power of two 2^e, e >= -126, with amax <= 448 * 2^e, from the bits of a finite amax >= 0:
// 448 = 1.75 * 2^8.
VT_BOTH int scale_exponent(uint32_t amax_bits) {
    const int e = (int)(amax_bits >> 23) - 8 + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return e < 1 ? 1 : e;
}

}  // namespace vt
