// The paged cache's handle and what its kernels share: where a token, a page and a row lie.
#pragma once
#include <math.h>

#include "lvr_internal.h"

#define LVR_PAGED_MAX_SEQS 4096

struct lvr_paged {
    lvr_paged_config cfg;
    int device;
    float sigma;
    uint64_t *turns;      // [64] turns per position of every pair, in units of 2^-64 turn (whole turns dropped)
    int32_t *axis;        // [64] axis of every pair
    float *part;          // partial results of the attention
    uint32_t *ticket;     // zero between calls
};

// What every kernel over a batch gets.
struct lvr_paged_batch {
    const int32_t *seq_start, *seq_len, *table;
    int32_t n_seqs, n_tokens, table_width;
    int32_t page_shift;        // log2 of the page size
    int32_t n_pages;
    int64_t page_stride, head_stride, row_stride;   // bytes
};

// work space of the attention, whatever the batch
size_t lvr_paged_partial_bytes();
size_t lvr_paged_ticket_bytes();
hipError_t lvr_launch_paged_attention(lvr_paged *pc, const lvr_paged_batch &b, const void *k_pages, const void *v_pages, const void *q,
                                      int64_t q_stride_bytes, int32_t window, void *out, hipStream_t st);

// A frequency's turns per position, frequency / 2 pi without the whole turns, in units of 2^-64 turn; off by less than one.  With the
// frequency m * 2^e (m a whole number of 53 bits), bits of 1 / 2 pi above 2^-e make whole turns alone and those 128 further down none that
// count, so that m times the 128 between them is all there is to it (M. Payne and R. Hanek, "Radian reduction for trigonometric functions", 1983).
inline uint64_t lvr_turns_of(double inv_freq) {
    // 1 / 2 pi, 1152 bits behind the point; the largest double needs 971 + 128 of them
    static const uint64_t per_radian[18] = {
        0x28be60db9391054a, 0x7f09d5f47d4d3770, 0x36d8a5664f10e410, 0x7f9458eaf7aef158, 0x6dc91b8e909374b8, 0x01924bba82746487,
        0x3f877ac72c4a69cf, 0xba208d7d4baed121, 0x3a671c09ad17df90, 0x4e64758e60d4ce7d, 0x272117e2ef7e4a0e, 0xc7fe25fff7816603,
        0xfbcbc462d6829b47, 0xdb4d9fb3c9f2c26d, 0xd3d18fd9a797fa8b, 0x5d49eeb1faf97c5e, 0xcf41ce7de294a4ba, 0x9afed7ec47e35742};
    typedef unsigned __int128 u128;
    int e;
    const uint64_t m = (uint64_t)ldexp(frexp(fabs(inv_freq), &e), 53);
    e -= 53;
    const int word = e > 0 ? e / 64 : 0, shift = e > 0 ? e % 64 : 0;
    auto bits = [&](int i) { return shift ? per_radian[i] << shift | per_radian[i + 1] >> (64 - shift) : per_radian[i]; };
    const u128 low = (u128)m * bits(word + 1), high = (u128)m * bits(word) + (low >> 64);
    uint64_t turns;
    if (e >= 0) turns = (uint64_t)high + ((uint64_t)low >> 63);
    else turns = e > -128 ? (uint64_t)((high + ((u128)1 << (-e - 1))) >> -e) : 0;
    return inv_freq < 0 ? 0 - turns : turns;
}

#ifdef __HIPCC__
// The page that holds a position of a sequence, or -1: a position outside the table, or an entry outside the pool.
__host__ __device__ __forceinline__ int32_t lvr_page_of(const lvr_paged_batch &b, int seq, int64_t position) {
    if (position < 0 || position >= (int64_t)b.table_width << b.page_shift) return -1;
    const int32_t page = b.table[(int64_t)seq * b.table_width + (position >> b.page_shift)];
    return page >= 0 && page < b.n_pages ? page : -1;
}
// Bytes from the start of a pool to the row of a position in that page.
__host__ __device__ __forceinline__ int64_t lvr_row_at(const lvr_paged_batch &b, int32_t page, int head, int64_t position) {
    return page * b.page_stride + head * b.head_stride + (position & (((int64_t)1 << b.page_shift) - 1)) * b.row_stride;
}

// The sequence a row of the packed arrays belongs to: the last one that starts at or before it (an empty one starts where its
// successor does).  -1 or n_seqs: none.  One load per 64 sequences and no dependent search; all lanes of a wave call it with the same t.
__device__ __forceinline__ int lvr_seq_of(const lvr_paged_batch &b, int t) {
    int before = 0;
    for (int i0 = 0; i0 <= b.n_seqs; i0 += 64) {
        const int i = i0 + lvr_lane();
        const bool starts = i <= b.n_seqs && b.seq_start[i] <= t;
        before += __popcll(__ballot(starts));
    }
    return before - 1;
}
#endif
