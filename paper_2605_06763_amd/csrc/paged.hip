// The paged cache: its handle, the calls' checks, and the kernels that move rows in (lvr_paged_append) and out
// (lvr_paged_gather).  The attention over the pages is paged_attention.hip.
//
// Both kernels are bound by HBM: every row is read once and written once, in 16-byte accesses.
#include <math.h>
#include <stdlib.h>
#include <string.h>

#include <new>

#include "paged.h"

namespace {

#define LVR_HIP(expr)                                             \
    do {                                                          \
        hipError_t e__ = (expr);                                  \
        if (e__ != hipSuccess) return lvr_note_hip_error(e__);    \
    } while (0)

constexpr int PAIRS = LVR_D / 2;
// Rows of a call (of K, V and q) from which a wave takes up to 24 of them and stores past the caches: it makes its sines and cosines
// once, and the rows are more than the caches would keep.  us with eight rows a wave through the caches / so: 12288 rows 5.2 / 5.1,
// with the attention behind it 21.4 / 23.0; 24576 rows 6.7 / 5.6; 98304 16.3 / 10.9; 393216 48.2 / 37.4 (4.2 / 5.4 TB/s).
constexpr int64_t APPEND_MANY = 16384;
// Bytes of K (and as many of V) from which gathered rows go past the caches.  Below that they wait in the memory-side cache for whoever
// reads them next.  us with lvr_build behind, through / past: 32 MiB 49.8 / 54.3, 128 MiB 189 / 200, 256 MiB 389 / 393; alone 256 MiB
// 202 / 191 (5.3 / 5.6 TB/s).
constexpr int64_t GATHER_STREAM = (int64_t)192 << 20;

// sin and cos of a fraction of a turn, given in units of 2^-32.  The nearest quarter turn is split off exactly (integers), the
// rest lies within an eighth of a turn, where the Taylor series to x^9 and x^10 are off by less than 2^-28.
__device__ __forceinline__ void sincos_turn(uint32_t phase, float &sn, float &cs) {
    const uint32_t quarter = (phase + 0x20000000u) >> 30;
    const int32_t rest = (int32_t)(phase - (quarter << 30));
    const float x = (float)rest * 1.46291807926715968e-9f;   // 2 pi / 2^32
    const float x2 = x * x;
    const float s = x + x * x2 * (-1.f / 6 + x2 * (1.f / 120 + x2 * (-1.f / 5040 + x2 * (1.f / 362880))));
    const float c = 1.f + x2 * (-0.5f + x2 * (1.f / 24 + x2 * (-1.f / 720 + x2 * (1.f / 40320 + x2 * (-1.f / 3628800)))));
    const bool odd = quarter & 1;
    sn = odd ? c : s;
    cs = odd ? s : c;
    if (quarter & 2) sn = -sn;
    if ((quarter + 1) & 2) cs = -cs;
}

// 16 bytes of a row, as elements and back.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ u32x4 load_piece(const char *p) { return *reinterpret_cast<const u32x4 *>(p); }
// STREAM: past the caches, which the rows would only pass through
template <bool STREAM>
__device__ __forceinline__ void store_piece(char *p, u32x4 v) {
    if (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<u32x4 *>(p));
    else *reinterpret_cast<u32x4 *>(p) = v;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 v = {(__bf16)lo, (__bf16)hi};   // rounds to nearest even, NaN stays NaN
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ void elements(u32x4 r, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = lvr_bf16_lo(r[i]);
        x[2 * i + 1] = lvr_bf16_hi(r[i]);
    }
}
__device__ __forceinline__ void elements(u32x4 r, float (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ u32x4 piece_of(const float (&x)[8]) {
    return u32x4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
}
__device__ __forceinline__ u32x4 piece_of(const float (&x)[4]) {
    return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
}

struct AppendArgs {
    const char *k, *v, *q;
    char *k_pages, *v_pages, *q_out;
    int64_t k_stride, v_stride, q_stride;   // bytes per token
    const int32_t *positions;
    const uint64_t *turns;
    const int32_t *axis;
    int32_t n_kv, n_rows, groups;           // rows of a token: n_kv of K, n_kv of V, then q's; waves to a token
    int32_t rot, axes;
};

// A wave takes PER times ROWS rows of one token.  A lane holds two pieces of a row, of E elements each: HALVES: the same one of both
// halves, rotated with each other; NEIGHBOURS: one in each half of the row, rotated within themselves; past the rotated coordinates two that are
// copied.  The lanes of a row touch neighbouring pieces in every access.  A lane needs the sines and cosines of E pairs, for all
// of its rows.  The angle is position times turns per position modulo one turn, which in 64-bit integers is one product with the
// overflow dropped: no far position loses anything.
//
// Bound by HBM where there are tokens enough: 8192 tokens (48 rows each, bf16) 37 us on one axis and 41 to 44 on three, 5.4 and 4.6 to 4.9 TB/s read and written;
// 1885 fp32 tokens of 80 rows 25 us, 6.2 TB/s.  One token: 4.2 us, the launch and three dependent trips (rows and lengths, table, store).
template <typename KT, bool NEIGHBOURS, int PER, bool STREAM>
__global__ void __launch_bounds__(256) paged_append_kernel(AppendArgs a, lvr_paged_batch b) {
    constexpr int ELT = sizeof(KT) == 4 ? 4 : 2, E = 16 / ELT, LANES = PAIRS / E, ROWS = 64 / LANES;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = lvr_lane(), li = lane % LANES;
    const uint32_t w = blockIdx.x * 4u + wave;
    const int t = (int)(w / (uint32_t)a.groups), row0 = (int)(w % (uint32_t)a.groups) * (ROWS * PER) + lane / LANES;
    if (t >= b.n_tokens) return;   // the whole wave

    int at0 = E * li, at1 = PAIRS + E * li;
    bool rot0 = at0 < a.rot, rot1 = at1 < a.rot;
    if (!NEIGHBOURS) {
        const int half = a.rot / 2, copied = li - half / E;
        rot0 = rot1 = copied < 0;
        at0 = rot0 ? E * li : a.rot + E * copied;
        at1 = rot0 ? half + E * li : at0 + E * (LANES - half / E);
    }
    u32x4 r0[PER], r1[PER];
#pragma unroll
    for (int c = 0; c < PER; ++c) {
        int row = row0 + c * ROWS;
        if (row >= a.n_rows) row = a.n_rows - 1;   // nothing is made of it
        const char *src = row < a.n_kv ? a.k + t * a.k_stride + (int64_t)row * (LVR_D * ELT)
                          : row < 2 * a.n_kv ? a.v + t * a.v_stride + (int64_t)(row - a.n_kv) * (LVR_D * ELT)
                                             : a.q + t * a.q_stride + (int64_t)(row - 2 * a.n_kv) * (LVR_D * ELT);
        r0[c] = load_piece(src + at0 * ELT);
        r1[c] = load_piece(src + at1 * ELT);
    }

    const int seq = lvr_seq_of(b, t);
    if (seq < 0 || seq >= b.n_seqs) return;
    const int64_t slot = (int64_t)b.seq_len[seq] - b.seq_start[seq + 1] + t;
    const int page = lvr_page_of(b, seq, slot);
    float sn[E], cs[E];
    if (rot0 || rot1) {
        int pos[4] = {(int)slot, (int)slot, (int)slot, (int)slot};
        if (a.positions)
#pragma unroll
            for (int i = 0; i < 4; ++i) pos[i] = i < a.axes ? a.positions[(int64_t)t * a.axes + i] : 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int pair = NEIGHBOURS ? (e < E / 2 ? 0 : PAIRS / 2 - E / 2) + E * li / 2 + e : E * li + e;
            int p = pos[0];
            if (a.axes > 1) {
                const int ax = a.axis[pair];
                p = ax < 2 ? (ax == 0 ? pos[0] : pos[1]) : (ax == 2 ? pos[2] : pos[3]);
            }
            // the upper half of the product's lower 64 bits
            const uint32_t lo = (uint32_t)a.turns[pair], hi = (uint32_t)(a.turns[pair] >> 32);
            sincos_turn((uint32_t)p * hi + __umulhi((uint32_t)p, lo) - (p < 0 ? lo : 0u), sn[e], cs[e]);
        }
    }
#pragma unroll
    for (int c = 0; c < PER; ++c) {
        const int row = row0 + c * ROWS;
        const bool of_q = row >= 2 * a.n_kv, of_v = row >= a.n_kv && !of_q;
        if (row >= a.n_rows || (!of_q && page < 0)) continue;
        if ((rot0 || rot1) && !of_v) {
            float x[E], y[E];
            elements(r0[c], x);
            elements(r1[c], y);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const bool second = e >= E / 2;
                float &u = NEIGHBOURS ? (second ? y : x)[2 * (e % (E / 2))] : x[e];
                float &z = NEIGHBOURS ? (second ? y : x)[2 * (e % (E / 2)) + 1] : y[e];
                const float first = u * cs[e] - z * sn[e];
                z = u * sn[e] + z * cs[e];
                u = first;
            }
            if (rot0) r0[c] = piece_of(x);
            if (rot1) r1[c] = piece_of(y);
        }
        char *dst = of_q ? a.q_out + ((int64_t)t * (a.n_rows - 2 * a.n_kv) + row - 2 * a.n_kv) * (LVR_D * ELT)
                         : (of_v ? a.v_pages : a.k_pages) + lvr_row_at(b, page, of_v ? row - a.n_kv : row, slot);
        store_piece<STREAM>(dst + at0 * ELT, r0[c]);
        store_piece<STREAM>(dst + at1 * ELT, r1[c]);
    }
}

// A wave takes 16 rows of one head, which lie in one page: one table entry, then 64 pieces of 16 bytes to an access, one behind the other
// where the rows are.  131072 keys of 8 heads 191 us, 5.6 TB/s read and written.
template <typename KT, bool STREAM>
__global__ void __launch_bounds__(256) paged_gather_kernel(const char *k_pages, const char *v_pages, char *K, char *V, int64_t n,
                                                           int32_t n_kv, lvr_paged_batch b) {
    constexpr int ROW = LVR_D * (sizeof(KT) == 4 ? 4 : 2), LANES = ROW / 16, ROWS = 64 / LANES, N = 16 / ROWS;
    const int lane = lvr_lane(), r0 = lane / LANES, at = lane % LANES * 16;
    const int64_t groups = (n + 15) / 16, total = groups * n_kv * b.n_seqs;
    const int64_t step = (int64_t)gridDim.x * 4;
    for (int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); w < total; w += step) {
        const int64_t bh = w / groups;
        const int64_t row0 = (w - bh * groups) * 16;
        const int seq = (int)(bh / n_kv), head = (int)(bh - (int64_t)seq * n_kv);
        int64_t end = b.seq_len[seq];
        if (end > n) end = n;
        if (row0 >= end) continue;
        const int page = lvr_page_of(b, seq, row0);   // the table ends with a page, so all 16 rows are in it or none
        if (page < 0) continue;
        const int64_t from = lvr_row_at(b, page, head, row0) + at;
        const int64_t to = (bh * n + row0) * ROW + at;
        const int last = (int)(end - row0 < 16 ? end - row0 : 16) - 1;
        u32x4 k[N], v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = i * ROWS + r0 < last ? i * ROWS + r0 : last;   // past the end: the last row once more
            k[i] = load_piece(k_pages + from + r * b.row_stride);
            v[i] = load_piece(v_pages + from + r * b.row_stride);
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i * ROWS + r0 <= last) {
                store_piece<STREAM>(K + to + (i * ROWS + r0) * ROW, k[i]);
                store_piece<STREAM>(V + to + (i * ROWS + r0) * ROW, v[i]);
            }
    }
}

int check_config(const lvr_paged_config *c) {
    if (!c) return LVR_E_INVALID;
    if (c->n_q_heads <= 0 || c->n_kv_heads <= 0 || c->n_q_heads % c->n_kv_heads != 0) return LVR_E_INVALID;
    if (c->kv_dtype != LVR_BF16 && c->kv_dtype != LVR_F32) return LVR_E_INVALID;
    if (!(c->scale >= 0.f) || isinf(c->scale)) return LVR_E_INVALID;
    if (c->page_size <= 0 || c->n_pages <= 0) return LVR_E_INVALID;
    if (c->rot_dim < 0 || c->rot_dim > c->head_dim || c->rot_dim % 2) return LVR_E_INVALID;
    if (c->rot_dim > 0 && (c->rot_axes < 1 || c->rot_axes > 4)) return LVR_E_INVALID;
    if (c->rot_pairs != LVR_ROT_HALVES && c->rot_pairs != LVR_ROT_NEIGHBOURS) return LVR_E_INVALID;
    const int64_t per16 = c->kv_dtype == LVR_BF16 ? 8 : 4;
    for (int i = 0; i < 3; ++i)
        if (c->page_strides[i] < 0 || c->page_strides[i] % per16 || c->page_strides[i] > (int64_t)1 << 40) return LVR_E_INVALID;
    if (c->page_strides[2] < c->head_dim) return LVR_E_INVALID;
    if (c->head_dim != LVR_D || c->rot_dim % 16 != 0) return LVR_E_UNSUPPORTED;
    if (c->n_q_heads > 1024 || c->n_kv_heads > 256) return LVR_E_UNSUPPORTED;
    if (c->page_size < 16 || c->page_size > 65536 || (c->page_size & (c->page_size - 1))) return LVR_E_UNSUPPORTED;
    if (c->n_pages > (int64_t)1 << 30) return LVR_E_UNSUPPORTED;
    if (c->page_strides[2] > (int64_t)1 << 24) return LVR_E_UNSUPPORTED;   // 16 rows of a page are told apart by 32-bit offsets
    return LVR_OK;
}

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// What the calls have in common; LVR_OK with *b filled, or the refusal.
int check_batch(const lvr_paged *pc, const void *k_pages, const void *v_pages, const int32_t *seq_start, bool needs_start,
                const int32_t *seq_len, const int32_t *table, int64_t table_width, int64_t n_seqs, int64_t n_tokens,
                lvr_paged_batch *b) {
    if (!pc || n_seqs < 0 || n_tokens < 0 || table_width < 0) return LVR_E_INVALID;
    if (n_seqs > LVR_PAGED_MAX_SEQS) return LVR_E_CAPACITY;
    if (table_width > ((int64_t)1 << 30) / pc->cfg.page_size) return LVR_E_CAPACITY;
    if (n_tokens > ((int64_t)1 << 27) / (pc->cfg.n_q_heads > 16 ? pc->cfg.n_q_heads : 16)) return LVR_E_CAPACITY;   // a launch's threads stay below 2^32
    if (n_seqs > 0 && (!k_pages || !v_pages || !seq_len || (needs_start && !seq_start) || (table_width > 0 && !table)))
        return LVR_E_INVALID;
    if (!aligned16(k_pages) || !aligned16(v_pages) || !aligned4(seq_start) || !aligned4(seq_len) || !aligned4(table))
        return LVR_E_INVALID;
    int d = -1;
    if (hipGetDevice(&d) != hipSuccess || d != pc->device) return LVR_E_STATE;
    const int64_t elt = pc->cfg.kv_dtype == LVR_BF16 ? 2 : 4;
    b->seq_start = seq_start;
    b->seq_len = seq_len;
    b->table = table;
    b->n_seqs = (int32_t)n_seqs;
    b->n_tokens = (int32_t)n_tokens;
    b->table_width = (int32_t)table_width;
    b->page_shift = __builtin_ctz((unsigned)pc->cfg.page_size);
    b->n_pages = (int32_t)pc->cfg.n_pages;
    b->page_stride = pc->cfg.page_strides[0] * elt;
    b->head_stride = pc->cfg.page_strides[1] * elt;
    b->row_stride = pc->cfg.page_strides[2] * elt;
    return LVR_OK;
}

// A stride between tokens of `heads` contiguous heads, in elements.
bool token_stride_ok(int64_t s, int heads, int64_t elt) {
    return s >= (int64_t)heads * LVR_D && s * elt % 16 == 0 && s <= (int64_t)1 << 32;
}

void free_all(lvr_paged *pc) {
    void *ptrs[] = {pc->turns};
    for (void *p : ptrs)
        if (p) (void)hipFree(p);
}

struct Sizes {
    size_t turns, axis, ticket, part, total;
};
Sizes sizes_of(const lvr_paged_config *) {
    auto al = [](size_t b) { return (b + 255) / 256 * 256; };
    Sizes s;
    s.turns = al(PAIRS * sizeof(uint64_t));
    s.axis = al(PAIRS * sizeof(int32_t));
    s.ticket = al(lvr_paged_ticket_bytes());
    s.part = al(lvr_paged_partial_bytes());
    s.total = s.turns + s.axis + s.ticket + s.part;
    return s;
}

}  // namespace

extern "C" {

size_t lvr_paged_bytes(const lvr_paged_config *cfg) {
    if (check_config(cfg) != LVR_OK) return 0;
    return sizes_of(cfg).total;
}

int lvr_paged_create(const lvr_paged_config *cfg, const double *inv_freq, const int32_t *axis, lvr_paged **out) {
    if (!out) return LVR_E_INVALID;
    const int rc = check_config(cfg);
    if (rc != LVR_OK) return rc;
    uint64_t turns[PAIRS] = {};
    int32_t axes[PAIRS] = {};
    if (cfg->rot_dim > 0) {
        if (!inv_freq) return LVR_E_INVALID;
        for (int c = 0; c < cfg->rot_dim / 2; ++c) {
            if (!isfinite(inv_freq[c])) return LVR_E_INVALID;
            if (axis && (axis[c] < 0 || axis[c] >= cfg->rot_axes)) return LVR_E_INVALID;
            axes[c] = axis ? axis[c] : 0;
            turns[c] = lvr_turns_of(inv_freq[c]);
        }
    }
    lvr_paged *pc = new (std::nothrow) lvr_paged();
    if (!pc) return LVR_E_NOMEM;
    memset(pc, 0, sizeof(*pc));
    pc->cfg = *cfg;
    pc->sigma = cfg->scale > 0.f ? cfg->scale : 1.0f / sqrtf((float)cfg->head_dim);
    const Sizes s = sizes_of(cfg);
    hipError_t e = hipGetDevice(&pc->device);
    if (e == hipSuccess) e = hipMalloc((void **)&pc->turns, s.total);
    if (e == hipSuccess) {
        char *at = reinterpret_cast<char *>(pc->turns) + s.turns;
        pc->axis = reinterpret_cast<int32_t *>(at);
        pc->ticket = reinterpret_cast<uint32_t *>(at + s.axis);
        pc->part = reinterpret_cast<float *>(at + s.axis + s.ticket);
        e = hipMemset(pc->turns, 0, s.turns + s.axis + s.ticket);
        if (e == hipSuccess) e = hipMemcpy(pc->turns, turns, sizeof(turns), hipMemcpyHostToDevice);
        if (e == hipSuccess) e = hipMemcpy(pc->axis, axes, sizeof(axes), hipMemcpyHostToDevice);
        if (e == hipSuccess) e = hipDeviceSynchronize();
    }
    if (e != hipSuccess) {
        free_all(pc);
        delete pc;
        (void)hipGetLastError();   // the failure is reported here, not by whatever HIP call comes next
        (void)lvr_note_hip_error(e);
        return e == hipErrorOutOfMemory ? LVR_E_NOMEM : LVR_E_HIP;
    }
    *out = pc;
    return LVR_OK;
}

int lvr_paged_destroy(lvr_paged *pc) {
    if (!pc) return LVR_E_INVALID;
    (void)hipDeviceSynchronize();
    free_all(pc);
    delete pc;
    return LVR_OK;
}

int lvr_paged_append(lvr_paged *pc, void *k_pages, void *v_pages, const void *k_new, const void *v_new, const void *q, void *q_out,
                     const int64_t strides[3], const int32_t *positions, const int32_t *seq_start, const int32_t *seq_len,
                     const int32_t *table, int64_t table_width, int64_t n_seqs, int64_t n_tokens, void *stream) {
    lvr_paged_batch b;
    const int rc = check_batch(pc, k_pages, v_pages, seq_start, true, seq_len, table, table_width, n_seqs, n_tokens, &b);
    if (rc != LVR_OK) return rc;
    if (!q != !q_out) return LVR_E_INVALID;
    if (n_tokens == 0 || n_seqs == 0) return LVR_OK;
    if (!k_new || !v_new || !strides) return LVR_E_INVALID;
    const lvr_paged_config &c = pc->cfg;
    const int64_t elt = c.kv_dtype == LVR_BF16 ? 2 : 4;
    if (!token_stride_ok(strides[0], c.n_kv_heads, elt) || !token_stride_ok(strides[1], c.n_kv_heads, elt)) return LVR_E_INVALID;
    if (q && !token_stride_ok(strides[2], c.n_q_heads, elt)) return LVR_E_INVALID;
    if (q && q == q_out && strides[2] != (int64_t)c.n_q_heads * LVR_D) return LVR_E_INVALID;
    if (!aligned16(k_new) || !aligned16(v_new) || !aligned16(q) || !aligned16(q_out) || !aligned4(positions)) return LVR_E_INVALID;
    AppendArgs a;
    a.k = static_cast<const char *>(k_new);
    a.v = static_cast<const char *>(v_new);
    a.q = static_cast<const char *>(q);
    a.k_pages = static_cast<char *>(k_pages);
    a.v_pages = static_cast<char *>(v_pages);
    a.q_out = static_cast<char *>(q_out);
    a.k_stride = strides[0] * elt;
    a.v_stride = strides[1] * elt;
    a.q_stride = q ? strides[2] * elt : 0;
    a.positions = positions;
    a.turns = pc->turns;
    a.axis = pc->axis;
    a.n_kv = c.n_kv_heads;
    a.n_rows = 2 * c.n_kv_heads + (q ? c.n_q_heads : 0);
    a.rot = c.rot_dim;
    a.axes = c.rot_axes;
    // Where there are tokens enough to fill the device a wave takes up to 24 rows, for which it makes sines and cosines once
    const int rows = c.kv_dtype == LVR_BF16 ? 8 : 4;   // a wave's at a time
    const bool many = n_tokens * a.n_rows >= APPEND_MANY;
    const int per_wave = many ? 24 : rows;
    a.groups = (a.n_rows + per_wave - 1) / per_wave;
    const dim3 grid((unsigned)((n_tokens * a.groups + 3) / 4));
    hipStream_t st = static_cast<hipStream_t>(stream);
#define LVR_APPEND_PER(KT, N, PER)                                                                                \
    do {                                                                                                          \
        if (many) hipLaunchKernelGGL((paged_append_kernel<KT, N, PER, true>), grid, dim3(256), 0, st, a, b);      \
        else hipLaunchKernelGGL((paged_append_kernel<KT, N, 1, false>), grid, dim3(256), 0, st, a, b);            \
    } while (0)
#define LVR_APPEND(KT, PER)                                                       \
    do {                                                                          \
        if (c.rot_pairs == LVR_ROT_NEIGHBOURS) LVR_APPEND_PER(KT, true, PER);     \
        else LVR_APPEND_PER(KT, false, PER);                                      \
    } while (0)
    if (c.kv_dtype == LVR_BF16) LVR_APPEND(lvr_bf16_t, 3);
    else LVR_APPEND(lvr_f32_t, 6);
#undef LVR_APPEND
#undef LVR_APPEND_PER
    LVR_HIP(hipGetLastError());
    return LVR_OK;
}

int lvr_paged_attention(lvr_paged *pc, const void *k_pages, const void *v_pages, const void *q, int64_t q_token_stride,
                        const int32_t *seq_start, const int32_t *seq_len, const int32_t *table, int64_t table_width,
                        int64_t n_seqs, int64_t n_tokens, int32_t window, void *out, void *stream) {
    lvr_paged_batch b;
    const int rc = check_batch(pc, k_pages, v_pages, seq_start, true, seq_len, table, table_width, n_seqs, n_tokens, &b);
    if (rc != LVR_OK) return rc;
    if (window < 0) return LVR_E_INVALID;
    if (n_tokens == 0 || n_seqs == 0) return LVR_OK;
    const int64_t elt = pc->cfg.kv_dtype == LVR_BF16 ? 2 : 4;
    if (!q || !out || q == out || !aligned16(q) || !aligned16(out)) return LVR_E_INVALID;
    if (!token_stride_ok(q_token_stride, pc->cfg.n_q_heads, elt)) return LVR_E_INVALID;
    LVR_HIP(lvr_launch_paged_attention(pc, b, k_pages, v_pages, q, q_token_stride * elt, window, out, static_cast<hipStream_t>(stream)));
    return LVR_OK;
}

int lvr_paged_gather(lvr_paged *pc, const void *k_pages, const void *v_pages, const int32_t *seq_len, const int32_t *table,
                     int64_t table_width, int64_t n_seqs, int64_t n, void *K_out, void *V_out, void *stream) {
    lvr_paged_batch b;
    const int rc = check_batch(pc, k_pages, v_pages, nullptr, false, seq_len, table, table_width, n_seqs, 0, &b);
    if (rc != LVR_OK) return rc;
    if (n < 0) return LVR_E_INVALID;
    if (n > (int64_t)1 << 30) return LVR_E_CAPACITY;
    if (n == 0 || n_seqs == 0) return LVR_OK;
    if (!K_out || !V_out || !aligned16(K_out) || !aligned16(V_out)) return LVR_E_INVALID;
    const int n_kv = pc->cfg.n_kv_heads;
    const int64_t total = (n + 15) / 16 * n_kv * n_seqs;
    const int64_t wgs = (total + 3) / 4 < 65536 ? (total + 3) / 4 : 65536;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool stream_out = n * n_kv * n_seqs * LVR_D * (pc->cfg.kv_dtype == LVR_BF16 ? 2 : 4) >= GATHER_STREAM;
#define LVR_GATHER(KT, S)                                                                                                             \
    hipLaunchKernelGGL((paged_gather_kernel<KT, S>), dim3((unsigned)wgs), dim3(256), 0, st, static_cast<const char *>(k_pages),       \
                       static_cast<const char *>(v_pages), static_cast<char *>(K_out), static_cast<char *>(V_out), n, n_kv, b)
    if (pc->cfg.kv_dtype == LVR_BF16) {
        if (stream_out) LVR_GATHER(lvr_bf16_t, true);
        else LVR_GATHER(lvr_bf16_t, false);
    } else {
        if (stream_out) LVR_GATHER(lvr_f32_t, true);
        else LVR_GATHER(lvr_f32_t, false);
    }
#undef LVR_GATHER
    LVR_HIP(hipGetLastError());
    return LVR_OK;
}

}  // extern "C"
