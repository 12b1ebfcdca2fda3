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

// Eight elements of a row from element `at` on, as they are stored.
__device__ __forceinline__ void load_raw8(const char *row, int at, lvr_raw8<lvr_bf16_t> &r) {
    r.a = *reinterpret_cast<const uint4 *>(row + at * 2);
}
__device__ __forceinline__ void load_raw8(const char *row, int at, lvr_raw8<lvr_f32_t> &r) {
    r.a = *reinterpret_cast<const float4 *>(row + at * 4);
    r.b = *reinterpret_cast<const float4 *>(row + at * 4 + 16);
}
__device__ __forceinline__ void store_raw8(char *row, int at, const lvr_raw8<lvr_bf16_t> &r) {
    *reinterpret_cast<uint4 *>(row + at * 2) = r.a;
}
__device__ __forceinline__ void store_raw8(char *row, int at, const lvr_raw8<lvr_f32_t> &r) {
    *reinterpret_cast<float4 *>(row + at * 4) = r.a;
    *reinterpret_cast<float4 *>(row + at * 4 + 16) = r.b;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 v = {(__bf16)lo, (__bf16)hi};   // rounds to nearest even, NaN stays NaN
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ void pack8(const float (&x)[8], lvr_raw8<lvr_bf16_t> &r) {
    r.a = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}
__device__ __forceinline__ void pack8(const float (&x)[8], lvr_raw8<lvr_f32_t> &r) {
    r.a = make_float4(x[0], x[1], x[2], x[3]);
    r.b = make_float4(x[4], x[5], x[6], x[7]);
}

struct AppendArgs {
    const char *k, *v, *q;
    char *k_pages, *v_pages, *q_out;
    int64_t k_stride, v_stride, q_stride;   // bytes per token
    const int32_t *positions;
    const uint64_t *turns;
    const int32_t *axis;
    int32_t n_kv, n_rows, chunks;           // rows of a token: n_kv of K, n_kv of V, then q's; chunks of eight rows
    int32_t rot, axes;
};

// A wave takes eight rows of one token, eight lanes to a row.  A lane holds 16 elements in two runs of eight that are rotated with
// each other (HALVES: the same run of both halves; NEIGHBOURS: 16 in a row), and so the sines and cosines of eight pairs; past
// the rotated coordinates it copies 16 in a row.  The angle is position times turns per position modulo one turn, which in
// 64-bit integers is one product with the overflow dropped: no far position loses anything.
template <typename KT, bool NEIGHBOURS>
__global__ void __launch_bounds__(256) paged_append_kernel(AppendArgs a, lvr_paged_batch b) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = lvr_lane(), li = lane & 7;
    const uint32_t w = blockIdx.x * 4u + wave;
    const int t = (int)(w / (uint32_t)a.chunks), row = (int)(w % (uint32_t)a.chunks) * 8 + (lane >> 3);
    if (t >= b.n_tokens) return;   // the whole wave

    constexpr int ELT = sizeof(KT) == 4 ? 4 : 2;
    const int half = a.rot / 2;
    const bool rotates = li * 16 < a.rot && !(row >= a.n_kv && row < 2 * a.n_kv);
    int at0 = li * 16, at1 = at0 + 8;
    if (!NEIGHBOURS && li * 16 < a.rot) {
        at0 = li * 8;
        at1 = half + at0;
    }
    const int head = row < a.n_kv ? row : (row < 2 * a.n_kv ? row - a.n_kv : row - 2 * a.n_kv);
    const char *src = row < a.n_kv ? a.k + t * a.k_stride : (row < 2 * a.n_kv ? a.v + t * a.v_stride : a.q + t * a.q_stride);
    lvr_raw8<KT> r0, r1;
    if (row < a.n_rows) {
        load_raw8(src + (int64_t)head * LVR_D * ELT, at0, r0);
        load_raw8(src + (int64_t)head * LVR_D * ELT, at1, r1);
    }

    const int seq = lvr_seq_of(b, t);
    if (seq < 0 || seq >= b.n_seqs || row >= a.n_rows) return;
    const int64_t slot = (int64_t)b.seq_len[seq] - b.seq_start[seq + 1] + t;
    char *dst = nullptr;
    if (row >= 2 * a.n_kv) {
        dst = a.q_out + ((int64_t)t * (a.n_rows - 2 * a.n_kv) + head) * LVR_D * ELT;
    } else {
        const int page = lvr_page_of(b, seq, slot);
        if (page >= 0) dst = (row < a.n_kv ? a.k_pages : a.v_pages) + lvr_row_at(b, page, head, slot);
    }
    if (!dst) return;

    if (rotates) {
        float x[8], y[8];
        lvr_unpack(r0, x);
        lvr_unpack(r1, y);
        int pos[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) pos[i] = a.positions ? (i < a.axes ? a.positions[(int64_t)t * a.axes + i] : 0) : (int)slot;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int ax = a.axis[li * 8 + e];
            const int p = ax < 2 ? (ax == 0 ? pos[0] : pos[1]) : (ax == 2 ? pos[2] : pos[3]);
            float sn, cs;
            sincos_turn((uint32_t)(((uint64_t)(int64_t)p * a.turns[li * 8 + e]) >> 32), sn, cs);
            float &u = NEIGHBOURS ? (e < 4 ? x[2 * (e & 3)] : y[2 * (e & 3)]) : x[e];
            float &z = NEIGHBOURS ? (e < 4 ? x[2 * (e & 3) + 1] : y[2 * (e & 3) + 1]) : y[e];
            const float first = u * cs - z * sn, second = u * sn + z * cs;
            u = first;
            z = second;
        }
        pack8(x, r0);
        pack8(y, r1);
    }
    store_raw8(dst, at0, r0);
    store_raw8(dst, at1, r1);
}

// A wave takes 16 rows of one head, which lie in one page: one table entry, then every row in one access of 16 lanes (fp32: two).
template <typename KT>
__global__ void __launch_bounds__(256) paged_gather_kernel(const char *k_pages, const char *v_pages, char *K, char *V, int64_t n,
                                                           int32_t n_kv, lvr_paged_batch b) {
    constexpr int ROW = LVR_D * (sizeof(KT) == 4 ? 4 : 2);
    const int lane = lvr_lane(), sub = lane >> 4, li = lane & 15;
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
        const int64_t from = lvr_row_at(b, page, head, row0);
        const int64_t to = (bh * n + row0) * ROW;
        const int last = (int)(end - row0 < 16 ? end - row0 : 16) - 1;
        lvr_raw8<KT> k[4], v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = i * 4 + sub < last ? i * 4 + sub : last;   // past the end: the last row once more
            load_raw8(k_pages + from + r * b.row_stride, li * 8, k[i]);
            load_raw8(v_pages + from + r * b.row_stride, li * 8, v[i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i * 4 + sub <= last) {
                store_raw8(K + to + (i * 4 + sub) * ROW, li * 8, k[i]);
                store_raw8(V + to + (i * 4 + sub) * ROW, li * 8, v[i]);
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
            // turns per position without the whole ones, as a fraction of 2^64 (80-bit arithmetic: off by a unit or two)
            long double f = (long double)inv_freq[c] / 6.283185307179586476925286766559L;
            f -= floorl(f);
            f = ldexpl(f, 64);
            turns[c] = f >= 18446744073709551615.0L ? 0 : (uint64_t)f;
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
    a.chunks = (a.n_rows + 7) / 8;
    a.rot = c.rot_dim;
    a.axes = c.rot_axes;
    const dim3 grid((unsigned)((n_tokens * a.chunks + 3) / 4));
    hipStream_t st = static_cast<hipStream_t>(stream);
#define LVR_APPEND(KT, N) hipLaunchKernelGGL((paged_append_kernel<KT, N>), grid, dim3(256), 0, st, a, b)
    if (c.kv_dtype == LVR_BF16) {
        if (c.rot_pairs == LVR_ROT_NEIGHBOURS) LVR_APPEND(lvr_bf16_t, true);
        else LVR_APPEND(lvr_bf16_t, false);
    } else {
        if (c.rot_pairs == LVR_ROT_NEIGHBOURS) LVR_APPEND(lvr_f32_t, true);
        else LVR_APPEND(lvr_f32_t, false);
    }
#undef LVR_APPEND
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
    if (pc->cfg.kv_dtype == LVR_BF16)
        hipLaunchKernelGGL(paged_gather_kernel<lvr_bf16_t>, dim3((unsigned)wgs), dim3(256), 0, st, static_cast<const char *>(k_pages),
                           static_cast<const char *>(v_pages), static_cast<char *>(K_out), static_cast<char *>(V_out), n, n_kv, b);
    else
        hipLaunchKernelGGL(paged_gather_kernel<lvr_f32_t>, dim3((unsigned)wgs), dim3(256), 0, st, static_cast<const char *>(k_pages),
                           static_cast<const char *>(v_pages), static_cast<char *>(K_out), static_cast<char *>(V_out), n, n_kv, b);
    LVR_HIP(hipGetLastError());
    return LVR_OK;
}

}  // extern "C"
