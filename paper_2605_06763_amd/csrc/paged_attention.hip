// Attention of new tokens over the pages (lvr_paged_attention).
//
// The query rows that share a KV head are packed: row = token * G + (head within the group), so that a token's G heads, and the
// tokens of a chunk, fill the columns of a matrix instruction whatever G is.  Both products are taken transposed,
//     S^T = K Q^T   (rows: keys, columns: query rows)        O^T = V^T P^T   (rows: coordinates, columns: query rows)
// so that a lane holds the scores of ONE query row: running maximum, sum and rescaling are values of a lane, and the scores
// become the second product's operand without leaving it.
//
// Softmax in one pass, base 2 (the logit is score * sigma * log2 e in one fused multiply-add with the running maximum).  The
// maximum is raised, and what was summed so far rescaled, only when a score passes it by more than RAISE: until then
// weights grow up to 2^RAISE, which costs nothing in fp32 sums, and no lane has to ask another one for a maximum.
#include "paged.h"

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float RAISE = 8.f;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 v = {(__bf16)lo, (__bf16)hi};   // rounds to nearest even, NaN stays NaN
    return __builtin_bit_cast(uint32_t, v);
}

struct AttnArgs {
    const char *k_pages, *v_pages, *q;
    char *out;
    int64_t q_stride;    // bytes per token
    int32_t n_kv, G, window;
    float unit;          // sigma * log2 e
};

// A tile of TM packed rows of one sequence: which, and what its rows see.
struct Tile {
    int seq, row0, rows;       // first packed row within the sequence; rows of the sequence
    int first_token;           // of the sequence, in the packed arrays
    int pos0;                  // position of the sequence's first new token
    int lo, hi;                // keys that any row of the tile sees: lo .. hi - 1
};

// Tiles are numbered sequence by sequence: those of sequence b start at seq_start[b] * G / TM + b, which leaves at most
// one number unused per sequence and needs no sum over the sequences before it.
template <int TM>
__device__ __forceinline__ bool find_tile(const lvr_paged_batch &b, int G, int window, int x, Tile &t) {
    int before = 0;
    for (int i0 = 0; i0 < b.n_seqs; i0 += 64) {
        const int i = i0 + lvr_lane();
        bool starts = false;
        if (i < b.n_seqs) {
            int s = b.seq_start[i];
            s = s < 0 ? 0 : (s > b.n_tokens ? b.n_tokens : s);
            starts = (s * G) / TM + i <= x;
        }
        before += __popcll(__ballot(starts));
    }
    if (before == 0) return false;
    t.seq = before - 1;
    int s0 = b.seq_start[t.seq], s1 = b.seq_start[t.seq + 1], n = b.seq_len[t.seq];
    s0 = s0 < 0 ? 0 : (s0 > b.n_tokens ? b.n_tokens : s0);
    s1 = s1 < s0 ? s0 : (s1 > b.n_tokens ? b.n_tokens : s1);
    n = n < 0 ? 0 : n;
    t.first_token = s0;
    t.rows = (s1 - s0) * G;
    t.row0 = (x - ((s0 * G) / TM + t.seq)) * TM;
    if (t.row0 < 0 || t.row0 >= t.rows) return false;
    t.pos0 = n - (s1 - s0);
    const int last_row = (t.row0 + TM < t.rows ? t.row0 + TM : t.rows) - 1;
    t.hi = t.pos0 + last_row / G + 1;
    if (t.hi > b.table_width << b.page_shift) t.hi = b.table_width << b.page_shift;
    t.lo = window ? t.pos0 + t.row0 / G - window + 1 : 0;
    if (t.lo < 0) t.lo = 0;
    return true;
}

// ---------------------------------------------------------------------------------------------------------------------------
// 16 rows to a tile.  A workgroup of four waves; a wave takes 32 keys at a time straight into registers.
//
// Matrix operand lanes: i = lane & 15, b = lane >> 4.  A score tile is 16 keys: row r = 4 b + j of the result is register j of
// lanes (., b), the column i is the query row.  As the second product's operand those scores are the keys that lanes (., b)
// contribute, so key r of the tile is held as V row 4 b + j by the lanes that load it: a row is read whole by 16 lanes, eight
// coordinates each, and which coordinates share a result tile is free as well (tile u: coordinates 8 i + u).
// bf16: two score tiles make one operand of 32 keys; a pair of V rows is woven into it by byte permutes.
// ---------------------------------------------------------------------------------------------------------------------------
template <typename KT>
struct Rows16;

template <>
struct Rows16<lvr_bf16_t> {
    static constexpr int ELT = 2;
    typedef bf16x8 Q[4];
    typedef uint4 K[2][4];
    typedef uint4 V[2][4];
    static __device__ __forceinline__ void load_q(const char *row, int b, Q &q) {
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
            q[kk] = row ? __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(row + kk * 64 + b * 16)) : bf16x8{};
    }
    static __device__ __forceinline__ void load_k(const char *row, int b, uint4 (&k)[4]) {
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) k[kk] = *reinterpret_cast<const uint4 *>(row + kk * 64 + b * 16);
    }
    static __device__ __forceinline__ void load_v(const char *row, int i, uint4 &v) { v = *reinterpret_cast<const uint4 *>(row + i * 16); }
    static __device__ __forceinline__ void zero_v(uint4 &v) { v = make_uint4(0, 0, 0, 0); }
    static __device__ __forceinline__ bool odd_v(const uint4 &v) {   // an infinity or a NaN among the eight
        bool bad = false;
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int c = 0; c < 4; ++c) bad |= (w[c] & 0x7f80u) == 0x7f80u || (w[c] & 0x7f800000u) == 0x7f800000u;
        return bad;
    }
    static __device__ __forceinline__ f32x4 score(const uint4 (&k)[4], const Q &q) {
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
            s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[kk]), q[kk], s, 0, 0, 0);
        return s;
    }
    static __device__ __forceinline__ float element(const char *row, int c) { return lvr_bf16_lo(*reinterpret_cast<const uint16_t *>(row + c * 2)); }
    // o[u] += V^T P^T over the 32 keys; l += the weights as rounded, which is what the second product sees
    static __device__ __forceinline__ void add(const V &v, const float (&p)[2][4], f32x4 (&o)[8], float &l) {
        uint32_t pw[4] = {pack_bf16(p[0][0], p[0][1]), pack_bf16(p[0][2], p[0][3]), pack_bf16(p[1][0], p[1][1]), pack_bf16(p[1][2], p[1][3])};
#pragma unroll
        for (int c = 0; c < 4; ++c) l += lvr_bf16_lo(pw[c]) + lvr_bf16_hi(pw[c]);
        const bf16x8 pb = __builtin_bit_cast(bf16x8, make_uint4(pw[0], pw[1], pw[2], pw[3]));
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            uint32_t a[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint4 &v0 = v[c >> 1][(c & 1) * 2], &v1 = v[c >> 1][(c & 1) * 2 + 1];
                const uint32_t w0 = u < 2 ? v0.x : (u < 4 ? v0.y : (u < 6 ? v0.z : v0.w));
                const uint32_t w1 = u < 2 ? v1.x : (u < 4 ? v1.y : (u < 6 ? v1.z : v1.w));
                a[c] = __builtin_amdgcn_perm(w1, w0, (u & 1) ? 0x07060302u : 0x05040100u);
            }
            o[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, make_uint4(a[0], a[1], a[2], a[3])), pb, o[u], 0, 0, 0);
        }
    }
    static __device__ __forceinline__ int coordinate(int r, int u) { return 8 * r + u; }   // of row r of result tile u
};

template <>
struct Rows16<lvr_f32_t> {
    static constexpr int ELT = 4;
    struct Raw { float4 a, b; };
    typedef float4 Q[8];
    typedef float4 K[2][8];
    typedef Raw V[2][4];
    static __device__ __forceinline__ void load_q(const char *row, int b, Q &q) {
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) q[kk] = row ? *reinterpret_cast<const float4 *>(row + kk * 64 + b * 16) : make_float4(0, 0, 0, 0);
    }
    static __device__ __forceinline__ void load_k(const char *row, int b, float4 (&k)[8]) {
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) k[kk] = *reinterpret_cast<const float4 *>(row + kk * 64 + b * 16);
    }
    static __device__ __forceinline__ void load_v(const char *row, int i, Raw &v) {
        v.a = *reinterpret_cast<const float4 *>(row + i * 16);
        v.b = *reinterpret_cast<const float4 *>(row + 256 + i * 16);
    }
    static __device__ __forceinline__ void zero_v(Raw &v) { v.a = v.b = make_float4(0, 0, 0, 0); }
    static __device__ __forceinline__ bool odd_v(const Raw &v) {
        bool bad = false;
#pragma unroll
        for (int u = 0; u < 8; ++u) bad |= (__float_as_uint(value(v, u)) & 0x7f800000u) == 0x7f800000u;
        return bad;
    }
    static __device__ __forceinline__ f32x4 score(const float4 (&k)[8], const Q &q) {
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) {   // the order of the coordinates is the same on both sides, and free
            s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[kk].x, q[kk].x, s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[kk].y, q[kk].y, s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[kk].z, q[kk].z, s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[kk].w, q[kk].w, s, 0, 0, 0);
        }
        return s;
    }
    static __device__ __forceinline__ float element(const char *row, int c) { return *reinterpret_cast<const float *>(row + c * 4); }
    static __device__ __forceinline__ float value(const Raw &v, int u) {
        const float4 &h = u < 4 ? v.a : v.b;
        return (u & 3) == 0 ? h.x : ((u & 3) == 1 ? h.y : ((u & 3) == 2 ? h.z : h.w));
    }
    static __device__ __forceinline__ void add(const V &v, const float (&p)[2][4], f32x4 (&o)[8], float &l) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                l += p[h][j];
#pragma unroll
                for (int u = 0; u < 8; ++u) o[u] = __builtin_amdgcn_mfma_f32_16x16x4f32(value(v[h][j], u), p[h][j], o[u], 0, 0, 0);
            }
    }
    static __device__ __forceinline__ int coordinate(int r, int u) { return u < 4 ? 4 * r + u : 64 + 4 * r + u - 4; }
};

template <typename KT>
__global__ void __launch_bounds__(256) paged_attention_rows16_kernel(AttnArgs a, lvr_paged_batch bt) {
    typedef Rows16<KT> R;
    __shared__ float s_m[4][16], s_l[4][16];
    __shared__ float s_o[4][16][LVR_D + 4];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = lvr_lane(), i = lane & 15, b = lane >> 4;
    const int kvh = blockIdx.x % a.n_kv;
    Tile t;
    if (!find_tile<16>(bt, a.G, a.window, blockIdx.x / a.n_kv, t)) return;   // the whole workgroup

    const int row = t.row0 + i;                      // this lane's query row (column i of the score tiles)
    const int token = row / a.G, head = kvh * a.G + row - token * a.G;
    const bool has_row = row < t.rows;
    typename R::Q q;
    R::load_q(has_row ? a.q + (int64_t)(t.first_token + token) * a.q_stride + (int64_t)head * LVR_D * R::ELT : nullptr, b, q);
    const int last = t.pos0 + token;                 // keys this row sees: first .. last
    const int first = a.window && last - a.window + 1 > 0 ? last - a.window + 1 : 0;
    const int row_end = t.pos0 + t.row0 / a.G + 1;   // keys before it, from row_begin on, are seen by every row of the tile
    const int last_pos = t.pos0 + ((t.row0 + 15 < t.rows ? t.row0 + 15 : t.rows - 1) / a.G);
    const int row_begin = a.window && last_pos - a.window + 1 > 0 ? last_pos - a.window + 1 : 0;

    float m = -INFINITY, l = 0.f;
    f32x4 o[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) o[u] = f32x4{0.f, 0.f, 0.f, 0.f};

    for (int k0 = (t.lo & ~31) + wave * 32; k0 < t.hi; k0 += 128) {   // uniform over the wave
        typename R::K k;
        typename R::V v;
        const char *vp[2];
        bool none[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {   // 16 keys: one page
            const int kt = k0 + h * 16;
            const int page = kt < t.hi ? __builtin_amdgcn_readfirstlane(lvr_page_of(bt, t.seq, kt)) : -1;
            none[h] = page < 0;
            const int64_t at = lvr_row_at(bt, none[h] ? 0 : page, kvh, none[h] ? 0 : kt);   // no page: some memory of the pool
            const char *kp = a.k_pages + at;
            vp[h] = a.v_pages + at;
            R::load_k(kp + i * bt.row_stride, b, k[h]);
#pragma unroll
            for (int j = 0; j < 4; ++j) R::load_v(vp[h] + (4 * b + j) * bt.row_stride, i, v[h][j]);
        }
        const bool partly = k0 < row_begin || k0 + 32 > row_end || none[0] || none[1];
        float p[2][4];
        bool poison = false;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const f32x4 s = R::score(k[h], q);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                p[h][j] = s[j];
                if (partly) {
                    const int key = k0 + h * 16 + 4 * b + j;
                    if (none[h] || key < first || key > last) p[h][j] = -INFINITY;
                    // a row of V that no query row sees is memory nobody has written; one that some see meets the others with
                    // weight zero, which an infinity or a NaN would survive
                    if (none[h] || key < t.lo || key >= t.hi) R::zero_v(v[h][j]);
                    else if (R::odd_v(v[h][j])) poison = true;
                }
            }
        }
        float top = p[0][0];
#pragma unroll
        for (int c = 1; c < 8; ++c) top = fmaxf(top, p[c >> 2][c & 3]);
        top *= a.unit;
        if (__any(top > m + RAISE)) {
            float all = fmaxf(top, __shfl_xor(top, 16, 64));
            all = fmaxf(all, __shfl_xor(all, 32, 64));
            const float raised = fmaxf(m, all);
            const float scale = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - raised);
            m = raised;
            l *= scale;
#pragma unroll
            for (int u = 0; u < 8; ++u) o[u] *= scale;
        }
        const float base = m == -INFINITY ? 0.f : m;   // nothing seen so far: every weight below is 2^-inf
#pragma unroll
        for (int c = 0; c < 8; ++c) p[c >> 2][c & 3] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[c >> 2][c & 3], a.unit, -base));
        if (__any(poison)) {
            // rare: key by key on the vector units, so that a row that does not see a key does not meet its value
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    l += p[h][j];
                    for (int b2 = 0; b2 < 4; ++b2) {
                        const int key = k0 + h * 16 + 4 * b2 + j;
                        const float w = __shfl(p[h][j], i + 16 * b2, 64);
                        if (none[h] || key < first || key > last) continue;
                        const char *vr = vp[h] + (4 * b2 + j) * bt.row_stride;
#pragma unroll
                        for (int c = 0; c < 4; ++c)
#pragma unroll
                            for (int u = 0; u < 8; ++u) o[u][c] += w * R::element(vr, R::coordinate(4 * b + c, u));
                    }
                }
        } else {
            R::add(v, p, o, l);
        }
    }
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);

    // the four waves' (m, l, o) become the rows' outputs
    if (b == 0) {
        s_m[wave][i] = m;
        s_l[wave][i] = l;
    }
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int u = 0; u < 8; u += 4)
            *reinterpret_cast<float4 *>(&s_o[wave][i][R::coordinate(4 * b + c, u)]) = make_float4(o[u][c], o[u + 1][c], o[u + 2][c], o[u + 3][c]);
    __syncthreads();
    const int r = threadIdx.x >> 4, c0 = (threadIdx.x & 15) * 8;
    if (t.row0 + r >= t.rows) return;
    const float M = fmaxf(fmaxf(s_m[0][r], s_m[1][r]), fmaxf(s_m[2][r], s_m[3][r]));
    float sum = 0.f, x[8];
    lvr_zero8(x);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float scale = s_m[w][r] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_m[w][r] - M);
        if (scale == 0.f && s_l[w][r] == 0.f) continue;
        sum += scale * s_l[w][r];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] += scale * s_o[w][r][c0 + e];
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;   // nothing seen: zeros
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= inv;
    const int otok = (t.row0 + r) / a.G, ohead = kvh * a.G + t.row0 + r - otok * a.G;
    char *dst = a.out + (((int64_t)(t.first_token + otok) * a.n_kv * a.G + ohead) * LVR_D + c0) * R::ELT;
    if constexpr (R::ELT == 2) {
        *reinterpret_cast<uint4 *>(dst) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
    } else {
        *reinterpret_cast<float4 *>(dst) = make_float4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<float4 *>(dst + 16) = make_float4(x[4], x[5], x[6], x[7]);
    }
}

}  // namespace

hipError_t lvr_launch_paged_attention(lvr_paged *pc, const lvr_paged_batch &b, const void *k_pages, const void *v_pages, const void *q,
                                      int64_t q_stride_bytes, int32_t window, void *out, hipStream_t st) {
    AttnArgs a;
    a.k_pages = static_cast<const char *>(k_pages);
    a.v_pages = static_cast<const char *>(v_pages);
    a.q = static_cast<const char *>(q);
    a.out = static_cast<char *>(out);
    a.q_stride = q_stride_bytes;
    a.n_kv = pc->cfg.n_kv_heads;
    a.G = pc->cfg.n_q_heads / pc->cfg.n_kv_heads;
    a.window = window;
    a.unit = pc->sigma * LOG2E;
    const int64_t tiles = (int64_t)b.n_tokens * a.G / 16 + b.n_seqs;
    const dim3 grid((unsigned)(tiles * a.n_kv));
    if (pc->cfg.kv_dtype == LVR_BF16) hipLaunchKernelGGL(paged_attention_rows16_kernel<lvr_bf16_t>, grid, dim3(256), 0, st, a, b);
    else hipLaunchKernelGGL(paged_attention_rows16_kernel<lvr_f32_t>, grid, dim3(256), 0, st, a, b);
    return hipGetLastError();
}
