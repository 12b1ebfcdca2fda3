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
#include "paged_division.h"

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float RAISE = 8.f;
constexpr int MERGE_WGS = 1024;
constexpr int FAN_BITS = 3, FAN = 1 << FAN_BITS;   // partial results of 16-row tiles that a wave merges at a time

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 v = {(__bf16)lo, (__bf16)hi};   // rounds to nearest even, NaN stays NaN
    return __builtin_bit_cast(uint32_t, v);
}

template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_or_zero(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float wave_sum(float v) {   // as lvr_wave_inclusive_sum; every lane gets the total
    v += dpp_or_zero<0x111, 0xf>(v);
    v += dpp_or_zero<0x112, 0xf>(v);
    v += dpp_or_zero<0x114, 0xf>(v);
    v += dpp_or_zero<0x118, 0xf>(v);
    v += dpp_or_zero<0x142, 0xa>(v);
    v += dpp_or_zero<0x143, 0xc>(v);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// What the division asks of a wave.
struct Wave {
    static constexpr int LANES = 64;
    static __device__ __forceinline__ int lane() { return lvr_lane(); }
    static __device__ __forceinline__ bool any(bool v) { return __any(v); }
    static __device__ __forceinline__ uint64_t ballot(bool v) { return __ballot(v); }
    static __device__ __forceinline__ float sum(float v) { return wave_sum(v); }
    static __device__ __forceinline__ int inclusive_sum(int v) { return lvr_wave_inclusive_sum(v); }
    static __device__ __forceinline__ int of(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
    static __device__ __forceinline__ float of_first(float v) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v))); }
    static __device__ __forceinline__ float reciprocal(float v) { return __builtin_amdgcn_rcpf(v); }
};

// Partial results of pieces of cut tiles of HEIGHT rows: per slot and KV head HEIGHT rows of 128 sums, then HEIGHT pairs of maximum
// and weight.  Those of 128-row tiles first.
template <int HEIGHT>
__device__ __forceinline__ float *partial(float *part, int slot, int n_kv, int kvh) {
    if (HEIGHT == 16) part += (int64_t)WIDE_ROOM * 128 * (LVR_D + 2);
    return part + ((int64_t)slot * n_kv + kvh) * (HEIGHT * (LVR_D + 2));
}

// Sums over several sets of keys, brought to a common maximum.
struct Merged {
    float m, l, o[8];
    __device__ __forceinline__ void clear() {
        m = -INFINITY;
        l = 0.f;
        lvr_zero8(o);
    }
    __device__ __forceinline__ void add(float m2, float l2, const float (&v)[8]) {
        const float raised = fmaxf(m, m2);
        const float old = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - raised);
        const float scale = m2 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m2 - raised);   // nothing seen there: all of it is zero
        m = raised;
        l = l * old + scale * l2;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = o[e] * old + scale * v[e];
    }
};
__device__ __forceinline__ void store_shared(float *p, float2 v) {
    __hip_atomic_store(reinterpret_cast<uint64_t *>(p), __builtin_bit_cast(uint64_t, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 load_shared(const float *p) {
    return __builtin_bit_cast(float2, __hip_atomic_load(reinterpret_cast<const uint64_t *>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// Where a packed row's output lies.
template <int ELT>
__device__ __forceinline__ char *output_row(const AttnArgs &a, const Tile &t, int kvh, int row) {
    const int token = token_of(a, row), head = kvh * a.G + row - token * a.G;
    return a.out + ((int64_t)(t.first_token + token) * a.n_kv * a.G + head) * LVR_D * ELT;
}
template <int ELT>
__device__ __forceinline__ void store_row(const AttnArgs &a, const Tile &t, int kvh, int row, int c0, const float (&y)[8]) {
    char *dst = output_row<ELT>(a, t, kvh, row) + c0 * ELT;
    if constexpr (ELT == 2) {
        *reinterpret_cast<uint4 *>(dst) = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
    } else {
        *reinterpret_cast<float4 *>(dst) = make_float4(y[0], y[1], y[2], y[3]);
        *reinterpret_cast<float4 *>(dst + 16) = make_float4(y[4], y[5], y[6], y[7]);
    }
}

// One query row over the keys k0 .. k0 + run - 1, then `step` further on, and so on before `end`, on the vector units: two coordinates a lane.
// For rows whose neighbours in a tile do not see a value that is infinite or no number: in a matrix product it would reach them
// with weight zero.
struct RowSum {
    float m, l, o0, o1;
};
template <int ELT>
__device__ __noinline__ RowSum one_row(AttnArgs a, lvr_paged_batch bt, Tile t, int kvh, int row, int k0, int run, int step) {
    const int lane = lvr_lane(), token = token_of(a, row), head = kvh * a.G + row - token * a.G;
    const int last = t.pos0 + token, first = a.window && last - a.window + 1 > 0 ? last - a.window + 1 : 0;
    auto pair = [&](const char *r) {
        if constexpr (ELT == 2) {
            const uint32_t w = *reinterpret_cast<const uint32_t *>(r + lane * 4);
            return make_float2(lvr_bf16_lo(w), lvr_bf16_hi(w));
        } else {
            return *reinterpret_cast<const float2 *>(r + lane * 8);
        }
    };
    const float2 q = pair(a.q + (int64_t)(t.first_token + token) * a.q_stride + (int64_t)head * LVR_D * ELT);
    RowSum s = {-INFINITY, 0.f, 0.f, 0.f};
    for (; k0 < t.end; k0 += step)
        for (int key = k0; key < k0 + run && key < t.end; ++key) {
            const int page = key < first || key > last ? -1 : lvr_page_of(bt, t.seq, key);
            if (page < 0) continue;
            const int64_t at = lvr_row_at(bt, page, kvh, key);
            const float2 k = pair(a.k_pages + at), v = pair(a.v_pages + at);
            const float x = wave_sum(q.x * k.x + q.y * k.y) * a.unit;
            const float raised = fmaxf(s.m, x);
            const float old = s.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s.m - raised);
            const float w = __builtin_amdgcn_exp2f(x - (raised == -INFINITY ? 0.f : raised));
            s.m = raised;
            s.l = s.l * old + w;
            s.o0 = s.o0 * old + w * v.x;
            s.o1 = s.o1 * old + w * v.y;
        }
    return s;
}

// ---------------------------------------------------------------------------------------------------------------------------
// 16 rows to a tile.  A workgroup of four waves; a wave takes 32 keys at a time straight into registers.
//
// Matrix operand lanes: i = lane & 15, b = lane >> 4.  A score tile is 16 keys: row r = 4 b + j of the result is register j of
// lanes (., b), the column i is the query row.  As the second product's operand those scores are the keys that lanes (., b)
// contribute, so key r of the tile is held as V row 4 b + j by the lanes that load it: a row is read whole by 16 lanes, eight
// coordinates each, and which coordinates share a result tile is free as well (tile u: coordinates 8 i + u).
// bf16: two score tiles make one operand of 32 keys; a pair of V rows is woven into it by byte permutes.
//
// Bound by the read of K and V: 131072 keys of one sequence 99 us, 48 ragged sequences of up to 32768 keys 362 us (1.97 GB), both 5.4 TB/s.
// Short contexts are bound by dependent trips (lengths, table, rows, products, partial results): 2048 keys 10 us, in runs of 64 keys, for which two of the
// four waves have none.  Rows asked for a turn ahead: no gain, and fp32 spills; eight waves to a workgroup: 12.1 us at 2048 keys where four took 11.3.
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
    // o[u] += V^T P^T over the 32 keys.  The weights are rounded to bf16, as the matrix instruction takes them beside V (a weight off by up to 2^-8 of
    // itself; with it outputs are off by 1.9e-3 to 2.4e-3 of their root mean square, 1.6e-3 with fp32 weights, most of both the last rounding); l sums
    // them as rounded, which is what the second product sees.
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

struct Rows16Lds {
    float m[4][16], l[4][16];
    float o[4][16][LVR_D + 4];
    unsigned arrived;
};

template <typename KT>
__device__ __forceinline__ void rows16_piece(const AttnArgs &a, const lvr_paged_batch &bt, const Tile &t, int kvh, Rows16Lds &lds) {
    typedef Rows16<KT> R;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = lvr_lane(), i = lane & 15, b = lane >> 4;

    const int row = t.row0 + i;                      // this lane's query row (column i of the score tiles)
    const int token = token_of(a, row), head = kvh * a.G + row - token * a.G;
    const bool has_row = row < t.rows;
    typename R::Q q;
    R::load_q(has_row ? a.q + (int64_t)(t.first_token + token) * a.q_stride + (int64_t)head * LVR_D * R::ELT : nullptr, b, q);
    const int last = t.pos0 + token;                 // keys this row sees: first .. last
    const int first = a.window && last - a.window + 1 > 0 ? last - a.window + 1 : 0;
    const int row_end = t.pos0 + token_of(a, t.row0) + 1;   // keys before it, from row_begin on, are seen by every row of the tile
    const int last_pos = t.pos0 + token_of(a, t.row0 + 15 < t.rows ? t.row0 + 15 : t.rows - 1);
    const int row_begin = a.window && last_pos - a.window + 1 > 0 ? last_pos - a.window + 1 : 0;

    bool redo = false;
    float m = -INFINITY, l = 0.f;
    f32x4 o[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) o[u] = f32x4{0.f, 0.f, 0.f, 0.f};

    for (int k0 = t.begin + wave * 32; k0 < t.end; k0 += 128) {   // uniform over the wave
        typename R::K k;
        typename R::V v;
        bool none[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {   // 16 keys: one page
            const int kt = k0 + h * 16;
            const int page = kt < t.hi ? __builtin_amdgcn_readfirstlane(lvr_page_of(bt, t.seq, kt)) : -1;
            none[h] = page < 0;
            const int64_t at = lvr_row_at(bt, none[h] ? 0 : page, kvh, none[h] ? 0 : kt);   // no page: some memory of the pool
            const char *kp = a.k_pages + at, *vp = a.v_pages + at;
            R::load_k(kp + i * bt.row_stride, b, k[h]);
#pragma unroll
            for (int j = 0; j < 4; ++j) R::load_v(vp + (4 * b + j) * bt.row_stride, i, v[h][j]);
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
        redo |= poison;
        R::add(v, p, o, l);
    }
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);

    // the four waves' (m, l, o) become the rows' outputs
    if (__any(redo)) {
        for (int r = 0; r < 16 && t.row0 + r < t.rows; ++r) {
            const RowSum s = one_row<R::ELT>(a, bt, t, kvh, t.row0 + r, t.begin + wave * 32, 32, 128);
            lds.m[wave][r] = s.m;
            lds.l[wave][r] = s.l;
            lds.o[wave][r][2 * lane] = s.o0;
            lds.o[wave][r][2 * lane + 1] = s.o1;
        }
    } else {
        if (b == 0) {
            lds.m[wave][i] = m;
            lds.l[wave][i] = l;
        }
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int u = 0; u < 8; u += 4)
                *reinterpret_cast<float4 *>(&lds.o[wave][i][R::coordinate(4 * b + c, u)]) = make_float4(o[u][c], o[u + 1][c], o[u + 2][c], o[u + 3][c]);
    }
    __syncthreads();
    const int r = threadIdx.x >> 4, c0 = (threadIdx.x & 15) * 8;
    const bool writes = t.row0 + r < t.rows;
    Merged x;
    auto from_lds = [&](int n) {   // the sums of n sets of keys
        x.clear();
        for (int w = 0; w < n; ++w) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = lds.o[w][r][c0 + e];
            x.add(lds.m[w][r], lds.l[w][r], v);
        }
    };
    from_lds(4);
    if (t.splits > 1) {
        // The last workgroup to end of every `fan` of a tile's runs merges those, and the last of these merges what they made, so that nobody
        // is left with all of them (one token over 8192 keys 13.1 us; all merged by one workgroup 15.2).  Four rows fill a wave, and where a tile has no
        // more the waves share the partials out; each takes up to FAN of them with all their loads in flight.  Partials cross
        // from one die to another: they are stored and read with accesses of device scope, and a workgroup waits for its own stores
        // before it takes a ticket, which wraps at the number of those who take it and so is zero again afterwards.
        const int rows = t.rows - t.row0, sharer_bits = rows <= 4 ? 2 : (rows <= 8 ? 1 : 0), sharers = 1 << sharer_bits, fan = FAN * sharers;
        const int slot0 = t.slot - t.split, fans = (t.splits + fan - 1) >> (FAN_BITS + sharer_bits), mine = t.split >> (FAN_BITS + sharer_bits);
        const int in_mine = mine + 1 < fans ? fan : t.splits - mine * fan;
        float *first_part = partial<16>(a.part, slot0, a.n_kv, kvh);
        const int64_t step = (int64_t)a.n_kv * (16 * (LVR_D + 2));
        auto put = [&](float *p) {
            if (!writes) return;
#pragma unroll
            for (int e = 0; e < 8; e += 2) store_shared(p + r * LVR_D + c0 + e, make_float2(x.o[e], x.o[e + 1]));
            if (c0 == 0) store_shared(p + 16 * LVR_D + r * 2, make_float2(x.m, x.l));
        };
        auto last_of = [&](int slot, int word, int n) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (threadIdx.x == 0) lds.arrived = atomicInc(a.ticket + ((int64_t)slot * a.n_kv + kvh) * LVR_CNT_STRIDE + word, (unsigned)n - 1u);
            __syncthreads();
            return lds.arrived == (unsigned)n - 1u;
        };
        auto merge = [&](const float *p, int64_t apart, int n) {
            const int share = wave >> (2 - sharer_bits), mr = (wave & ((4 >> sharer_bits) - 1)) * 4 + (lane >> 4);   // whose turn, which row
            x.clear();
            for (int p0 = share; p0 < n; p0 += fan) {
                float2 ml[FAN], v[FAN][4];
#pragma unroll
                for (int k = 0; k < FAN; ++k) {   // past the last one the last once more
                    const float *from = p + (p0 + k * sharers < n ? p0 + k * sharers : n - 1) * apart;
                    ml[k] = load_shared(from + 16 * LVR_D + mr * 2);
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[k][e] = load_shared(from + mr * LVR_D + c0 + 2 * e);
                }
#pragma unroll
                for (int k = 0; k < FAN; ++k) {
                    if (p0 + k * sharers >= n || mr >= rows) continue;   // (rows that are none hold anything)
                    const float y[8] = {v[k][0].x, v[k][0].y, v[k][1].x, v[k][1].y, v[k][2].x, v[k][2].y, v[k][3].x, v[k][3].y};
                    x.add(ml[k].x, ml[k].y, y);
                }
            }
            if (sharers == 1) return;
            if (c0 == 0) {
                lds.m[share][mr] = x.m;
                lds.l[share][mr] = x.l;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) lds.o[share][mr][c0 + e] = x.o[e];
            __syncthreads();
            from_lds(sharers);
        };
        put(first_part + t.split * step);
        if (!last_of(slot0 + mine * fan, 0, in_mine)) return;
        merge(first_part + mine * fan * step, step, in_mine);
        if (fans > 1) {
            put(first_part + mine * fan * step);
            if (!last_of(slot0, 1, fans)) return;
            merge(first_part, fan * step, fans);
        }
    }
    if (!writes) return;
    const float inv = x.l == 0.f ? 0.f : 1.f / x.l;   // nothing seen: zeros
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = x.o[e] * inv;
    store_row<R::ELT>(a, t, kvh, t.row0 + r, c0, y);
}

// ---------------------------------------------------------------------------------------------------------------------------
// 128 rows to a tile, 32 to each of four waves.  K and V tiles pass through LDS, two of each: while one is worked on the next is on
// its way, past the registers.
//
// Matrix operand lanes: n = lane & 31 (query row), h = lane >> 5.  Score tile: 32 keys, result row 8 i + 4 h + j is register 4 i + j.
// bf16 (tiles of 64 keys): registers 8 t .. 8 t + 7 of a score tile are at once the second product's operand for 16 keys, of which lanes
// (., h) contribute 8 h .. 8 h + 7; for that K row 16 (i / 2) + 8 h + 4 (i % 2) + j is stored as row 8 i + 4 h + j.  V is
// read transposed (four keys of one coordinate per lane and read).
// fp32 (tiles of 32 keys): register r is the operand for the keys 8 i + 4 h + j themselves, and a lane's 16-byte read of V holds
// the coordinates 4 n .. 4 n + 3, one for each of four result tiles.
// 16-byte pieces of a row are stored at their number xor something of the row's, so that rows do not meet in the same banks (bf16: no bank
// conflicts counted; fp32, whose V rows lie as they are: conflicts in 13 % of the clocks that LDS works).
//
// 32 rows to a wave and two workgroups to a compute unit: 128 KiB of LDS and up to 256 registers a lane, so that one workgroup's matrix
// instructions meet the other's exponentials.  A prompt of 16384 tokens (32 heads on 8, 2.2 TFLOP): 2.1 to 2.25 ms on different cards, 980 to
// 1050 TFLOP/s; matrix units busy 46 % and vector units 42 % of the clocks, where the library's product of 8192 x 8192 matrices reaches
// 1148 TFLOP/s.  fp32, 8192 tokens: 134 TFLOP/s of the 154 the library reaches.  Tried without gain: the scores of the next tile made
// between the exponentials of this one (-2 %), wave priorities around the products, tiles through registers (653 TFLOP/s: the loads were
// waited for at once).
// ---------------------------------------------------------------------------------------------------------------------------
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <typename KT>
struct Rows128;

template <>
struct Rows128<lvr_bf16_t> {
    static constexpr int ELT = 2, ROWB = 256, TK = 64, NT = 2, PIECES = 16;
    typedef bf16x8 Q[8];
    static __device__ __forceinline__ void load_q(const char *row, int h, Q &q) {
#pragma unroll
        for (int s = 0; s < 8; ++s)
            q[s] = row ? __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(row + (2 * s + h) * 16)) : bf16x8{};
    }
    static __device__ __forceinline__ int key_of_k_row(int r) { return (r & 35) | ((r & 16) ? 16 : 0) | ((r & 4) << 1) | ((r & 8) >> 1); }
    static __device__ __forceinline__ int k_piece(int r, int c) { return c ^ (r & 15); }
    static __device__ __forceinline__ int v_piece(int key, int c) { return c ^ ((key & 3) << 2); }
    static __device__ __forceinline__ int key_of(int h, int kt, int r) { return 32 * kt + 16 * (r >> 3) + 8 * h + (r & 7); }
    static __device__ __forceinline__ int coordinate(int h, int dt, int r) { return 32 * dt + 8 * (r >> 2) + 4 * h + (r & 3); }
    static __device__ __forceinline__ void scores(const char *k, const Q &q, int n, int h, f32x16 (&s)[NT]) {
#pragma unroll
        for (int kt = 0; kt < NT; ++kt) {
            f32x16 c = {0.f};
            const char *row = k + (kt * 32 + n) * ROWB;
#pragma unroll
            for (int st = 0; st < 8; ++st) {
                const bf16x8 a = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(row + k_piece(n, 2 * st + h) * 16));
                c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, q[st], c, 0, 0, 0);
            }
            s[kt] = c;
        }
    }
    static __device__ __forceinline__ void add(const char *v, const f32x16 (&p)[NT], int lane, f32x16 (&o)[4], float &l) {
        const int i16 = lane & 15, key = (lane >> 5) * 8 + (i16 >> 2);
        const char *at = v + key * ROWB + (i16 & 1) * 8;
        const int piece = ((lane >> 4) & 1) * 2 + ((i16 & 3) >> 1);
#pragma unroll
        for (int kt = 0; kt < NT; ++kt)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                uint32_t w[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    w[c] = pack_bf16(p[kt][8 * t + 2 * c], p[kt][8 * t + 2 * c + 1]);
                    l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w[c]), bf16x2{(__bf16)1.f, (__bf16)1.f}, l, false);
                }
                const bf16x8 pb = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
#pragma unroll
                for (int dt = 0; dt < 4; ++dt) {
                    const char *src = at + (32 * kt + 16 * t) * ROWB + v_piece(key, dt * 4 + piece) * 16;
                    typedef __attribute__((address_space(3))) s16x4 *Lds;
                    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(src));
                    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(src + 4 * ROWB));
                    const bf16x8 a = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                    o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pb, o[dt], 0, 0, 0);
                }
            }
    }
    static __device__ __forceinline__ bool odd(const uint4 &v) { return Rows16<lvr_bf16_t>::odd_v(v); }
};

template <>
struct Rows128<lvr_f32_t> {
    static constexpr int ELT = 4, ROWB = 512, TK = 32, NT = 1, PIECES = 32;
    typedef float4 Q[16];
    static __device__ __forceinline__ void load_q(const char *row, int h, Q &q) {
#pragma unroll
        for (int s = 0; s < 16; ++s) q[s] = row ? *reinterpret_cast<const float4 *>(row + (2 * s + h) * 16) : make_float4(0, 0, 0, 0);
    }
    static __device__ __forceinline__ int key_of_k_row(int r) { return r; }
    static __device__ __forceinline__ int k_piece(int r, int c) { return c ^ (r & 31); }
    static __device__ __forceinline__ int v_piece(int, int c) { return c; }
    static __device__ __forceinline__ int key_of(int h, int, int r) { return 8 * (r >> 2) + 4 * h + (r & 3); }
    static __device__ __forceinline__ int coordinate(int h, int dt, int r) { return 4 * (8 * (r >> 2) + 4 * h + (r & 3)) + dt; }
    static __device__ __forceinline__ void scores(const char *k, const Q &q, int n, int h, f32x16 (&s)[NT]) {
        f32x16 c = {0.f};
        const char *row = k + n * ROWB;
#pragma unroll
        for (int st = 0; st < 16; ++st) {
            const float4 a = *reinterpret_cast<const float4 *>(row + k_piece(n, 2 * st + h) * 16);
            c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x, q[st].x, c, 0, 0, 0);
            c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.y, q[st].y, c, 0, 0, 0);
            c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.z, q[st].z, c, 0, 0, 0);
            c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.w, q[st].w, c, 0, 0, 0);
        }
        s[0] = c;
    }
    static __device__ __forceinline__ void add(const char *v, const f32x16 (&p)[NT], int lane, f32x16 (&o)[4], float &l) {
        const int n = lane & 31, h = lane >> 5;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            l += p[0][r];
            const float4 a = *reinterpret_cast<const float4 *>(v + key_of(h, 0, r) * ROWB + n * 16);
            o[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x, p[0][r], o[0], 0, 0, 0);
            o[1] = __builtin_amdgcn_mfma_f32_32x32x2f32(a.y, p[0][r], o[1], 0, 0, 0);
            o[2] = __builtin_amdgcn_mfma_f32_32x32x2f32(a.z, p[0][r], o[2], 0, 0, 0);
            o[3] = __builtin_amdgcn_mfma_f32_32x32x2f32(a.w, p[0][r], o[3], 0, 0, 0);
        }
    }
    static __device__ __forceinline__ bool odd(const uint4 &v) {
        return (v.x & 0x7f800000u) == 0x7f800000u || (v.y & 0x7f800000u) == 0x7f800000u || (v.z & 0x7f800000u) == 0x7f800000u ||
               (v.w & 0x7f800000u) == 0x7f800000u;
    }
};

// 16 bytes per lane from global memory into LDS, the wave's 1 KiB in a row from `to` on.  vmcnt counts it.
__device__ __forceinline__ void load_to_lds(const char *from, uint32_t offset, char *to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t *)(from + offset),
                                     (__attribute__((address_space(3))) uint32_t *)to, 16, 0, 0);
}

template <typename KT>
struct Rows128Lds {
    __align__(16) char k[2][Rows128<KT>::TK * Rows128<KT>::ROWB], v[2][Rows128<KT>::TK * Rows128<KT>::ROWB];
};

template <typename KT>
__device__ __forceinline__ void rows128_piece(const AttnArgs &a, const lvr_paged_batch &bt, const Tile &t, int kvh, Rows128Lds<KT> &lds) {
    typedef Rows128<KT> R;
    constexpr int TK = R::TK, LPR = R::PIECES, RPI = 64 / LPR;   // lanes to a row, rows to a load of the wave
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = lvr_lane(), n = lane & 31, h = lane >> 5;

    const int row0 = t.row0 + wave * 32, row = row0 + n;
    const int token = token_of(a, row), head = kvh * a.G + row - token * a.G;
    const bool has_row = row < t.rows;
    typename R::Q q;
    R::load_q(has_row ? a.q + (int64_t)(t.first_token + token) * a.q_stride + (int64_t)head * LVR_D * R::ELT : nullptr, h, q);
    const int last = t.pos0 + token;                 // keys this row sees: first .. last
    const int first = a.window && last - a.window + 1 > 0 ? last - a.window + 1 : 0;
    // some of the wave's rows see wlo .. whi - 1, all of them all_lo .. all_hi - 1
    const int wfirst = t.pos0 + token_of(a, row0), wlast = t.pos0 + token_of(a, row0 + 31 < t.rows ? row0 + 31 : t.rows - 1);
    const int whi = row0 < t.rows ? wlast + 1 : 0, wlo = a.window ? wfirst - a.window + 1 : 0;
    const int all_hi = wfirst + 1, all_lo = a.window ? wlast - a.window + 1 : 0;

    bool redo = false;   // a value that some rows must not meet
    float m = -INFINITY, l = 0.f;
    f32x16 o[4];
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) o[dt] = f32x16{0.f};

    // A wave brings four loads' worth of rows of K and of V, which lie in one page; each lane's place within the page's 16 rows
    // stays the same.  The lanes look up the pages of all groups of 16 keys of a tile at once, a tile ahead of the rows.
    const int srow = wave * 4 * RPI + lane / LPR, piece = lane % LPR, group = wave * 4 * RPI & ~15;
    uint32_t k_off[4], v_off[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = srow + i * RPI;
        k_off[i] = (uint32_t)(R::key_of_k_row(r) - group) * (uint32_t)bt.row_stride + R::k_piece(r, piece) * 16;
        v_off[i] = (uint32_t)(r - group) * (uint32_t)bt.row_stride + R::v_piece(r, piece) * 16;
    }
    auto pages_of = [&](int k0) {
        const int key = k0 + 16 * (lane % (TK / 16));
        return key < t.hi ? lvr_page_of(bt, t.seq, key) : -1;
    };
    auto load = [&](int k0, int pages, int buf) {
        const int page = __builtin_amdgcn_readlane(pages, group / 16);
        const int64_t at = page < 0 ? kvh * bt.head_stride : lvr_row_at(bt, page, kvh, k0 + group);   // no page: some memory of the pool
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            load_to_lds(a.k_pages + at, k_off[i], lds.k[buf] + (wave * 4 + i) * 1024);
            load_to_lds(a.v_pages + at, v_off[i], lds.v[buf] + (wave * 4 + i) * 1024);
        }
        return (uint32_t)__ballot(pages < 0) & ((1u << TK / 16) - 1u);   // groups without a page
    };
    auto arrived = [] {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    int buf = 0;
    uint32_t none = 0, next_none = 0;
    if (t.begin < t.end) none = load(t.begin, pages_of(t.begin), 0);
    int pages = pages_of(t.begin + TK);
    arrived();
    for (int k0 = t.begin; k0 < t.end; k0 += TK, buf ^= 1, none = next_none) {   // uniform over the workgroup
        if (k0 + TK < t.end) {
            next_none = load(k0 + TK, pages, buf ^ 1);
            pages = pages_of(k0 + 2 * TK);
        }
        if (k0 < t.lo || k0 + TK > t.hi || none != 0) {   // a row of V that no query row sees may be memory nobody has written
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key = srow + i * RPI;
                if (k0 + key < t.lo || k0 + key >= t.hi || (none >> (key >> 4) & 1))
                    *reinterpret_cast<uint4 *>(lds.v[buf] + key * R::ROWB + piece * 16) = make_uint4(0, 0, 0, 0);
            }
            arrived();
        }
        if (k0 < whi && k0 + TK > wlo) {
            f32x16 p[R::NT];
            R::scores(lds.k[buf], q, n, h, p);
            const bool partly = k0 < all_lo || k0 + TK > all_hi || none != 0;
            if (partly) {
                asm volatile("");   // a branch, not 32 selects in every tile
#pragma unroll 1
                for (int c = 0; c < TK * R::ROWB / 1024; ++c) redo |= R::odd(*reinterpret_cast<const uint4 *>(lds.v[buf] + c * 1024 + lane * 16));
#pragma unroll
                for (int kt = 0; kt < R::NT; ++kt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int key = R::key_of(h, kt, r);
                        if (k0 + key < first || k0 + key > last || (none >> (key >> 4) & 1)) p[kt][r] = -INFINITY;
                    }
            }
            float top = p[0][0];
#pragma unroll
            for (int kt = 0; kt < R::NT; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) top = fmaxf(top, p[kt][r]);
            top *= a.unit;
            if (__any(top > m + RAISE)) {
                const float raised = fmaxf(m, fmaxf(top, __shfl_xor(top, 32, 64)));
                const float scale = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - raised);
                m = raised;
                l *= scale;
#pragma unroll
                for (int dt = 0; dt < 4; ++dt) o[dt] *= scale;
            }
            const float base = m == -INFINITY ? 0.f : m;   // nothing seen so far: every weight below is 2^-inf
#pragma unroll
            for (int kt = 0; kt < R::NT; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) p[kt][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[kt][r], a.unit, -base));
            R::add(lds.v[buf], p, lane, o, l);
        }
        arrived();
    }
    l += __shfl_xor(l, 32, 64);
    if (__any(redo)) {
        for (int r = row0; r < row0 + 32 && r < t.rows; ++r) {
            RowSum s = one_row<R::ELT>(a, bt, t, kvh, r, t.begin, 1 << 30, 1 << 30);
            if (t.splits > 1) {
                float *mine = partial<128>(a.part, t.slot, a.n_kv, kvh);
                *reinterpret_cast<float2 *>(mine + (r - t.row0) * LVR_D + 2 * lane) = make_float2(s.o0, s.o1);
                *reinterpret_cast<float2 *>(mine + 128 * LVR_D + (r - t.row0) * 2) = make_float2(s.m, s.l);
                continue;
            }
            const float inv = s.l == 0.f ? 0.f : 1.f / s.l;
            char *dst = output_row<R::ELT>(a, t, kvh, r);
            if constexpr (R::ELT == 2) *reinterpret_cast<uint32_t *>(dst + lane * 4) = pack_bf16(s.o0 * inv, s.o1 * inv);
            else *reinterpret_cast<float2 *>(dst + lane * 8) = make_float2(s.o0 * inv, s.o1 * inv);
        }
        return;
    }
    if (!has_row) return;
    if (t.splits > 1) {
        float *mine = partial<128>(a.part, t.slot, a.n_kv, kvh) + (wave * 32 + n) * LVR_D;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float4 v = R::ELT == 2 ? make_float4(o[i >> 2][(i & 3) * 4], o[i >> 2][(i & 3) * 4 + 1], o[i >> 2][(i & 3) * 4 + 2], o[i >> 2][(i & 3) * 4 + 3])
                                         : make_float4(o[0][i], o[1][i], o[2][i], o[3][i]);
            *reinterpret_cast<float4 *>(mine + (R::ELT == 2 ? R::coordinate(h, i >> 2, (i & 3) * 4) : R::coordinate(h, 0, i))) = v;
        }
        if (h == 0) *reinterpret_cast<float2 *>(partial<128>(a.part, t.slot, a.n_kv, kvh) + 128 * LVR_D + (wave * 32 + n) * 2) = make_float2(m, l);
        return;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;   // nothing seen: zeros
    char *dst = output_row<R::ELT>(a, t, kvh, row);
    if constexpr (R::ELT == 2) {
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *reinterpret_cast<uint2 *>(dst + R::coordinate(h, dt, r) * 2) =
                    make_uint2(pack_bf16(o[dt][r] * inv, o[dt][r + 1] * inv), pack_bf16(o[dt][r + 2] * inv, o[dt][r + 3] * inv));
    } else {
#pragma unroll
        for (int r = 0; r < 16; ++r)
            *reinterpret_cast<float4 *>(dst + R::coordinate(h, 0, r) * 4) = make_float4(o[0][r] * inv, o[1][r] * inv, o[2][r] * inv, o[3][r] * inv);
    }
}

// Launches are n_kv x pieces workgroups: those of a KV head follow each other on one die where there are eight of them (a die has its
// own cache, and workgroups go to the eight dies in turn).
constexpr int GRID_Y = 32768;
__device__ __forceinline__ int piece_of_block() { return blockIdx.z * GRID_Y + blockIdx.y; }
inline dim3 grid_of(int n_kv, int64_t pieces) {
    return dim3((unsigned)n_kv, (unsigned)(pieces < GRID_Y ? pieces : GRID_Y), (unsigned)((pieces + GRID_Y - 1) / GRID_Y));
}

// Tiles of 16 rows alone: batches in which every sequence brings a token or so.
template <typename KT>
__global__ void __launch_bounds__(256, 2) paged_attention_rows16_kernel(AttnArgs a, lvr_paged_batch bt) {
    __shared__ Rows16Lds lds;
    const int kvh = blockIdx.x;
    Tile t;
    Division<false, Wave> d(a, bt);
    if (d.divide(a.target) && d.template locate<false>(piece_of_block(), t)) rows16_piece<KT>(a, bt, t, kvh, lds);
}

// Any batch: every sequence in the tiles that suit it.
template <typename KT>
__global__ void __launch_bounds__(256, 2) paged_attention_mixed_kernel(AttnArgs a, lvr_paged_batch bt) {
    __shared__ union { Rows16Lds narrow; Rows128Lds<KT> wide; } lds;
    const int kvh = blockIdx.x;
    Tile t;
    Division<true, Wave> d(a, bt);
    if (!d.divide(a.target) || !d.template locate<false>(piece_of_block(), t)) return;
    if (t.height == 128) rows128_piece<KT>(a, bt, t, kvh, lds.wide);
    else rows16_piece<KT>(a, bt, t, kvh, lds.narrow);
}

// Merges the runs of cut 128-row tiles.  16 rows of a tile at a time, 16 lanes to a row; the workgroups share them out.  A launch of its own, unlike
// for tiles of 16 rows: a partial result of 128 rows is 66 KiB, and the last workgroup of a tile would read all of them alone.  Bound by that read:
// 512 partial results (34 MB) 10 us.
template <typename KT>
__global__ void __launch_bounds__(256) paged_attention_merge_kernel(AttnArgs a, lvr_paged_batch bt) {
    Division<true, Wave> d(a, bt);
    if (!d.divide(a.target)) return;
    const int c0 = (threadIdx.x & 15) * 8;
    const int64_t step = (int64_t)a.n_kv * (128 * (LVR_D + 2));
    for (int item = blockIdx.x;; item += gridDim.x) {
        const int kvh = item % a.n_kv, r = item / a.n_kv % 8 * 16 + (threadIdx.x >> 4);
        Tile t;
        if (!d.template locate<true>(item / a.n_kv / 8, t)) return;
        if (t.splits == 1 || t.row0 + r >= t.rows) continue;
        const float *first_part = partial<128>(a.part, t.slot, a.n_kv, kvh);
        Merged x;
        x.clear();
#pragma unroll 4
        for (int p = 0; p < t.splits; ++p) {
            const float2 ml = *reinterpret_cast<const float2 *>(first_part + p * step + 128 * LVR_D + r * 2);
            const float4 v0 = *reinterpret_cast<const float4 *>(first_part + p * step + r * LVR_D + c0);
            const float4 v1 = *reinterpret_cast<const float4 *>(first_part + p * step + r * LVR_D + c0 + 4);
            const float v[8] = {v0.x, v0.y, v0.z, v0.w, v1.x, v1.y, v1.z, v1.w};
            x.add(ml.x, ml.y, v);
        }
        const float inv = x.l == 0.f ? 0.f : 1.f / x.l;
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = x.o[e] * inv;
        store_row<sizeof(KT) == 4 ? 4 : 2>(a, t, kvh, t.row0 + r, c0, y);
    }
}

}  // namespace

size_t lvr_paged_partial_bytes() { return ((size_t)WIDE_ROOM * 128 + (size_t)NARROW_ROOM * 16) * (LVR_D + 2) * sizeof(float); }
size_t lvr_paged_ticket_bytes() { return (size_t)NARROW_ROOM * LVR_CNT_STRIDE * sizeof(uint32_t); }

hipError_t lvr_launch_paged_attention(lvr_paged *pc, const lvr_paged_batch &b, const void *k_pages, const void *v_pages, const void *q,
                                      int64_t q_stride_bytes, int32_t window, void *out, hipStream_t st) {
    AttnArgs a;
    a.k_pages = static_cast<const char *>(k_pages);
    a.v_pages = static_cast<const char *>(v_pages);
    a.q = static_cast<const char *>(q);
    a.out = static_cast<char *>(out);
    a.q_stride = q_stride_bytes;
    a.window = window < 1 << 30 ? window : 0;   // no sequence is longer
    a.unit = pc->sigma * LOG2E;
    a.part = pc->part;
    a.ticket = pc->ticket;
    const bool bf16 = pc->cfg.kv_dtype == LVR_BF16;
    const PagedLaunch launch = paged_launch(a, b, pc->cfg.n_q_heads, pc->cfg.n_kv_heads, bf16);
    const dim3 grid = grid_of(a.n_kv, launch.pieces);
    if (!launch.mixed) {
        if (bf16) hipLaunchKernelGGL(paged_attention_rows16_kernel<lvr_bf16_t>, grid, dim3(256), 0, st, a, b);
        else hipLaunchKernelGGL(paged_attention_rows16_kernel<lvr_f32_t>, grid, dim3(256), 0, st, a, b);
        return hipGetLastError();
    }
    if (bf16) hipLaunchKernelGGL(paged_attention_mixed_kernel<lvr_bf16_t>, grid, dim3(256), 0, st, a, b);
    else hipLaunchKernelGGL(paged_attention_mixed_kernel<lvr_f32_t>, grid, dim3(256), 0, st, a, b);
    if (a.target > 0) {
        const dim3 merge(MERGE_WGS);
        if (bf16) hipLaunchKernelGGL(paged_attention_merge_kernel<lvr_bf16_t>, merge, dim3(256), 0, st, a, b);
        else hipLaunchKernelGGL(paged_attention_merge_kernel<lvr_f32_t>, merge, dim3(256), 0, st, a, b);
    }
    return hipGetLastError();
}
