// Attention of new tokens over the pages (lvr_paged_attention, lvr_paged_sink_attention).
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
//
// Pages in 4 bits are read as they are, a code and its scale making a bf16 value exactly; from there on everything is as for bf16 pages.  (Matrix
// instructions that take the codes themselves would need weights in fewer bits than bf16, and add up with some 14 bits.)
//
// First keys that stay visible beside a window are the first places of what a tile sees, the window's follow them: nothing in between is read.
#include "paged_division.h"

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float RAISE = 8.f;
constexpr int MERGE_WGS = 1024;
constexpr int COMPUTE_UNITS = 256, IN_STEP_RUN = 1024;
constexpr int FAN_BITS = 3, FAN = 1 << FAN_BITS;   // partial results of 16-row tiles that a wave merges at a time

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
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

// Partial results of pieces of cut tiles: per slot and KV head 128 (or 16) rows of 128 sums, then as many pairs of maximum and weight.
// Those of 128-row tiles first.
__device__ __forceinline__ float *partial128(float *part, int slot, int n_kv, int kvh) { return part + ((int64_t)slot * n_kv + kvh) * (128 * (LVR_D + 2)); }

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

// One query row over the places k0 .. k0 + run - 1, then `step` further on, and so on before `end`, on the vector units: two coordinates a lane.
// For rows whose neighbours in a tile do not see a value that is infinite or no number: in a matrix product it would reach them
// with weight zero.
struct RowSum {
    float m, l, o0, o1;
};
// The key at a place, and whether a row that sees first .. last (and the first keys) sees it.
// SINKS: there may be first keys that stay visible; the rest is the same without them, and less.
template <bool SINKS>
__device__ __forceinline__ int key_at(const Tile &t, int place) { return SINKS ? place + (place >= t.fold ? t.shift : 0) : place; }
template <bool SINKS>
__device__ __forceinline__ bool hidden(const AttnArgs &a, int key, int first, int last) { return key > last || (key < first && !(SINKS && key < a.sinks)); }
// `size` keys from `key` on: all of them seen by rows that see at least first .. end - 1; one of them by none of the tile's rows.
template <bool SINKS>
__device__ __forceinline__ bool all_seen(const AttnArgs &a, int key, int size, int first, int end) {
    return key + size <= end && (key >= first || (SINKS && key + size <= a.sinks));
}

// KT: the type of the pages
template <typename KT, bool SINKS>
__device__ __noinline__ RowSum one_row(AttnArgs a, lvr_paged_batch bt, Tile t, int kvh, int row, int k0, int run, int step) {
    const int lane = lvr_lane(), token = token_of(a, row), head = kvh * a.G + row - token * a.G;
    const int last = t.pos0 + token, first = a.window && last - a.window + 1 > 0 ? last - a.window + 1 : 0;
    constexpr int ELT = sizeof(KT) == 4 ? 4 : 2;
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
        for (int place = k0; place < k0 + run && place < t.end; ++place) {
            const int key = key_at<SINKS>(t, place);
            const int page = hidden<SINKS>(a, key, first, last) ? -1 : lvr_page_of(bt, t.seq, key);
            if (page < 0) continue;
            const int64_t at = lvr_row_at(bt, page, kvh, key);
            float2 k, v;
            if constexpr (__is_same(KT, lvr_fp4_t)) {
                const int64_t sc = lvr_scales_at(bt, page, kvh, key) + lane / 16;
                auto two = [&](const char *pages) {
                    const auto x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((uint8_t)pages[at + lane], lvr_fp4_scale((uint8_t)pages[sc]), 0);
                    return make_float2((float)x[0], (float)x[1]);
                };
                k = two(a.k_pages), v = two(a.v_pages);
            } else {
                k = pair(a.k_pages + at), v = pair(a.v_pages + at);
            }
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
// Bound by the read of K and V: 131072 keys of one sequence 98 us, 48 ragged sequences of up to 32768 keys 361 us (1.97 GB), both 5.5 TB/s.
// Short contexts are bound by dependent trips (lengths, table, rows, products, partial results): 2048 keys 8.5 us, in runs of 64 keys, for which two
// of the four waves have none.  Rows asked for a turn ahead: no gain, and fp32 spills; eight waves to a workgroup: 12.1 us at 2048 keys where four
// took 11.3.  First keys: 24 sequences, 21 of them longer than a window of 4096 and four first keys, 89 us (387 MB, 4.3 TB/s): 560 pieces of 1018 to
// 1472 keys on 256 compute units, bound by the end of the last.
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

// Pages in 4 bits.  Lanes (i, b) hold block b of a key's row, 32 coordinates with one scale, and of V the eight coordinates that they hold in bf16;
// both become bf16 in registers, exactly.
//
// Bound by the read where a batch is even (5.6 TB/s): 131072 keys of one sequence 33 us (143 MB; the launch, the division and two merges take 8 of
// them), 48 ragged sequences of up to 32768 keys 111 us (522 MB, 4.7 TB/s: the pieces' starts and ends weigh four times as much as beside bf16 rows).
// 2048 keys 8.5 us as in bf16, by the same dependent trips.  Weights are rounded to bf16 as there: see Rows16<lvr_bf16_t>::add.
template <>
struct Rows16<lvr_fp4_t> {
    static constexpr int ELT = 2;
    struct Key { uint4 codes; uint32_t scale; };
    struct Values { uint32_t codes[4], scales; };   // eight coordinates of four keys; the scales of one of them
    typedef bf16x8 Q[4];
    typedef Key K[2];
    typedef Values V[2];
    static __device__ __forceinline__ void load_q(const char *row, int b, Q &q) {
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
            q[kk] = row ? __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(row + b * 64 + kk * 16)) : bf16x8{};
    }
    static __device__ __forceinline__ f32x4 score(const Key &k, const Q &q) {
        const float scale = lvr_fp4_scale(k.scale);
        const uint32_t w[4] = {k.codes.x, k.codes.y, k.codes.z, k.codes.w};
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lvr_fp4_values(w[kk], scale), q[kk], s, 0, 0, 0);
        return s;
    }
    // The four lanes of a quad, which hold coordinates of the same block, have the scales of a key each.
    template <int J>
    static __device__ __forceinline__ float scale_of(float own) {
        return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(own), J * 0x55, 0xf, 0xf, true));
    }
    static __device__ __forceinline__ uint32_t own_scale(const Values &v) { return v.scales >> (threadIdx.x & 12) * 2 & 255; }
    // Two coordinates of all eight keys at a time: what is widened is used at once.
    template <int M>
    static __device__ __forceinline__ void add_pair(const V &v, const float (&scale)[8], bf16x8 pb, f32x4 (&o)[8]) {
        uint32_t w[8], lo[4], hi[4];
#pragma unroll
        for (int c = 0; c < 8; ++c) w[c] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v[c >> 2].codes[c & 3], scale[c], M));
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            lo[c] = __builtin_amdgcn_perm(w[2 * c + 1], w[2 * c], 0x05040100u);
            hi[c] = __builtin_amdgcn_perm(w[2 * c + 1], w[2 * c], 0x07060302u);
        }
        o[2 * M] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, make_uint4(lo[0], lo[1], lo[2], lo[3])), pb, o[2 * M], 0, 0, 0);
        o[2 * M + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, make_uint4(hi[0], hi[1], hi[2], hi[3])), pb, o[2 * M + 1], 0, 0, 0);
    }
    static __device__ __forceinline__ void add(const V &v, const float (&p)[2][4], f32x4 (&o)[8], float &l) {
        float scale[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float own = lvr_fp4_scale(own_scale(v[h]));
            scale[4 * h] = scale_of<0>(own);
            scale[4 * h + 1] = scale_of<1>(own);
            scale[4 * h + 2] = scale_of<2>(own);
            scale[4 * h + 3] = scale_of<3>(own);
        }
        const uint32_t pw[4] = {pack_bf16(p[0][0], p[0][1]), pack_bf16(p[0][2], p[0][3]), pack_bf16(p[1][0], p[1][1]), pack_bf16(p[1][2], p[1][3])};
#pragma unroll
        for (int c = 0; c < 4; ++c) l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pw[c]), bf16x2{(__bf16)1.f, (__bf16)1.f}, l, false);
        const bf16x8 pb = __builtin_bit_cast(bf16x8, make_uint4(pw[0], pw[1], pw[2], pw[3]));
        add_pair<0>(v, scale, pb, o);
        add_pair<1>(v, scale, pb, o);
        add_pair<2>(v, scale, pb, o);
        add_pair<3>(v, scale, pb, o);
    }
    static __device__ __forceinline__ int coordinate(int r, int u) { return Rows16<lvr_bf16_t>::coordinate(r, u); }
};

struct Rows16Lds {
    float m[4][16], l[4][16];
    float o[4][16][LVR_D + 4];
    unsigned arrived;
};

// ALONE: there are tiles of 16 rows alone
template <typename KT, bool SINKS, bool ALONE>
__device__ __forceinline__ void rows16_piece(const AttnArgs &a, const lvr_paged_batch &bt, const Tile &t, int kvh, Rows16Lds &lds) {
    typedef Rows16<KT> R;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = lvr_lane(), i = lane & 15, b = lane >> 4;

    const int q_row = t.row0 + i;                    // this lane's query row (column i of the score tiles)
    const int token = token_of(a, q_row), head = kvh * a.G + q_row - token * a.G;
    const bool has_row = q_row < t.rows;
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

    struct Keys {   // 32 of them on their way
        typename R::K k;
        typename R::V v;
        bool none[2];
    };
    constexpr bool FP4 = __is_same(KT, lvr_fp4_t);
    static_assert(LVR_FP4_CODES / LVR_FP4_SCALES == 16, "");
    const uint32_t row = (uint32_t)bt.row_stride;
    uint32_t k_place = i * row + b * 16, k_scale = i * (row / 16) + b, v_place[4], v_scales = (4 * b + (i & 3)) * (row / 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) v_place[j] = (4 * b + j) * row + i * 4;
    const int first_place = t.begin + wave * 32, turns = first_place < t.end ? (t.end - first_place + 127) / 128 : 0;
    auto key_of_turn = [&](int turn) { return key_at<SINKS>(t, first_place + turn * 128); };
    // fp32, tiles of a sequence that read the same long runs, a workgroup to a compute unit at most: all loads of a turn go before its products,
    // which keeps the tiles together.  us so / with the loads among the products, one sequence, 32 heads on 8: 8 tokens over 32768 keys 66 / 71,
    // 16 tokens 101 / 111, over 131072 keys 364 / 400.  With more workgroups the products of one hide the loads of another, and short runs end
    // sooner: 8 x 16 tokens over 32768 keys 869 / 752, 12 tokens of one sequence 152 / 136, one token over 64 keys 6.7 / 6.4, 2048 keys
    // 12.1 / 11.6.  bf16: no gain (one token over 64 keys 4.85 / 4.75, 131072 keys 97 / 97).
    const bool in_step = ALONE && __is_same(KT, lvr_f32_t) && t.rows > 16 && t.end - t.begin >= IN_STEP_RUN &&
                         (int64_t)bt.n_seqs * ((t.rows + 15) >> 4) * t.splits * a.n_kv <= COMPUTE_UNITS;
    // There, and on pages in 4 bits, the pages of 32 turns are looked up at once, by one lane for each 16 keys, which lie in one page.  Where there is
    // none, some memory of the pool.  (Other tiles often end after a turn or two: 1024 single tokens over 200 keys, bf16, 260 us so, 250 with a
    // look-up for each 16 keys.)
    struct {
        int page;                   // or, of FP4, what is added to a pool's address for the codes (low, high), and to that for the scales
        uint32_t low, high;
        int32_t scales;
    } place_of = {};
    uint64_t without = 0;           // (FP4) which of them have no page
    auto look_up = [&](int turn) {
        const int place = first_place + (turn + (lane >> 1)) * 128;
        const int key = place < t.end ? key_at<SINKS>(t, place) + (lane & 1) * 16 : t.hi;
        place_of.page = key < t.hi ? lvr_page_of(bt, t.seq, key) : -1;
        if constexpr (FP4) {        // a page is at most 2^30 bytes of codes
            const uint32_t in_page = (uint32_t)kvh * (uint32_t)bt.head_stride + ((uint32_t)key & ((1u << bt.page_shift) - 1)) * row;
            const bool none = place_of.page < 0;
            const uint64_t at = none ? 0 : (uint64_t)(uint32_t)place_of.page * (uint64_t)bt.page_stride + in_page;
            place_of.low = (uint32_t)at;
            place_of.high = (uint32_t)(at >> 32);
            place_of.scales = (int32_t)bt.scales + (none ? 0 : (int32_t)(in_page / 16) - (int32_t)in_page);
            without = __ballot(none);
        }
    };
    auto ask_rows = [&](int page, int key, Keys &x, int h) {   // (not FP4)
        if constexpr (!FP4) {
            const int64_t at = lvr_row_at(bt, page < 0 ? 0 : page, kvh, page < 0 ? 0 : key);   // no page: some memory of the pool
            const char *kp = a.k_pages + at, *vp = a.v_pages + at;
            R::load_k(kp + i * bt.row_stride, b, x.k[h]);
#pragma unroll
            for (int j = 0; j < 4; ++j) R::load_v(vp + (4 * b + j) * bt.row_stride, i, x.v[h][j]);
        }
    };
    auto ask = [&](int turn, Keys &x) {
        if (FP4 && turn >= turns) turn = turns - 1;
        if ((turn & 31) == 0) look_up(turn);
        const int k0 = key_of_turn(turn);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int who = 2 * (turn & 31) + h;
            if constexpr (FP4) {
                // One address for the wave and a lane's 32-bit place behind it, in the load itself (the places are made opaque here, or they
                // are widened before the loop and added up in registers that loads are on their way to).
                x.none[h] = without >> who & 1;
                const uint64_t at = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(place_of.high, who) << 32 | (uint32_t)__builtin_amdgcn_readlane(place_of.low, who);
                const int32_t scales = __builtin_amdgcn_readlane(place_of.scales, who);
                const char *kp = a.k_pages + at, *vp = a.v_pages + at, *ks = kp + scales, *vs = vp + scales;
                asm volatile("" : "+v"(k_place), "+v"(k_scale), "+v"(v_scales));
                x.k[h].codes = *reinterpret_cast<const uint4 *>(kp + k_place);
                x.k[h].scale = (uint8_t)ks[k_scale];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    asm volatile("" : "+v"(v_place[j]));
                    x.v[h].codes[j] = *reinterpret_cast<const uint32_t *>(vp + v_place[j]);
                }
                x.v[h].scales = *reinterpret_cast<const uint32_t *>(vs + v_scales);
            } else {
                const int page = __builtin_amdgcn_readlane(place_of.page, who);
                x.none[h] = page < 0;
                ask_rows(page, k0 + h * 16, x, h);
            }
        }
    };
    // 16 keys from `key0` on, not all of which every row of the tile sees; whether V has a value that some rows must not meet.
    auto hide = [&](int key0, bool none, float (&p)[4], auto &v) {
        bool poison = false;
        // Without a page nothing is seen.  A bound that says so saves a branch for each of the four where this is most of the work: us with the
        // bound / with branches, one token, bf16 and a window of 64 8.6 / 8.9, 250 keys 8.7 / 9.0, fp32 10.4 / 10.7 and 10.5 / 10.7.  Beside tiles
        // of 128 rows fp32 loses by it (30 x 16 tokens over 3000 keys 298 / 287), and 4 bits have no registers for it.
        constexpr bool BY_BOUND = ALONE && !FP4;
        const int row_last = BY_BOUND && none ? -1 : last;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int key = key0 + 4 * b + j;
            if ((!BY_BOUND && none) || hidden<SINKS>(a, key, first, row_last)) p[j] = -INFINITY;
            // a row of V that no query row sees is memory nobody has written; one that some see meets the others with
            // weight zero, which an infinity or a NaN would survive
            const bool unseen = none || hidden<SINKS>(a, key, t.lo, t.hi - 1);
            if constexpr (FP4) v.codes[j] = unseen ? 0 : v.codes[j];
            else if (unseen) R::zero_v(v[j]);
            else if (R::odd_v(v[j])) poison = true;
        }
        if constexpr (FP4) {   // the key whose scales this lane has
            if (none || hidden<SINKS>(a, key0 + 4 * b + (i & 3), t.lo, t.hi - 1)) v.scales = 0x7f7f7f7f;
            else if (R::own_scale(v) == 255) poison = true;
        }
        return poison;
    };
    // The scores become weights.
    auto weigh = [&](float (&p)[2][4]) {
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
    };
    auto work = [&](int k0, Keys &x) {
        const bool partly = !all_seen<SINKS>(a, k0, 32, row_begin, row_end) || x.none[0] || x.none[1];
        float p[2][4];
        bool poison = false;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const f32x4 s = R::score(x.k[h], q);
#pragma unroll
            for (int j = 0; j < 4; ++j) p[h][j] = s[j];
        }
        if (partly) {
            if (FP4) asm volatile("");   // one branch
#pragma unroll
            for (int h = 0; h < 2; ++h) poison |= hide(k0 + h * 16, x.none[h], p[h], x.v[h]);
        }
        weigh(p);
        redo |= poison;
        R::add(x.v, p, o, l);
    };
    if constexpr (FP4) {
        if (turns > 0) {
            // Rows are asked for a turn ahead.  The last turn asks for its own again, so that there are always as many loads behind the ones that
            // are waited for.  (Two turns ahead take registers that a fourth workgroup on a compute unit needs: 2 to 5 % slower.)
            Keys x, y;
            ask(0, x);
            for (int turn = 0;;) {
                ask(turn + 1, y);
                work(key_of_turn(turn), x);
                if (++turn >= turns) break;
                ask(turn + 1, x);
                work(key_of_turn(turn), y);
                if (++turn >= turns) break;
            }
        }
    } else if (in_step) {
        for (int turn = 0; turn < turns; ++turn) {   // uniform over the wave
            Keys x;
            ask(turn, x);
            __builtin_amdgcn_sched_barrier(0);   // all loads on their way before one is waited for
            work(key_of_turn(turn), x);
        }
    } else {
        for (int place = first_place; place < t.end; place += 128) {   // uniform over the wave
            const int k0 = key_at<SINKS>(t, place);
            Keys x;
#pragma unroll
            for (int h = 0; h < 2; ++h) {   // 16 keys: one page
                const int key = k0 + h * 16, page = key < t.hi ? __builtin_amdgcn_readfirstlane(lvr_page_of(bt, t.seq, key)) : -1;
                x.none[h] = page < 0;
                ask_rows(page, key, x, h);
            }
            const bool partly = !all_seen<SINKS>(a, k0, 32, row_begin, row_end) || x.none[0] || x.none[1];
            float p[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {   // (masked one by one, so that the second half's loads may follow the first half's products)
                const f32x4 s = R::score(x.k[h], q);
#pragma unroll
                for (int j = 0; j < 4; ++j) p[h][j] = s[j];
                if (partly) redo |= hide(k0 + h * 16, x.none[h], p[h], x.v[h]);
            }
            weigh(p);
            R::add(x.v, p, o, l);
        }
    }
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);

    // the four waves' (m, l, o) become the rows' outputs
    if (__any(redo)) {
        for (int r = 0; r < 16 && t.row0 + r < t.rows; ++r) {
            const RowSum s = one_row<KT, SINKS>(a, bt, t, kvh, t.row0 + r, t.begin + wave * 32, 32, 128);
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
    const int r = threadIdx.x >> 4, c0 = (threadIdx.x & 15) * 8;
    const bool writes = t.row0 + r < t.rows;
    Merged x;
    auto from_lds = [&](int sets) {   // the sums of the waves' sets of keys, or of their shares of partials
        __syncthreads();
        x.clear();
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = lds.o[w][r][c0 + e];
            if (w < sets) x.add(lds.m[w][r], lds.l[w][r], v);
        }
    };
    auto write = [&]() {
        if (!writes) return;
        const float inv = x.l == 0.f ? 0.f : 1.f / x.l;   // nothing seen: zeros
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = x.o[e] * inv;
        store_row<R::ELT>(a, t, kvh, t.row0 + r, c0, y);
    };
    if (t.splits == 1) {
        from_lds(4);
        write();
        return;
    }
    // The last workgroup to end of every `fan` of a tile's runs merges those, and the last of these merges what they made, so that nobody
    // is left with all of them (one token over 8192 keys 13.1 us; all merged by one workgroup 15.2).  Four rows fill a wave, and where a tile has no
    // more the waves share the partials out; each takes up to FAN of them with all their loads in flight.  Partials cross
    // from one die to another: they are stored and read with accesses of device scope, and a workgroup waits for its own stores
    // before it takes a ticket, which wraps at the number of those who take it and so is zero again afterwards.
    // All of this is code that one workgroup in many runs, and fetches as it goes: it is kept short.
    const int rows = t.rows - t.row0, sharer_bits = rows <= 4 ? 2 : (rows <= 8 ? 1 : 0), sharers = 1 << sharer_bits, fan = FAN * sharers;
    const int slot0 = t.slot - t.split, fans = (t.splits + fan - 1) >> (FAN_BITS + sharer_bits), mine = t.split >> (FAN_BITS + sharer_bits);
    const int levels = fans == 1 ? 1 : 2;
    int slot = t.slot, first_slot = slot0 + mine * fan, apart = 1, n = mine + 1 < fans ? fan : t.splits - mine * fan;
    const uint32_t part_size = 16 * (LVR_D + 2) * sizeof(float);
    const auto parts = __builtin_amdgcn_make_buffer_rsrc(a.part + (int64_t)WIDE_ROOM * 128 * (LVR_D + 2), 0, NARROW_ROOM * part_size, 0x00027000);
    constexpr int DEVICE = 16;   // sc1
    int sets = 4;
#pragma unroll 1
    for (int level = 0;; ++level) {
        if (level == 0 || sharers > 1) from_lds(sets);
        if (level == levels) break;
        if (writes) {
            const uint32_t at = (slot * a.n_kv + kvh) * part_size;
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{x.o[0], x.o[1], x.o[2], x.o[3]}), parts, (r * LVR_D + c0) * 4, at, DEVICE);
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{x.o[4], x.o[5], x.o[6], x.o[7]}), parts, (r * LVR_D + c0) * 4 + 16, at, DEVICE);
            if (c0 == 0) __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(x.m), __float_as_uint(x.l)}, parts, (16 * LVR_D + r * 2) * 4, at, DEVICE);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (threadIdx.x == 0) lds.arrived = atomicInc(a.ticket + ((int64_t)first_slot * a.n_kv + kvh) * LVR_CNT_STRIDE + level, (unsigned)n - 1u);
        __syncthreads();
        if (lds.arrived != (unsigned)n - 1u) return;
        const int share = wave >> (2 - sharer_bits), mr = (wave & ((4 >> sharer_bits) - 1)) * 4 + (lane >> 4);   // whose turn, which row
        x.clear();
#pragma unroll 1
        for (int p0 = share; p0 < n; p0 += fan) {
            u32x2 ml[FAN];
            u32x4 v[FAN][2];
#pragma unroll
            for (int k = 0; k < FAN; ++k) {   // past the last one the last once more
                const uint32_t at = ((first_slot + (p0 + k * sharers < n ? p0 + k * sharers : n - 1) * apart) * a.n_kv + kvh) * part_size;
                ml[k] = __builtin_amdgcn_raw_buffer_load_b64(parts, (16 * LVR_D + mr * 2) * 4, at, DEVICE);
                v[k][0] = __builtin_amdgcn_raw_buffer_load_b128(parts, (mr * LVR_D + c0) * 4, at, DEVICE);
                v[k][1] = __builtin_amdgcn_raw_buffer_load_b128(parts, (mr * LVR_D + c0) * 4 + 16, at, DEVICE);
            }
            asm volatile("" ::: "memory");   // all of them asked for before one is waited for
#pragma unroll
            for (int k = 0; k < FAN; ++k) {   // (rows that are none hold anything, and go nowhere)
                if (p0 + k * sharers >= n) break;
                const f32x4 y0 = __builtin_bit_cast(f32x4, v[k][0]), y1 = __builtin_bit_cast(f32x4, v[k][1]);
                const float y[8] = {y0[0], y0[1], y0[2], y0[3], y1[0], y1[1], y1[2], y1[3]};
                x.add(__uint_as_float(ml[k][0]), __uint_as_float(ml[k][1]), y);
            }
        }
        if (sharers > 1) {
            if (c0 == 0) {
                lds.m[share][mr] = x.m;
                lds.l[share][mr] = x.l;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) lds.o[share][mr][c0 + e] = x.o[e];
            sets = sharers;
        }
        slot = first_slot;   // where the second level finds it
        first_slot = slot0;
        apart = fan;
        n = fans;
    }
    write();
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
// instructions meet the other's exponentials.  A prompt of 16384 tokens (32 heads on 8, 2.2 TFLOP): 2.08 to 2.15 ms on different cards, 1020 to
// 1060 TFLOP/s; matrix units busy 48 % and vector units 43 % of the clocks, where the library's product of 8192 x 8192 matrices reaches
// 1148 to 1409 TFLOP/s.  fp32, 8192 tokens: 135 TFLOP/s of the 154 the library reaches.  One workgroup to a compute unit takes 1.43 times as long as
// two, whose instructions meet for the most part.  Tried without gain: the scores of the next tile made between the exponentials of this one (-2 %),
// V's operands read a step ahead (bf16 0 to 1 %, 4 bits -1 %), priority for exponentials (-2 to -6 %), tiles through registers (653 TFLOP/s: the
// loads were waited for at once).
//
// A tile's loads are not waited for before its products, which overlaps them where few workgroups are left: 40 ragged sequences of up to 20 new tokens
// of 20000 378 us with such a wait and 285 without.  Even batches of few rows over long runs, bound by the read, lose a little by it: 8 x 16 tokens
// over 32768 keys 194 and 199.
// ---------------------------------------------------------------------------------------------------------------------------
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

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
        // 32 keys' operands are read at once, the other 32 keys' while those are worked on (read as they are needed: 1 to 4 % slower)
        static_assert(NT == 2, "");
        bf16x8 f[NT][8];
        s[0] = f32x16{0.f}, s[1] = f32x16{0.f};
        auto read = [&](int kt, int st) { f[kt][st] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(k + (kt * 32 + n) * ROWB + k_piece(n, 2 * st + h) * 16)); };
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int st = 0; st < 8; ++st) read(0, st);
#pragma unroll
        for (int st = 0; st < 8; ++st) {
            __builtin_amdgcn_sched_barrier(0);
            read(1, st);
            s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[0][st], q[st], s[0], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int st = 0; st < 8; ++st) s[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[1][st], q[st], s[1], 0, 0, 0);
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
    // Largest magnitudes, of each half of the words apart; whether one is an infinity or a NaN.
    static __device__ __forceinline__ void largest(uint4 &m, const uint4 &v) {
        typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
        m = __builtin_bit_cast(uint4, __builtin_elementwise_max(__builtin_bit_cast(u16x8, m), (u16x8)(__builtin_bit_cast(u16x8, v) & (uint16_t)0x7fff)));
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
    static __device__ __forceinline__ void largest(uint4 &m, const uint4 &v) {
        m = __builtin_bit_cast(uint4, __builtin_elementwise_max(__builtin_bit_cast(u32x4, m), __builtin_bit_cast(u32x4, v) & 0x7fffffffu));
    }
    static __device__ __forceinline__ bool odd(const uint4 &v) {
        return (v.x & 0x7f800000u) == 0x7f800000u || (v.y & 0x7f800000u) == 0x7f800000u || (v.z & 0x7f800000u) == 0x7f800000u ||
               (v.w & 0x7f800000u) == 0x7f800000u;
    }
};

// Pages in 4 bits: a tile becomes bf16 on its way into LDS and is worked on as such.  Codes pass through registers, a block and its scale a lane; they
// are asked for a tile ahead and widened while this one's products run.  Bound as in bf16: the prompt of 16384 tokens 2.06 to 2.14 ms, widening hides
// behind the read that it saves (matrix units busy 44 % and vector units 46 % of the clocks).
template <>
struct Rows128<lvr_fp4_t> : Rows128<lvr_bf16_t> {};

// 16 bytes per lane from global memory into LDS, the wave's 1 KiB in a row from `to` on.  vmcnt counts it.
__device__ __forceinline__ void load_to_lds(const char *from, uint32_t offset, char *to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t *)(from + offset),
                                     (__attribute__((address_space(3))) uint32_t *)to, 16, 0, 0);
}

template <typename KT>
struct Rows128Lds {
    __align__(16) char k[2][Rows128<KT>::TK * Rows128<KT>::ROWB], v[2][Rows128<KT>::TK * Rows128<KT>::ROWB];
    uint32_t odd[2][4];   // (FP4) whether a wave's rows of V have a block that is no number
};

// urgent: a second product goes before what the other workgroup on the compute unit has to do.  Two that begin together else stay in step, both at
// their products and then both at their exponentials.  us without / with, bf16, fp32, 4 bits:
//   one round of pieces: 1000 new tokens of 12000            215 / 209    1505 / 1486    216 / 204
//                        two sequences of 512 new of 8192     157 / 153   1049 / 1037    157 / 150
//   two rounds, one or two sequences: prompt of 4096          164 / 158   1161 / 1096    164 / 155
//               prompt of 2048                                 65 / 64     350 / 319      66 / 62
//               two prompts of 2048                            94 / 93     618 / 581      93 / 93
//   two rounds, more of them: four prompts of 1024             66 / 68     397 / 415      66 / 69
//               16 ragged ones of up to 500 new of 3000        62 / 67     305 / 331      61 / 64
//               four of 1024 new of 4096, a window of 1000     98 / 104    550 / 554      93 / 98
// Batches of one round and a half go either way: a prompt of 3000 loses by it (94 / 98, 627 / 628, 93 / 98), three prompts of 1000 would gain
// (53 / 53, 290 / 287, 56 / 55), the 16 ragged ones are such a batch too.
// In three rounds workgroups are out of step by themselves (prompt of 16384 nothing, of 8192 with a window of 2048 288 / 297).
template <typename KT, bool SINKS>
__device__ __forceinline__ void rows128_piece(const AttnArgs &a, const lvr_paged_batch &bt, const Tile &t, int kvh, bool urgent, Rows128Lds<KT> &lds) {
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
    // (entries as the table has them, so that nobody waits for them before the rows are asked for)
    auto pages_of = [&](int place) {
        const int key = key_at<SINKS>(t, place) + 16 * (lane % (TK / 16));
        return key < t.hi && key < bt.table_width << bt.page_shift ? bt.table[(int64_t)t.seq * bt.table_width + (key >> bt.page_shift)] : -1;
    };
    constexpr bool FP4 = __is_same(KT, lvr_fp4_t);
    // Of FP4: a lane brings a block of a row of K and of V, 32 codes and their scale, and makes four pieces of each.  Four rows of K side by side
    // go to different banks; V's pieces are taken in an order that differs from row to row, so that they do.
    struct { uint4 k, v; uint32_t ks, vs; } raw;
    const int fp4_row = lane >> 2, fp4_block = lane & 3, fp4_key = group + fp4_row;
    const uint32_t fp4_place = (uint32_t)fp4_row * (uint32_t)bt.row_stride + fp4_block * 16, fp4_scale = (uint32_t)fp4_row * ((uint32_t)bt.row_stride / 16) + fp4_block;
    const int to_k0 = R::key_of_k_row(fp4_key) * R::ROWB + R::k_piece(R::key_of_k_row(fp4_key), fp4_block * 4) * 16;   // (that permutation is its own inverse)
    const int to_v0 = fp4_key * R::ROWB + (R::v_piece(fp4_key, fp4_block * 4) ^ (fp4_key & 3)) * 16;
    auto load = [&](int place, int pages, char *to_k, char *to_v) {
        const int k0 = key_at<SINKS>(t, place);
        pages = pages < bt.n_pages ? pages : -1;
        const int page = __builtin_amdgcn_readlane(pages, group / 16);
        const int64_t at = page < 0 ? kvh * bt.head_stride : lvr_row_at(bt, page, kvh, k0 + group);   // no page: some memory of the pool
        if constexpr (FP4) {
            const int64_t sc = lvr_scales_at(bt, page < 0 ? 0 : page, kvh, page < 0 ? 0 : k0 + group);
            raw.k = *reinterpret_cast<const uint4 *>(a.k_pages + at + fp4_place);
            raw.v = *reinterpret_cast<const uint4 *>(a.v_pages + at + fp4_place);
            raw.ks = (uint8_t)a.k_pages[sc + fp4_scale];
            raw.vs = (uint8_t)a.v_pages[sc + fp4_scale];
            return (uint32_t)__ballot(pages < 0) & ((1u << TK / 16) - 1u);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            load_to_lds(a.k_pages + at, k_off[i], to_k + (wave * 4 + i) * 1024);
            load_to_lds(a.v_pages + at, v_off[i], to_v + (wave * 4 + i) * 1024);
        }
        return (uint32_t)__ballot(pages < 0) & ((1u << TK / 16) - 1u);   // groups without a page
    };
    // Of FP4: what was loaded for the tile at `place`, into LDS.  A row of V that no query row sees may be memory nobody has written.
    auto unfold = [&](int place, uint32_t none, char *to_k, char *to_v, uint32_t *odd) {
        const int k0 = key_at<SINKS>(t, place);
        if (!all_seen<SINKS>(a, k0, TK, t.lo, t.hi) || none != 0)
            if ((none >> (group >> 4) & 1) || hidden<SINKS>(a, k0 + fp4_key, t.lo, t.hi - 1)) {
                raw.v = make_uint4(0, 0, 0, 0);
                raw.vs = 127;
            }
        const bool some_odd = __any(raw.vs == 255);
        if (lane == 0) odd[wave] = some_odd;
        const bool swap1 = fp4_key & 1, swap2 = fp4_key & 2;
        const uint32_t x0 = swap1 ? raw.v.y : raw.v.x, x1 = swap1 ? raw.v.x : raw.v.y, x2 = swap1 ? raw.v.w : raw.v.z, x3 = swap1 ? raw.v.z : raw.v.w;
        const uint32_t kw[4] = {raw.k.x, raw.k.y, raw.k.z, raw.k.w}, vw[4] = {swap2 ? x2 : x0, swap2 ? x3 : x1, swap2 ? x0 : x2, swap2 ? x1 : x3};
        const float ks = lvr_fp4_scale(raw.ks), vs = lvr_fp4_scale(raw.vs);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            *reinterpret_cast<lvr_bf16x8 *>(to_k + (to_k0 ^ c * 16)) = lvr_fp4_values(kw[c], ks);
            *reinterpret_cast<lvr_bf16x8 *>(to_v + (to_v0 ^ c * 16)) = lvr_fp4_values(vw[c], vs);
        }
    };
    auto arrived = [] {
        // (the built-in wait: one in assembly is no news to the compiler, which would wait once more for whatever was loaded before)
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0) lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    uint32_t none = 0;
    if (t.begin < t.end) none = load(t.begin, pages_of(t.begin), lds.k[0], lds.v[0]);
    int pages = pages_of(t.begin + TK);
    if constexpr (FP4)
        if (t.begin < t.end) unfold(t.begin, none, lds.k[0], lds.v[0], lds.odd[0]);
    // A tile is worked on while the next one is on its way.  The buffers are told apart for the compiler, which else waits for what comes into one
    // before it reads the other.
    auto step = [&](int place, int buf, const char *__restrict k, char *__restrict v, char *__restrict next_k, char *__restrict next_v) __attribute__((always_inline)) {
        const int k0 = key_at<SINKS>(t, place);
        uint32_t next_none = 0;
        if (place + TK < t.end) {
            next_none = load(place + TK, pages, next_k, next_v);
            pages = pages_of(place + 2 * TK);
        }
        if (!FP4 && (!all_seen<SINKS>(a, k0, TK, t.lo, t.hi) || none != 0)) {   // a row of V that no query row sees may be memory nobody has written
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key = srow + i * RPI;
                if (hidden<SINKS>(a, k0 + key, t.lo, t.hi - 1) || (none >> (key >> 4) & 1))
                    *reinterpret_cast<uint4 *>(v + key * R::ROWB + piece * 16) = make_uint4(0, 0, 0, 0);
            }
            arrived();
        }
        if (k0 < whi && (k0 + TK > wlo || (SINKS && k0 < a.sinks))) {
            f32x16 p[R::NT];
            R::scores(k, q, n, h, p);
            const bool partly = !all_seen<SINKS>(a, k0, TK, all_lo, all_hi) || none != 0;
            if (partly) {
                asm volatile("");   // a branch, not 32 selects in every tile
                if constexpr (FP4) {
                    redo |= (lds.odd[buf][0] | lds.odd[buf][1] | lds.odd[buf][2] | lds.odd[buf][3]) != 0;
                } else {
                    uint4 worst = make_uint4(0, 0, 0, 0);
#pragma unroll 4
                    for (int c = 0; c < TK * R::ROWB / 1024; ++c) R::largest(worst, *reinterpret_cast<const uint4 *>(v + c * 1024 + lane * 16));
                    redo |= R::odd(worst);
                }
                // keys from_here .. from_here + count of the tile are seen, and with first keys among them those before sink_end
                const int from_here = (last < first ? 1 << 30 : first) - k0 - R::key_of(h, 0, 0), count = last < first ? 0 : last - first;
                const int sink_end = (a.sinks < last + 1 ? a.sinks : last + 1) - k0 - R::key_of(h, 0, 0);
                const bool sink_here = SINKS && k0 < a.sinks;
#pragma unroll
                for (int kt = 0; kt < R::NT; ++kt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int key = R::key_of(0, kt, r);   // (the lane's own 8 or 4 h is in from_here)
                        if ((uint32_t)(key - from_here) > (uint32_t)count && !(sink_here && key < sink_end)) p[kt][r] = -INFINITY;
                    }
                if (none != 0) {
#pragma unroll
                    for (int kt = 0; kt < R::NT; ++kt)
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            if (none >> (R::key_of(h, kt, r) >> 4) & 1) p[kt][r] = -INFINITY;
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
            if (urgent) __builtin_amdgcn_s_setprio(1);
            R::add(v, p, lane, o, l);
            if (urgent) __builtin_amdgcn_s_setprio(0);
        }
        if constexpr (FP4)
            if (place + TK < t.end) unfold(place + TK, next_none, next_k, next_v, lds.odd[buf ^ 1]);
        none = next_none;
        arrived();
    };
    arrived();
    int buf = 0;
    for (int place = t.begin; place < t.end; place += TK, buf ^= 1)   // uniform over the workgroup
        step(place, buf, lds.k[buf], lds.v[buf], lds.k[buf ^ 1], lds.v[buf ^ 1]);
    l += __shfl_xor(l, 32, 64);
    if (__any(redo)) {
        for (int r = row0; r < row0 + 32 && r < t.rows; ++r) {
            RowSum s = one_row<KT, SINKS>(a, bt, t, kvh, r, t.begin, 1 << 30, 1 << 30);
            if (t.splits > 1) {
                float *mine = partial128(a.part, t.slot, a.n_kv, kvh);
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
        float *mine = partial128(a.part, t.slot, a.n_kv, kvh) + (wave * 32 + n) * LVR_D;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float4 v = R::ELT == 2 ? make_float4(o[i >> 2][(i & 3) * 4], o[i >> 2][(i & 3) * 4 + 1], o[i >> 2][(i & 3) * 4 + 2], o[i >> 2][(i & 3) * 4 + 3])
                                         : make_float4(o[0][i], o[1][i], o[2][i], o[3][i]);
            *reinterpret_cast<float4 *>(mine + (R::ELT == 2 ? R::coordinate(h, i >> 2, (i & 3) * 4) : R::coordinate(h, 0, i))) = v;
        }
        if (h == 0) *reinterpret_cast<float2 *>(partial128(a.part, t.slot, a.n_kv, kvh) + 128 * LVR_D + (wave * 32 + n) * 2) = make_float2(m, l);
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
// Where a token's heads lie side by side in 4 bits, a line of memory holds rows of two heads and scales of all: there the heads of a piece follow each
// other on one die, eight pieces on the eight dies (48 ragged single tokens 199 us with a KV head to a die, 170 so).
template <typename KT>
__device__ __forceinline__ int piece_of_block(const AttnArgs &a, const lvr_paged_batch &bt, int &kvh) {
    const int piece = blockIdx.z * GRID_Y + blockIdx.y;
    kvh = blockIdx.x;
    if constexpr (__is_same(KT, lvr_fp4_t)) {
        if (bt.row_stride == LVR_FP4_CODES || (piece | 7) >= (int)(gridDim.y * gridDim.z)) return piece;
        const int in_eight = (piece & 7) * a.n_kv + kvh;   // of the workgroups of eight pieces
        kvh = in_eight >> 3;
        return (piece & ~7) + (in_eight & 7);
    }
    return piece;
}
inline dim3 grid_of(int n_kv, int64_t pieces) {
    return dim3((unsigned)n_kv, (unsigned)(pieces < GRID_Y ? pieces : GRID_Y), (unsigned)((pieces + GRID_Y - 1) / GRID_Y));
}

template <typename KT, bool SINKS>
constexpr bool may_be_uncut = SINKS || __is_same(KT, lvr_fp4_t);

// Tiles of 16 rows alone: batches in which every sequence brings a token or so.
template <typename KT, bool SINKS>
__global__ void __launch_bounds__(256, __is_same(KT, lvr_fp4_t) ? 4 : 2) paged_attention_rows16_kernel(AttnArgs a, lvr_paged_batch bt) {
    __shared__ Rows16Lds lds;
    int kvh;
    const int piece = piece_of_block<KT>(a, bt, kvh);
    Tile t;
    Division<false, Wave, SINKS, may_be_uncut<KT, SINKS>> d(a, bt);
    if (d.divide(a.target) && d.template locate<false>(piece, t)) rows16_piece<KT, SINKS, true>(a, bt, t, kvh, lds);
}

// Any batch: every sequence in the tiles that suit it.
template <typename KT, bool SINKS>
__global__ void __launch_bounds__(256, 2) paged_attention_mixed_kernel(AttnArgs a, lvr_paged_batch bt) {
    __shared__ union { Rows16Lds narrow; Rows128Lds<KT> wide; } lds;
    int kvh;
    const int piece = piece_of_block<KT>(a, bt, kvh);
    Tile t;
    Division<true, Wave, SINKS, may_be_uncut<KT, SINKS>> d(a, bt);
    if (!d.divide(a.target) || !d.template locate<false>(piece, t)) return;
    if (t.height == 128) rows128_piece<KT, SINKS>(a, bt, t, kvh, d.n_wide * a.n_kv <= (bt.n_seqs <= 2 ? 2 : 1) * MIXED_PIECES, lds.wide);
    else rows16_piece<KT, SINKS, false>(a, bt, t, kvh, lds.narrow);
}

// Merges the runs of cut 128-row tiles.  16 rows of a tile at a time, 16 lanes to a row; the workgroups share them out.  A launch of its own, unlike
// for tiles of 16 rows: a partial result of 128 rows is 66 KiB, and the last workgroup of a tile would read all of them alone.  Bound by that read:
// 512 partial results (34 MB) 10 us.
template <typename KT, bool SINKS>
__global__ void __launch_bounds__(256) paged_attention_merge_kernel(AttnArgs a, lvr_paged_batch bt) {
    Division<true, Wave, SINKS> d(a, bt);
    if (!d.divide(a.target)) return;
    const int c0 = (threadIdx.x & 15) * 8;
    const int64_t step = (int64_t)a.n_kv * (128 * (LVR_D + 2));
    for (int item = blockIdx.x;; item += gridDim.x) {
        const int kvh = item % a.n_kv, r = item / a.n_kv % 8 * 16 + (threadIdx.x >> 4);
        Tile t;
        if (!d.template locate<true>(item / a.n_kv / 8, t)) return;
        if (t.splits == 1 || t.row0 + r >= t.rows) continue;
        const float *first_part = partial128(a.part, t.slot, a.n_kv, kvh);
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
                                      int64_t q_stride_bytes, int32_t window, int32_t sinks, void *out, hipStream_t st) {
    AttnArgs a;
    a.k_pages = static_cast<const char *>(k_pages);
    a.v_pages = static_cast<const char *>(v_pages);
    a.q = static_cast<const char *>(q);
    a.out = static_cast<char *>(out);
    a.q_stride = q_stride_bytes;
    a.window = window;
    a.sinks = sinks;
    a.unit = pc->sigma * LOG2E;
    a.part = pc->part;
    a.ticket = pc->ticket;
    const int type = pc->cfg.kv_dtype;
    const PagedLaunch launch = paged_launch(a, b, pc->cfg.n_q_heads, pc->cfg.n_kv_heads, type != LVR_F32, type == LVR_FP4);
    const dim3 grid = grid_of(a.n_kv, launch.pieces);
#define LVR_LAUNCH(KERNEL, KT, GRID)                                                                                  \
    do {                                                                                                              \
        if (a.sinks) hipLaunchKernelGGL((KERNEL<KT, true>), GRID, dim3(256), 0, st, a, b);                            \
        else hipLaunchKernelGGL((KERNEL<KT, false>), GRID, dim3(256), 0, st, a, b);                                   \
    } while (0)
#define LVR_BY_TYPE(KERNEL, GRID)                                             \
    do {                                                                      \
        if (type == LVR_BF16) LVR_LAUNCH(KERNEL, lvr_bf16_t, GRID);           \
        else if (type == LVR_F32) LVR_LAUNCH(KERNEL, lvr_f32_t, GRID);        \
        else LVR_LAUNCH(KERNEL, lvr_fp4_t, GRID);                             \
    } while (0)
    if (!launch.mixed) {
        LVR_BY_TYPE(paged_attention_rows16_kernel, grid);
        return hipGetLastError();
    }
    LVR_BY_TYPE(paged_attention_mixed_kernel, grid);
    if (a.target > 0) {   // (what it merges is fp32, what it writes fp32 or bf16)
        const dim3 merge(MERGE_WGS);
        if (type == LVR_F32) LVR_LAUNCH(paged_attention_merge_kernel, lvr_f32_t, merge);
        else LVR_LAUNCH(paged_attention_merge_kernel, lvr_bf16_t, merge);
    }
#undef LVR_BY_TYPE
#undef LVR_LAUNCH
    return hipGetLastError();
}
