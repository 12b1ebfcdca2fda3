// The paged cache: its handle, the calls' checks, and the kernels that move rows in (lvr_paged_append) and out
// (lvr_paged_gather).  The attention over the pages is paged_attention.hip.
//
// Both are bound by HBM where there is enough to move: every row is read once and written once, in 16-byte accesses (rows in 4 bits: of 4 to 16 bytes).
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

// The same in 64 bits, of a fraction in units of 2^-64: series to x^15 and x^16, off by less than 2^-50.
__device__ __forceinline__ void sincos_turn(uint64_t phase, double &sn, double &cs) {
    const uint64_t quarter = (phase + ((uint64_t)1 << 61)) >> 62;
    const double x = (double)(int64_t)(phase - (quarter << 62)) * 3.4061215800304736e-19;   // 2 pi / 2^64
    const double x2 = x * x;
    double s = -1. / 1307674368000, c = 1. / 20922789888000;
    const double s_of[] = {1. / 6227020800, -1. / 39916800, 1. / 362880, -1. / 5040, 1. / 120, -1. / 6, 1.};
    const double c_of[] = {-1. / 87178291200, 1. / 479001600, -1. / 3628800, 1. / 40320, -1. / 720, 1. / 24, -0.5, 1.};
#pragma unroll
    for (int i = 0; i < 7; ++i) s = __builtin_fma(s, x2, s_of[i]);
#pragma unroll
    for (int i = 0; i < 8; ++i) c = __builtin_fma(c, x2, c_of[i]);
    s *= x;
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
    const char *q_weight, *k_weight;        // of the norms; NULL: ones
    float eps;
};

// What a lane holds of a row: two pieces, `at0` and `at1` coordinates into it, and whether they are rotated.
struct Pieces {
    int at0, at1;
    bool rot0, rot1;
};
template <int E, bool NEIGHBOURS>
__device__ __forceinline__ Pieces pieces_of(int li, int rot) {
    constexpr int LANES = PAIRS / E;
    Pieces p = {E * li, PAIRS + E * li, E * li < rot, PAIRS + E * li < rot};
    if (!NEIGHBOURS) {
        const int half = rot / 2, copied = li - half / E;
        p.rot0 = p.rot1 = copied < 0;
        p.at0 = p.rot0 ? E * li : rot + E * copied;
        p.at1 = p.rot0 ? half + E * li : p.at0 + E * (LANES - half / E);
    }
    return p;
}
// Which pair of the rotation the e-th of a lane is.
template <int E, bool NEIGHBOURS>
__device__ __forceinline__ int pair_of(int li, int e) { return NEIGHBOURS ? (e < E / 2 ? 0 : PAIRS / 2 - E / 2) + E * li / 2 + e : E * li + e; }

// What a lane needs to turn a pair, asked for before the token's position is known.
struct Angle {
    uint64_t turns = 0;
    int position = 0;
    __device__ __forceinline__ Angle(const AppendArgs &a, int t) {
        const int pair = lvr_lane();
        if (pair >= a.rot / 2) return;
        turns = a.turns[pair];
        if (a.positions) position = a.positions[(int64_t)t * a.axes + (a.axes > 1 ? a.axis[pair] : 0)];
    }
};

// A sum, or the largest, over the LANES lanes of a row (8 or 16, which start at a multiple of that); every one of them gets it.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false); }
template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(double, (uint64_t)dpp<CTRL>((uint32_t)(u >> 32)) << 32 | dpp<CTRL>((uint32_t)u));
}
constexpr int DPP_XOR1 = 0xb1, DPP_XOR2 = 0x4e, DPP_MIRROR8 = 0x141, DPP_MIRROR16 = 0x140;
template <int LANES>
__device__ __forceinline__ double row_sum(double v) {
    static_assert(LANES == 8 || LANES == 16, "");
    v += dpp<DPP_XOR1>(v);
    v += dpp<DPP_XOR2>(v);
    v += dpp<DPP_MIRROR8>(v);
    if (LANES == 16) v += dpp<DPP_MIRROR16>(v);
    return v;
}
__device__ __forceinline__ uint32_t row_max8(uint32_t v) {
    auto larger = [](uint32_t x, uint32_t y) { return x > y ? x : y; };
    v = larger(v, dpp<DPP_XOR1>(v));
    v = larger(v, dpp<DPP_XOR2>(v));
    return larger(v, dpp<DPP_MIRROR8>(v));
}
// The sines and cosines of a token's pairs, made by a lane each and handed round in LDS, the wave's own: a lane needs those of E pairs, and eight (or
// four) lanes need the same.
template <typename T>
struct Turn { T sn, cs; };
template <typename T>
struct Turns {
    Turn<T> of[PAIRS];
    __device__ __forceinline__ void make(const AppendArgs &a, const Angle &angle, int64_t slot) {
        const int pair = lvr_lane();
        if (pair < a.rot / 2) {
            const uint64_t phase = (uint64_t)(int64_t)(a.positions ? angle.position : (int)slot) * angle.turns;
            Turn<T> t;
            if constexpr (sizeof(T) == 8) sincos_turn(phase, t.sn, t.cs);
            else sincos_turn((uint32_t)(phase >> 32), t.sn, t.cs);
            of[pair] = t;
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
};
union WaveTurns {
    Turns<float> f32;
    Turns<double> f64;
};

// 1 / sqrt(sum of squares / 128 + eps).  Squares are summed in 64 bits: those of large bf16 and fp32 values pass the fp32 range.
__device__ __forceinline__ double norm_of(double squares, float eps) {
    const double x = squares * (1. / LVR_D) + (double)eps;
    const double r = __builtin_amdgcn_rsq(x);
    if (x == __builtin_inf()) return 0.;
    return r * __builtin_fma(-0.5 * x * r, r, 1.5);   // the instruction's 2^-26 or so become 2^-50
}
// The sum of squares of what a lane has of a row.  bf16: two products a step, exact in fp32, and sums of 16 values in it; where they leave its range,
// as for all else, in 64 bits.
template <int ELT>
__device__ __forceinline__ double squares_of(u32x4 r0, u32x4 r1) {
    if constexpr (ELT == 2) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w0 = r0[i], w1 = r1[i];
            s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w0), __builtin_bit_cast(bf16x2, w0), s, false);
            s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w1), __builtin_bit_cast(bf16x2, w1), s, false);
        }
        if (!__any(!(s > 0x1p-90f && s < 0x1p120f))) return s;   // (squares below 2^-126 would be 2^-36 of it)
    }
    constexpr int E = 16 / ELT;
    float x[E], y[E];
    elements(r0, x);
    elements(r1, y);
    double squares = 0.;
#pragma unroll
    for (int e = 0; e < E; ++e) squares += (double)x[e] * x[e] + (double)y[e] * y[e];
    return squares;
}
// The norm times a row's values, in fp32 without leaving its range on the way.
struct Normed {
    float r;
    int e;
    __device__ __forceinline__ Normed(double norm) : r((float)__builtin_amdgcn_frexp_mant(norm)), e(__builtin_amdgcn_frexp_exp(norm)) {}
    __device__ __forceinline__ float operator()(float x) const { return __builtin_amdgcn_ldexpf(x, e) * r; }
};
template <int ELT>
__device__ __forceinline__ u32x4 weights_at(const char *w, int at) {
    const uint32_t one = ELT == 2 ? 0x3f803f80u : 0x3f800000u;
    return w ? load_piece(w + at * ELT) : u32x4{one, one, one, one};
}

// Pages in 4 bits.  The least e with A <= 7 * 2^e, A the largest magnitude of 32 values: 7 rounds to 6, the largest code, and 6.99 is no further
// from it than 5 from 4, so that no value is off by more than 2^e, half of the widest gap.  As a scale byte e + 127, held between 7 and 252: all
// products of a code and a scale are normal bf16 values then, and so is what lies between two of them.  (bf16 goes up to 7.97 * 2^125: from 7 * 2^125
// on values become 6 * 2^125, off by up to twice as much, and keys that a norm's weight or a rotation takes further by more.)  Bits of A in, as the
// order of fp32 has them; 255 for infinities and NaN.
__device__ __forceinline__ uint32_t fp4_scale_byte(uint32_t bits) {
    if (bits >= 0x7f800000u) return 255;
    const int s = (int)((bits + 0x1fffffu) >> 23) - 2;   // 7 = 1.75 * 4: past a mantissa of 1.75 the next power of two
    return s < 7 ? 7 : (s > 252 ? 252 : s);
}
// Eight values as codes; rounds to nearest, ties to even, and to 6 what is larger.
__device__ __forceinline__ uint32_t fp4_codes(const float (&x)[8], float scale) {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
}
// A value in 64 bits as an fp32 value that rounds to the same code and scale: cut to 21 bits, the last of which says whether anything was cut.  Beyond
// the range of fp32 its largest number, which has the largest scale and code; below 2^-126, far under the least code, something that small.  `most`
// keeps the largest upper half seen: infinities and NaN are told by it.
__device__ __forceinline__ float sticky(double v, uint32_t &most) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)u, hi = (uint32_t)(u >> 32), mag = hi & 0x7fffffffu;
    most = mag > most ? mag : most;
    int32_t m = (int32_t)mag - ((1023 - 127) << 20);   // exponent and 20 bits, with the bias of fp32
    m = m < 0 ? 0 : (m > (255 << 20) - 1 ? (255 << 20) - 1 : m);
    return __uint_as_float((hi & 0x80000000u) | (uint32_t)m << 3 | (lo < 1 ? lo : 1));
}

// Eight K rows and eight V rows of one token into pages in 4 bits, by one wave; lanes hold pieces as in paged_append_kernel.  K is normed and rotated
// in 64 bits: values beside a border between two codes, which fp32 would leave on either side of it, go to the exact value's but within 2^-49 of the
// border, relative to a pair's size, and the angle's |position| * 2^-64 of a turn.
template <bool NEIGHBOURS, bool NORM>
__device__ __forceinline__ void append_fp4(const AppendArgs &a, const lvr_paged_batch &b, int t, int row, Turns<double> &turns) {
    constexpr int E = 8, LANES = 8;
    const int li = lvr_lane() % LANES;
    const Pieces p = pieces_of<E, NEIGHBOURS>(li, a.rot);
    const bool real = row < a.n_kv;
    if (!real) row = a.n_kv - 1;   // nothing is made of it
    u32x4 k0 = load_piece(a.k + t * a.k_stride + (int64_t)row * (LVR_D * 2) + p.at0 * 2), k1 = load_piece(a.k + t * a.k_stride + (int64_t)row * (LVR_D * 2) + p.at1 * 2);
    u32x4 v0 = load_piece(a.v + t * a.v_stride + (int64_t)row * (LVR_D * 2) + p.at0 * 2), v1 = load_piece(a.v + t * a.v_stride + (int64_t)row * (LVR_D * 2) + p.at1 * 2);
    const Angle angle(a, t);
    u32x4 w0, w1;
    if (NORM) w0 = weights_at<2>(a.k_weight, p.at0), w1 = weights_at<2>(a.k_weight, p.at1);

    const lvr_token at_batch = lvr_find_token(b, t);
    const int seq = at_batch.seq;
    const int64_t slot = at_batch.position;
    if (seq < 0 || seq >= b.n_seqs) return;
    const int page = lvr_page_of(b, seq, slot);
    if (page < 0) return;
    if (a.rot > 0) turns.make(a, angle, slot);

    float x[E], y[E];
    uint32_t most0 = 0, most1 = 0;   // of what is normed or rotated
    elements(k0, x);
    elements(k1, y);
    if (NORM || p.rot0 || p.rot1) {   // (p.rot* differ from lane to lane of a row)
        double norm = 1.;
        float wx[E], wy[E];
        if (NORM) {
            double squares = 0.;
#pragma unroll
            for (int e = 0; e < E; ++e) squares += (double)x[e] * x[e] + (double)y[e] * y[e];
            norm = norm_of(row_sum<LANES>(squares), a.eps);
            elements(w0, wx);
            elements(w1, wy);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const bool second = e >= E / 2;
            float &fu = NEIGHBOURS ? (second ? y : x)[2 * (e % (E / 2))] : x[e];
            float &fz = NEIGHBOURS ? (second ? y : x)[2 * (e % (E / 2)) + 1] : y[e];
            double u = fu, z = fz;
            if (NORM) {
                u *= norm * (double)(NEIGHBOURS ? (second ? wy : wx)[2 * (e % (E / 2))] : wx[e]);
                z *= norm * (double)(NEIGHBOURS ? (second ? wy : wx)[2 * (e % (E / 2)) + 1] : wy[e]);
            }
            if (NEIGHBOURS && second ? p.rot1 : p.rot0) {
                const Turn<double> turn = turns.of[pair_of<E, NEIGHBOURS>(li, e)];
                const double first = u * turn.cs - z * turn.sn;
                z = u * turn.sn + z * turn.cs;
                u = first;
            }
            fu = sticky(u, NEIGHBOURS && second ? most1 : most0);
            fz = sticky(z, NEIGHBOURS && !second ? most0 : most1);
        }
    }

    // the scales of the row's four blocks; a lane's pieces lie in one block each
    const int c0 = p.at0 / 32, c1 = p.at1 / 32;
    auto store = [&](char *pages, const float (&x)[E], const float (&y)[E], bool odd0, bool odd1) {
        uint32_t m0 = odd0 ? 0x7f800000u : 0, m1 = odd1 ? 0x7f800000u : 0, packed = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const uint32_t bx = __float_as_uint(x[e]) & 0x7fffffffu, by = __float_as_uint(y[e]) & 0x7fffffffu;
            m0 = bx > m0 ? bx : m0;
            m1 = by > m1 ? by : m1;
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const uint32_t mine = c0 == c ? (c1 == c && m1 > m0 ? m1 : m0) : (c1 == c ? m1 : 0);
            packed |= fp4_scale_byte(row_max8(mine)) << 8 * c;
        }
        if (!real) return;
        char *codes = pages + lvr_row_at(b, page, row, slot);
        *reinterpret_cast<uint32_t *>(codes + p.at0 / 2) = fp4_codes(x, lvr_fp4_scale(packed >> 8 * c0 & 255));
        *reinterpret_cast<uint32_t *>(codes + p.at1 / 2) = fp4_codes(y, lvr_fp4_scale(packed >> 8 * c1 & 255));
        if (li == 0) *reinterpret_cast<uint32_t *>(pages + lvr_scales_at(b, page, row, slot)) = packed;
    };
    store(a.k_pages, x, y, most0 >= 0x7ff00000u, most1 >= 0x7ff00000u);
    elements(v0, x);
    elements(v1, y);
    store(a.v_pages, x, y, false, false);
}

// A wave takes PER times ROWS rows of one token.  A lane holds two pieces of a row, of E elements each: HALVES: the same one of both
// halves, rotated with each other; NEIGHBOURS: one in each half of the row, rotated within themselves; past the rotated coordinates two that are
// copied.  The lanes of a row touch neighbouring pieces in every access.  A lane needs the sines and cosines of E pairs, for all
// of its rows.  The angle is position times turns per position modulo one turn, which in 64-bit integers is one product with the
// overflow dropped: no far position loses anything.
//
// Bound by HBM where there are tokens enough: 8192 tokens (48 rows each, bf16) 36 us on one axis and 34 on three, 5.6 and 6.0 TB/s read and written;
// 1885 fp32 tokens of 80 rows 24.5 us, 6.3 TB/s.  One token: 4.3 to 4.9 us a call, which the host takes 4.0 us to make; the kernel 2.7, the launch and
// three dependent trips (rows and lengths, table, store).
//
// NORM: rows of K and q are normed first, the squares summed over the row's lanes while the sines are made (8192 such tokens on three axes 38 us, one
// token as without).  FP4 (KT is the type of new rows then): the first waves of a token take K and V, eight heads each, the others q.  Those need the
// largest magnitude of every block after the norm and the rotation, in 64 bits: 8192 tokens of the same heads on one axis 35 us, 101 MB read and 76
// written, 5.0 TB/s.
template <typename KT, bool NEIGHBOURS, int PER, bool STREAM, bool NORM, bool FP4>
__global__ void __launch_bounds__(256) paged_append_kernel(AppendArgs a, lvr_paged_batch b) {
    constexpr int ELT = sizeof(KT) == 4 ? 4 : 2, E = 16 / ELT, LANES = PAIRS / E, ROWS = 64 / LANES;
    __shared__ WaveTurns turns[4];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = lvr_lane(), li = lane % LANES;
    const uint32_t w = blockIdx.x * 4u + wave;
    const int t = (int)(w / (uint32_t)a.groups);
    int group = (int)(w % (uint32_t)a.groups);
    if (t >= b.n_tokens) return;   // the whole wave
    if constexpr (FP4) {
        const int of_kv = (a.n_kv + 7) / 8;
        if (group < of_kv) {
            append_fp4<NEIGHBOURS, NORM>(a, b, t, group * 8 + lane / 8, turns[wave].f64);
            return;
        }
        group -= of_kv;
    }
    const int row0 = (FP4 ? 2 * a.n_kv : 0) + group * (ROWS * PER) + lane / LANES;

    const auto [at0, at1, rot0, rot1] = pieces_of<E, NEIGHBOURS>(li, a.rot);
    u32x4 r0[PER], r1[PER], kw0, kw1, qw0, qw1;
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
    const Angle angle(a, t);
    if (NORM) {
        kw0 = weights_at<ELT>(a.k_weight, at0), kw1 = weights_at<ELT>(a.k_weight, at1);
        qw0 = weights_at<ELT>(a.q_weight, at0), qw1 = weights_at<ELT>(a.q_weight, at1);
    }

    const lvr_token at_batch = lvr_find_token(b, t);
    const int seq = at_batch.seq;
    const int64_t slot = at_batch.position;
    if (seq < 0 || seq >= b.n_seqs) return;
    const int page = lvr_page_of(b, seq, slot);
    float sn[E], cs[E];
    if (a.rot > 0) {
        turns[wave].f32.make(a, angle, slot);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const Turn<float> turn = turns[wave].f32.of[pair_of<E, NEIGHBOURS>(li, e)];   // (of pairs that are none: anything)
            sn[e] = turn.sn;
            cs[e] = turn.cs;
        }
    }
    // The rows were asked for before the token's place and are there by now.  Told so, the compiler waits for nothing between the stores; else each
    // pair of them for the one before (fp32, 8192 tokens 73.2 us without this and 69.9 with it, unrotated 73.0 and 69.6; 2000 tokens of 32 rows 11.2
    // and 12.0).  bf16 gains nothing, norms lose where the last group of rows is a small one (8192 tokens of 10 rows 15.4 and 16.2).
    if (ELT == 4 && !NORM) __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
#pragma unroll
    for (int c = 0; c < PER; ++c) {
        const int row = row0 + c * ROWS;
        const bool of_q = row >= 2 * a.n_kv, of_v = row >= a.n_kv && !of_q;
        if (row >= a.n_rows || (!of_q && page < 0)) continue;
        if (NORM && !of_v) {
            float x[E], y[E], wx[E], wy[E];
            elements(r0[c], x);
            elements(r1[c], y);
            const Normed norm(norm_of(row_sum<LANES>(squares_of<ELT>(r0[c], r1[c])), a.eps));
            elements(of_q ? qw0 : kw0, wx);
            elements(of_q ? qw1 : kw1, wy);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                x[e] = norm(x[e]) * wx[e];
                y[e] = norm(y[e]) * wy[e];
            }
            if (rot0 || rot1) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const bool second = e >= E / 2;
                    if (NEIGHBOURS && !(second ? rot1 : rot0)) continue;
                    float &u = NEIGHBOURS ? (second ? y : x)[2 * (e % (E / 2))] : x[e];
                    float &z = NEIGHBOURS ? (second ? y : x)[2 * (e % (E / 2)) + 1] : y[e];
                    const float first = u * cs[e] - z * sn[e];
                    z = u * sn[e] + z * cs[e];
                    u = first;
                }
            }
            r0[c] = piece_of(x);
            r1[c] = piece_of(y);
        } else if ((rot0 || rot1) && !of_v) {
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
// wgs: the workgroups of the launch, which lie behind the arguments otherwise, in a line of memory more (2000 keys of 8 heads 4.94 us so, 4.81 as
// it is).
template <typename KT, bool STREAM>
__global__ void __launch_bounds__(256) paged_gather_kernel(const char *k_pages, const char *v_pages, char *K, char *V, int64_t n,
                                                           int32_t n_kv, int32_t wgs, lvr_paged_batch b) {
    constexpr int ROW = LVR_D * (sizeof(KT) == 4 ? 4 : 2), LANES = ROW / 16, ROWS = 64 / LANES, N = 16 / ROWS;
    const int lane = lvr_lane(), r0 = lane / LANES, at = lane % LANES * 16;
    const int64_t groups = (n + 15) / 16, total = groups * n_kv * b.n_seqs;
    const int64_t step = (int64_t)wgs * 4;
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

// Pages in 4 bits, as rows of bf16.  Four lanes' worth of codes are one block: a lane takes eight of them to 16 bytes.  Bound by the store of rows
// that are 3.8 times as long as what is read: 32768 keys of 8 heads 30 us (134 MB written, 36 read), 5.7 TB/s.
template <bool STREAM>
__global__ void __launch_bounds__(256) paged_gather_fp4_kernel(const char *k_pages, const char *v_pages, char *K, char *V, int64_t n,
                                                               int32_t n_kv, int32_t wgs, lvr_paged_batch b) {
    constexpr int ROW = LVR_D * 2, N = 4;
    const int lane = lvr_lane(), r0 = lane / 16, dword = lane % 16;
    const int64_t groups = (n + 15) / 16, total = groups * n_kv * b.n_seqs;
    const int64_t step = (int64_t)wgs * 4;
    for (int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); w < total; w += step) {
        const int64_t bh = w / groups;
        const int64_t row0 = (w - bh * groups) * 16;
        const int seq = (int)(bh / n_kv), head = (int)(bh - (int64_t)seq * n_kv);
        int64_t end = b.seq_len[seq];
        if (end > n) end = n;
        if (row0 >= end) continue;
        const int page = lvr_page_of(b, seq, row0);   // the table ends with a page, so all 16 rows are in it or none
        if (page < 0) continue;
        const int64_t from = lvr_row_at(b, page, head, row0) + dword * 4, scales = lvr_scales_at(b, page, head, row0) + dword / 4;
        const int64_t to = (bh * n + row0) * ROW + dword * 16;
        const int last = (int)(end - row0 < 16 ? end - row0 : 16) - 1;
        uint32_t k[N], v[N], ks[N], vs[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = 4 * i + r0 < last ? 4 * i + r0 : last;   // past the end: the last row once more
            const int64_t c = r * b.row_stride, s = c / (LVR_FP4_CODES / LVR_FP4_SCALES);
            k[i] = *reinterpret_cast<const uint32_t *>(k_pages + from + c);
            v[i] = *reinterpret_cast<const uint32_t *>(v_pages + from + c);
            ks[i] = (uint8_t)k_pages[scales + s];
            vs[i] = (uint8_t)v_pages[scales + s];
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (4 * i + r0 <= last) {
                store_piece<STREAM>(K + to + (4 * i + r0) * ROW, __builtin_bit_cast(u32x4, lvr_fp4_values(k[i], lvr_fp4_scale(ks[i]))));
                store_piece<STREAM>(V + to + (4 * i + r0) * ROW, __builtin_bit_cast(u32x4, lvr_fp4_values(v[i], lvr_fp4_scale(vs[i]))));
            }
    }
}

// Bytes of an element of new rows, queries and outputs.
inline int64_t element(const lvr_paged_config &c) { return c.kv_dtype == LVR_F32 ? 4 : 2; }
// Pages in 4 bits: bytes of codes, and of codes and scales, of a page.
inline int64_t fp4_codes_of_page(const lvr_paged_config &c) { return (int64_t)c.n_kv_heads * c.page_size * LVR_FP4_CODES; }
inline int64_t fp4_page(const lvr_paged_config &c) { return (int64_t)c.n_kv_heads * c.page_size * (LVR_FP4_CODES + LVR_FP4_SCALES); }

int check_config(const lvr_paged_config *c) {
    if (!c) return LVR_E_INVALID;
    if (c->n_q_heads <= 0 || c->n_kv_heads <= 0 || c->n_q_heads % c->n_kv_heads != 0) return LVR_E_INVALID;
    const bool fp4 = c->kv_dtype == LVR_FP4;
    if (c->kv_dtype != LVR_BF16 && c->kv_dtype != LVR_F32 && !fp4) return LVR_E_INVALID;
    if (!(c->scale >= 0.f) || isinf(c->scale)) return LVR_E_INVALID;
    if (c->page_size <= 0 || c->n_pages <= 0) return LVR_E_INVALID;
    if (c->rot_dim < 0 || c->rot_dim > c->head_dim || c->rot_dim % 2) return LVR_E_INVALID;
    if (c->rot_dim > 0 && (c->rot_axes < 1 || c->rot_axes > 4)) return LVR_E_INVALID;
    if (c->rot_pairs != LVR_ROT_HALVES && c->rot_pairs != LVR_ROT_NEIGHBOURS) return LVR_E_INVALID;
    const int64_t per16 = fp4 ? 16 : (c->kv_dtype == LVR_BF16 ? 8 : 4);   // strides of pages in 4 bits are bytes
    for (int i = 0; i < 3; ++i)
        if (c->page_strides[i] < 0 || c->page_strides[i] % per16 || c->page_strides[i] > (int64_t)1 << 40) return LVR_E_INVALID;
    if (c->page_strides[2] < (fp4 ? c->head_dim / 2 : c->head_dim)) return LVR_E_INVALID;
    if (c->head_dim != LVR_D || c->rot_dim % 16 != 0) return LVR_E_UNSUPPORTED;
    if (c->n_q_heads > 1024 || c->n_kv_heads > 256) return LVR_E_UNSUPPORTED;
    if (c->page_size < 16 || c->page_size > 65536 || (c->page_size & (c->page_size - 1))) return LVR_E_UNSUPPORTED;
    if (c->n_pages > (int64_t)1 << 30) return LVR_E_UNSUPPORTED;
    if (c->page_strides[2] > (int64_t)1 << 24) return LVR_E_UNSUPPORTED;   // 16 rows of a page are told apart by 32-bit offsets
    if (fp4) {
        if (c->n_pages > 1 && c->page_strides[0] < fp4_page(*c)) return LVR_E_INVALID;
        const bool heads_first = c->page_strides[2] == LVR_FP4_CODES && (c->page_strides[1] == (int64_t)LVR_FP4_CODES * c->page_size || c->n_kv_heads == 1);
        const bool tokens_first = c->page_strides[1] == LVR_FP4_CODES && c->page_strides[2] == (int64_t)LVR_FP4_CODES * c->n_kv_heads;
        if (!heads_first && !tokens_first) return LVR_E_UNSUPPORTED;
    }
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
    const int64_t elt = pc->cfg.kv_dtype == LVR_FP4 ? 1 : element(pc->cfg);
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
    b->scales = pc->cfg.kv_dtype == LVR_FP4 ? fp4_codes_of_page(pc->cfg) : 0;
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

// lvr_paged_append and lvr_paged_norm_append
int append(lvr_paged *pc, void *k_pages, void *v_pages, const void *k_new, const void *v_new, const void *q, void *q_out, const int64_t strides[3],
           bool norm, const void *q_weight, const void *k_weight, float eps, const int32_t *positions, const int32_t *seq_start, const int32_t *seq_len,
           const int32_t *table, int64_t table_width, int64_t n_seqs, int64_t n_tokens, void *stream) {
    lvr_paged_batch b;
    const int rc = check_batch(pc, k_pages, v_pages, seq_start, true, seq_len, table, table_width, n_seqs, n_tokens, &b);
    if (rc != LVR_OK) return rc;
    if (!q != !q_out) return LVR_E_INVALID;
    if (norm && (!(eps >= 0.f) || isinf(eps))) return LVR_E_INVALID;
    if (n_tokens == 0 || n_seqs == 0) return LVR_OK;
    if (!k_new || !v_new || !strides) return LVR_E_INVALID;
    const lvr_paged_config &c = pc->cfg;
    const int64_t elt = element(c);
    if (!token_stride_ok(strides[0], c.n_kv_heads, elt) || !token_stride_ok(strides[1], c.n_kv_heads, elt)) return LVR_E_INVALID;
    if (q && !token_stride_ok(strides[2], c.n_q_heads, elt)) return LVR_E_INVALID;
    if (q && q == q_out && strides[2] != (int64_t)c.n_q_heads * LVR_D) return LVR_E_INVALID;
    if (!aligned16(k_new) || !aligned16(v_new) || !aligned16(q) || !aligned16(q_out) || !aligned4(positions)) return LVR_E_INVALID;
    if (!aligned16(q_weight) || !aligned16(k_weight)) return LVR_E_INVALID;
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
    a.q_weight = static_cast<const char *>(q_weight);
    a.k_weight = static_cast<const char *>(k_weight);
    a.eps = eps;
    // Where there are tokens enough to fill the device a wave takes up to 24 rows, for which it makes sines and cosines once
    const bool fp4 = c.kv_dtype == LVR_FP4;
    const int rows = elt == 2 ? 8 : 4;   // a wave's at a time
    const bool many = n_tokens * a.n_rows >= APPEND_MANY;
    const int per_wave = many ? 24 : rows;
    a.groups = fp4 ? (c.n_kv_heads + 7) / 8 + (a.n_rows - 2 * c.n_kv_heads + per_wave - 1) / per_wave : (a.n_rows + per_wave - 1) / per_wave;
    const dim3 grid((unsigned)((n_tokens * a.groups + 3) / 4));
    hipStream_t st = static_cast<hipStream_t>(stream);
#define LVR_APPEND_NORM(KT, N, PER, S, FP4)                                                                                         \
    do {                                                                                                                            \
        if (norm) hipLaunchKernelGGL((paged_append_kernel<KT, N, PER, S, true, FP4>), grid, dim3(256), 0, st, a, b);                \
        else hipLaunchKernelGGL((paged_append_kernel<KT, N, PER, S, false, FP4>), grid, dim3(256), 0, st, a, b);                    \
    } while (0)
#define LVR_APPEND_PER(KT, N, PER, FP4)                           \
    do {                                                          \
        if (many) LVR_APPEND_NORM(KT, N, PER, true, FP4);         \
        else LVR_APPEND_NORM(KT, N, 1, false, FP4);               \
    } while (0)
#define LVR_APPEND(KT, PER, FP4)                                                       \
    do {                                                                               \
        if (c.rot_pairs == LVR_ROT_NEIGHBOURS) LVR_APPEND_PER(KT, true, PER, FP4);     \
        else LVR_APPEND_PER(KT, false, PER, FP4);                                      \
    } while (0)
    if (fp4) LVR_APPEND(lvr_bf16_t, 3, true);
    else if (elt == 2) LVR_APPEND(lvr_bf16_t, 3, false);
    else LVR_APPEND(lvr_f32_t, 6, false);
#undef LVR_APPEND
#undef LVR_APPEND_PER
#undef LVR_APPEND_NORM
    LVR_HIP(hipGetLastError());
    return LVR_OK;
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
    return append(pc, k_pages, v_pages, k_new, v_new, q, q_out, strides, false, nullptr, nullptr, 0.f, positions, seq_start, seq_len, table,
                  table_width, n_seqs, n_tokens, stream);
}

int lvr_paged_norm_append(lvr_paged *pc, void *k_pages, void *v_pages, const void *k_new, const void *v_new, const void *q, void *q_out,
                          const int64_t strides[3], const void *q_weight, const void *k_weight, float eps, const int32_t *positions,
                          const int32_t *seq_start, const int32_t *seq_len, const int32_t *table, int64_t table_width, int64_t n_seqs,
                          int64_t n_tokens, void *stream) {
    return append(pc, k_pages, v_pages, k_new, v_new, q, q_out, strides, true, q_weight, k_weight, eps, positions, seq_start, seq_len, table,
                  table_width, n_seqs, n_tokens, stream);
}

int lvr_paged_attention(lvr_paged *pc, const void *k_pages, const void *v_pages, const void *q, int64_t q_token_stride,
                        const int32_t *seq_start, const int32_t *seq_len, const int32_t *table, int64_t table_width,
                        int64_t n_seqs, int64_t n_tokens, int32_t window, void *out, void *stream) {
    return lvr_paged_sink_attention(pc, k_pages, v_pages, q, q_token_stride, seq_start, seq_len, table, table_width, n_seqs, n_tokens, window, 0,
                                    out, stream);
}

int lvr_paged_sink_attention(lvr_paged *pc, const void *k_pages, const void *v_pages, const void *q, int64_t q_token_stride,
                             const int32_t *seq_start, const int32_t *seq_len, const int32_t *table, int64_t table_width,
                             int64_t n_seqs, int64_t n_tokens, int32_t window, int32_t sinks, void *out, void *stream) {
    lvr_paged_batch b;
    const int rc = check_batch(pc, k_pages, v_pages, seq_start, true, seq_len, table, table_width, n_seqs, n_tokens, &b);
    if (rc != LVR_OK) return rc;
    if (window < 0 || sinks < 0) return LVR_E_INVALID;
    if (n_tokens == 0 || n_seqs == 0) return LVR_OK;
    const int64_t elt = element(pc->cfg);
    if (!q || !out || q == out || !aligned16(q) || !aligned16(out)) return LVR_E_INVALID;
    if (!token_stride_ok(q_token_stride, pc->cfg.n_q_heads, elt)) return LVR_E_INVALID;
    LVR_HIP(lvr_launch_paged_attention(pc, b, k_pages, v_pages, q, q_token_stride * elt, window, sinks, out, static_cast<hipStream_t>(stream)));
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
    const bool stream_out = n * n_kv * n_seqs * LVR_D * element(pc->cfg) >= GATHER_STREAM;
#define LVR_GATHER(...)                                                                                                               \
    hipLaunchKernelGGL((__VA_ARGS__), dim3((unsigned)wgs), dim3(256), 0, st, static_cast<const char *>(k_pages),                      \
                       static_cast<const char *>(v_pages), static_cast<char *>(K_out), static_cast<char *>(V_out), n, n_kv, (int32_t)wgs, b)
    if (pc->cfg.kv_dtype == LVR_FP4) {
        if (stream_out) LVR_GATHER(paged_gather_fp4_kernel<true>);
        else LVR_GATHER(paged_gather_fp4_kernel<false>);
    } else if (pc->cfg.kv_dtype == LVR_BF16) {
        if (stream_out) LVR_GATHER(paged_gather_kernel<lvr_bf16_t, true>);
        else LVR_GATHER(paged_gather_kernel<lvr_bf16_t, false>);
    } else {
        if (stream_out) LVR_GATHER(paged_gather_kernel<lvr_f32_t, true>);
        else LVR_GATHER(paged_gather_kernel<lvr_f32_t, false>);
    }
#undef LVR_GATHER
    LVR_HIP(hipGetLastError());
    return LVR_OK;
}

}  // extern "C"
