// How lvr_paged_attention divides a batch into pieces of work: the launch's part on the host, and what every wave works out on the device.
// Compiles for the host as well, with a wave of one lane.
#pragma once
#include "paged.h"

namespace {

// Pieces of work a launch aims at, over all KV heads: of tiles of 16 rows alone, and where there are tiles of 128 rows.  A piece costs a
// workgroup's start and, where its tile is cut, a partial result to be written and read; too few leave compute units idle at the end.
// us with 256 / 512 / 1024 pieces (8 KV heads), tiles of 16 rows: one sequence of 32768 keys 30 / 34 / 38, four ragged ones (32 tiles)
// 37 / 34 / 32, eight 76 / 63 / 62, 48 of them 428 / 375 / 381, in 4 bits 132 / 115 / 116; tiles of 128: 32 tokens over 131072 keys
// 126 / 139 / 176, 512 of 8192 99 / 85 / 98, 1000 of 12000 250 / 202 / 215, 1000 of 12000 beside 31 single tokens 290 / 286 / 274, fp32 prompt
// of 2048 394 / 317 / 344.
constexpr int ROWS16_PIECES = 512, ROWS16_PIECES_FEW = 256, MIXED_PIECES = 512;
constexpr int FEW_TILES = 32;   // sequences times KV heads up to which a batch of single tokens makes few pieces
// Keys of the shortest run.  us with 64 / 128 / 256 / 512: one token over 1024 keys 8.5 / 9.2 / 10.2 / 12.1, over 2048 8.7 / 9.4 / 10.3 / 12.3,
// in 4 bits 8.7 / 8.6 / 9.1 / 10.3, over 8192 13.0 / 13.1 / 13.0 / 14.0; four prompts of 1024 64.5 / 65.6 / 65.7 / 64.3.
constexpr int MIN_RUN = 64;
// Rows of a sequence up to which it is taken in tiles of 16.  A wave of a 128-row tile works on 32 of them however many there are, and on
// fp32 takes so long that reading the keys again costs less (us, 64 rows over 32768 keys: bf16 55 in a tile of 128 / 51 in four of 16,
// eight such sequences 200 / 341 and of 4096 keys 42 / 57; fp32 174 / 107, 1025 / 771 and 160 / 117).  The rule goes by the rows alone, and for
// bf16 takes the side on which many sequences gain.
constexpr int NARROW_BF16 = 32, NARROW_F32 = 64;
// Of all sequences together, on pages in 4 bits (16 tokens, 32 heads on 8, over 32768 keys: 49 us in a tile of 128, 28 in four of 16; 9 tokens over
// 3000 21 and 12).
constexpr int NARROW_FP4_ALONE = 64;
// Keys up to which a tile of 16 rows is not cut, on pages in 4 bits and on bf16 ones with first keys: a workgroup takes 0.6 us for 128 of them in
// 4 bits, merging takes three.  us uncut / in runs of 64: one token over 256 keys in 4 bits 5.7 / 8.2, 512 6.9 / 8.3, 16 of them over 512 7.4 / 10.4;
// bf16, a window of 64 with four first keys 7.5 / 9.2.  fp32 goes either way (11.4 / 11.5, over 200 keys 11.5 / 10.8, 16 sequences 12.8 / 16.5) and is
// cut.  So is bf16 without first keys beyond 64 keys, as it was before there was this rule; it would gain as much by it (one token over 100 keys
// 5.7 / 8.4, 200 7.0 / 8.4, 256 6.6 / 8.2).
constexpr int UNCUT_FP4 = 512, UNCUT_BF16 = 256;
constexpr int WIDE_ROOM = 2 * MIXED_PIECES, NARROW_ROOM = 3 * (ROWS16_PIECES > MIXED_PIECES ? ROWS16_PIECES : MIXED_PIECES);   // partial results

struct AttnArgs {
    const char *k_pages, *v_pages, *q;
    char *out;
    int64_t q_stride;    // bytes per token
    int32_t n_kv, G, window;
    uint32_t g_mul;      // row / G = row * g_mul >> g_shift
    int32_t g_shift;
    float unit;          // sigma * log2 e
    int32_t narrow;      // rows of a sequence up to which it is taken in tiles of 16
    int32_t target;      // pieces of work to make of the batch per KV head; 0: tiles are not cut
    float *part;
    uint32_t *ticket;    // a line for each slot of a cut tile
    int32_t sinks;       // first keys that stay visible beside a window; 0 without one.  window + sinks is at most 2^30
    int32_t uncut;       // keys that a tile of 16 rows may see and is not cut
};

// A piece of work: a tile of TM packed rows of one sequence against a run of the keys they see.
struct Tile {
    int height;                // TM: 16 or 128
    int seq, row0, rows;       // first packed row within the sequence; rows of the sequence
    int first_token;           // of the sequence, in the packed arrays
    int pos0;                  // position of the sequence's first new token
    int lo, hi;                // keys that any row of the tile sees: lo .. hi - 1, and those before a.sinks
    int begin, end;            // the run, of places: place x is key x, or x + shift from `fold` on
    int fold, shift;           // (both multiples of 64: where the first keys and the window's lie apart, the places skip what is between)
    int split, splits;         // which run of how many
    int slot;                  // where its partial result goes, if there is more than one run
};

// The division of the batch stands before everything else a workgroup does, in code that is fetched anew by every launch: it is
// kept short.  a / b is a handful of instructions less where it may be off by one,
template <typename WAVE>
__host__ __device__ __forceinline__ int about(int a, int b) { return (int)((float)a * WAVE::reciprocal((float)b)); }
// for quotients below 2^21 one comparison either way puts that right,
template <typename WAVE>
__host__ __device__ __forceinline__ int divide_small(int a, int b) {
    int q = about<WAVE>(a, b);
    const int r = a - q * b;
    q += r >= b;
    q -= r < 0;
    return q;
}
// and for the query heads of a KV head the host has the reciprocal (rows are fewer than 2^28).
__host__ __device__ __forceinline__ int token_of(const AttnArgs &a, int row) { return (int)((uint64_t)(uint32_t)row * a.g_mul >> a.g_shift); }

// How a batch is divided into pieces, for one KV head.  The host knows neither how many tokens a sequence brings nor how many keys it
// holds, so every workgroup works it out for itself, each wave on its own, a lane to a sequence (64 at a time).  MIXED: sequences of
// up to a.narrow rows are taken in tiles of 16, others in tiles of 128; else all in tiles of 16.
//
// A sequence's tiles are cut into runs of keys of one length, as many as make about `target` pieces of the batch (but none under
// MIN_RUN keys; target 0: no cuts).  L is the keys of all tiles over target, where a tile sees half of the sequence's own new keys.
// Tiles of 128 rows are cut into span / L runs, rounded, so that equal ones fill whole rounds of workgroups; beside them tiles of 16 rows,
// whose partial results are small, into runs of a quarter of that.  Without tiles of 128 rows the number is rounded up (but see level).  There is
// room for the partial results of 2 * target pieces of cut 128-row tiles and for 3 * target pieces of cut tiles altogether, and the
// launch has as many workgroups beside one for each tile: should there be more, L grows until there are not (prompts of a few hundred tokens
// get there with the shortest runs).
//
// A batch of up to 64 sequences stays in registers.  Of a larger one every wave reads the lengths anew, to divide it and to find its piece: single
// tokens over 64 keys, 8 KV heads: 64 sequences 7.3 us, 256 25, 1024 173, 4096 1806 (the read of their keys: 2.8, 11, 45, 180); over 2048 keys 256
// sequences 360 us and 1024 1441, the read's rate.
//
// SINKS: a.sinks may be more than 0; UNCUT: a.uncut may be (without them the code has nothing of that).
template <bool MIXED, typename WAVE, bool SINKS = true, bool UNCUT = true>
struct Division {
    const AttnArgs &a;
    const lvr_paged_batch &b;
    int G, window, narrow, L;
    int n_wide;                              // pieces of 128-row tiles, which come first
    bool any_wide;
    static constexpr int LANES = WAVE::LANES;
    static constexpr int NO_CUTS = 1 << 30;   // an L
    int s0, s1, n, tiles, span;              // this lane's sequence
    int run = 0, runs = 1;

    __host__ __device__ __forceinline__ bool wide(int rows) const { return MIXED && rows > narrow; }
    __host__ __device__ __forceinline__ void look(int i) {
        s0 = s1 = n = tiles = span = 0;
        if (i < b.n_seqs) {   // whatever the arrays hold, rows stay within the packed arrays and the table
            s0 = b.seq_start[i];
            s1 = b.seq_start[i + 1];
            n = b.seq_len[i];
            s0 = s0 < 0 ? 0 : (s0 > b.n_tokens ? b.n_tokens : s0);
            s1 = s1 < s0 ? s0 : (s1 > b.n_tokens ? b.n_tokens : s1);
            n = n < 0 ? 0 : (n > 1 << 30 ? 1 << 30 : n);
            const int rows = (s1 - s0) * G;
            tiles = wide(rows) ? (rows + 127) / 128 : (rows + 15) / 16;
            const int reach = window ? window + 128 + (SINKS ? (a.sinks + 63) & ~63 : 0) : n;   // keys a tile can see, at most
            span = n < reach ? n : reach;
            if (span > b.table_width << b.page_shift) span = b.table_width << b.page_shift;
            if (span < 1) span = 1;
        }
    }
    __host__ __device__ __forceinline__ bool is_wide() const { return wide((s1 - s0) * G); }
    __host__ __device__ __forceinline__ void cut() {
        runs = 1;
        if (L == NO_CUTS || (UNCUT && span <= a.uncut && !is_wide())) return;
        int L1 = L;
        if (MIXED && any_wide && !is_wide()) L1 = L1 > 4 * MIN_RUN ? L1 >> 2 : (L1 < MIN_RUN ? L1 : MIN_RUN);
        if (MIXED) {
            runs = about<WAVE>(span + (is_wide() ? L1 >> 1 : L1 - 1), L1);
            if (runs < 1) runs = 1;
        } else {   // rounded up, and never more than that
            runs = about<WAVE>(span - 1, L1) + 1;
            runs -= (runs - 1) * L1 >= span;
        }
        run = (about<WAVE>(span, runs) + 64) & ~63;   // the last run takes what is left, whatever was rounded
    }
    // Sequences of one tile each that all go into as many runs: where rounding up made more pieces than wanted, as many as are wanted at most.  Pieces
    // of one length that pass a whole round by a few end late (us rounded up / so, 8 KV heads: 12 sequences of 8192 keys bf16 88 / 78, 4 bits 31 / 25.5,
    // fp32 165 / 145; 20 of 4096 73 / 66; 5 of 8192 43 / 37.5; 3 of them 26.8 / 22.3).
    __host__ __device__ __forceinline__ void level(int target) {
        const uint64_t with = WAVE::ballot(tiles == 1);
        if (with == 0) return;
        const int r = WAVE::of(runs, __builtin_ctzll(with)), count = __builtin_popcountll(with);
        if (r * count <= target || WAVE::any(tiles > 1 || (tiles == 1 && runs != r))) return;
        const int less = divide_small<WAVE>(target, count);
        if (less < 2) return;
        runs = less;
        run = (about<WAVE>(span, runs) + 64) & ~63;
    }
    __host__ __device__ __forceinline__ Division(const AttnArgs &args, const lvr_paged_batch &bt) : a(args), b(bt), G(a.G), window(a.window), narrow(a.narrow) {}
    // false: seq_start is not ascending, no piece is where another expects it
    __host__ __device__ __forceinline__ bool divide(int target) {
        float keys = 0.f, tokens = 0.f;
        any_wide = false;
        for (int i0 = 0; i0 < b.n_seqs; i0 += LANES) {
            look(i0 + WAVE::lane());
            const int own = (s1 - s0 < span ? s1 - s0 : span) / 2;   // (new tokens past the table bring no keys)
            tokens += (float)(s1 - s0);
            any_wide |= WAVE::any(is_wide());
            keys += (float)tiles * (float)(window || !MIXED ? span : span - own);
        }
        if (b.n_seqs > 1) {
            if (WAVE::sum(tokens) > (float)b.n_tokens) return false;   // whole numbers below 2^24 where it matters
            keys = WAVE::sum(keys);
        } else {
            keys = WAVE::of_first(keys);
        }
        L = NO_CUTS;
        if (target > 0) {
            const float want = keys * 1.001f / (float)target;   // (more than what the sum was rounded by)
            L = want < (float)MIN_RUN ? MIN_RUN : (want > 1e9f ? NO_CUTS : ((int)want + 63) & ~63);
        }
        if (!MIXED) {   // at most target pieces more than tiles, and at most 2 * target of cut tiles, since L is all keys over target
            n_wide = 0;
            if (b.n_seqs <= LANES) {
                cut();
                level(target);
            }
            return true;
        }
        for (;; L = L < 1 << 28 ? (L + L / 2 + 63) & ~63 : NO_CUTS) {   // by half and never by less than 64: some 38 steps at most
            int cut_wide = 0, cut_narrow = 0;
            n_wide = 0;
            for (int i0 = 0; i0 < b.n_seqs; i0 += LANES) {
                if (b.n_seqs > LANES) look(i0 + WAVE::lane());
                cut();
                const int cut_here = runs > 1 ? tiles * runs : 0;
                n_wide += WAVE::of(WAVE::inclusive_sum(is_wide() ? tiles * runs : 0), LANES - 1);
                cut_wide += WAVE::of(WAVE::inclusive_sum(is_wide() ? cut_here : 0), LANES - 1);
                cut_narrow += WAVE::of(WAVE::inclusive_sum(is_wide() ? 0 : cut_here), LANES - 1);
            }
            if (cut_wide <= 2 * target && cut_wide + cut_narrow <= 3 * target) break;   // as it is at the latest without cuts
        }
        return true;
    }
    // Piece x, or for CUT tile x of the 128-row tiles that are cut (its first run).  Long pieces come first: those of 128-row tiles, of a
    // sequence's tiles the last ones, and the first runs of all of them before the second ones: a tile's last run is short, and
    // workgroups that go to one compute unit lie a fixed number apart (fp32 prompt of 2048 tokens, tile by tile 464 us).
    template <bool CUT>
    __host__ __device__ __forceinline__ bool locate(int x, Tile &t) {
        int before = 0, cut_before = 0;
        const bool in_wide = CUT || x < n_wide;
        if (!in_wide) x -= n_wide;
        for (int i0 = 0; i0 < b.n_seqs; i0 += LANES) {
            if (b.n_seqs > LANES) {
                look(i0 + WAVE::lane());
                cut();
            }
            const int pieces = is_wide() == in_wide ? tiles * runs : 0, of_cut = runs > 1 ? pieces : 0;
            const int count = CUT ? (of_cut ? tiles : 0) : pieces;
            const int upto = before + WAVE::inclusive_sum(count);
            const int cut_upto = cut_before + WAVE::inclusive_sum(of_cut);
            const uint64_t past = WAVE::ballot(upto > x);
            if (past) {
                const int at = __builtin_ctzll(past);
                auto of = [&](int v) { return WAVE::of(v, at); };
                const int seq_runs = of(runs), seq_run = of(run);
                const int seq_tiles = of(tiles), k = x - of(upto - count);   // which of the sequence's pieces, run by run
                t.split = CUT || seq_runs == 1 ? 0 : divide_small<WAVE>(k, seq_tiles);
                const int from_last = k - t.split * seq_tiles;
                t.slot = of(cut_upto - of_cut) + from_last * seq_runs + t.split;
                t.seq = i0 + at;
                const int first = of(s0), tokens = of(s1) - first;
                t.first_token = first;
                t.rows = tokens * G;
                t.height = wide(t.rows) ? 128 : 16;
                t.row0 = (seq_tiles - 1 - from_last) * t.height;
                t.pos0 = of(n) - tokens;
                const int last_row = (t.row0 + t.height < t.rows ? t.row0 + t.height : t.rows) - 1;
                t.hi = t.pos0 + token_of(a, last_row) + 1;
                if (t.hi > b.table_width << b.page_shift) t.hi = b.table_width << b.page_shift;
                t.lo = window ? t.pos0 + token_of(a, t.row0) - window + 1 : 0;
                if (t.lo < 0) t.lo = 0;
                int from = t.lo & ~63, to = t.hi;
                t.fold = t.shift = 0;
                if (SINKS && a.sinks) {
                    t.fold = (a.sinks + 63) & ~63;
                    if (from > t.fold) {
                        t.shift = from - t.fold;
                        to = to > from ? to - t.shift : (to < t.fold ? to : t.fold);
                    }
                    from = 0;
                }
                t.splits = 1;
                if (seq_runs > 1 && to > from) {
                    t.splits = about<WAVE>(to - from - 1, seq_run) + 1;   // the same for all pieces of the tile
                    if (t.splits > seq_runs) t.splits = seq_runs;
                }
                if (t.split >= t.splits) return false;   // a run past what this tile sees
                t.begin = from + t.split * seq_run;
                t.end = t.split + 1 < t.splits ? t.begin + seq_run : to;
                return true;
            }
            before = WAVE::of(upto, LANES - 1);
            cut_before = WAVE::of(cut_upto, LANES - 1);
        }
        return false;
    }
};

struct PagedLaunch {
    bool mixed;
    int64_t pieces;   // workgroups per KV head: at least as many as the division makes pieces
};
// Everything of `a` that the division reads.  In: a.window and a.sinks as the call has them (0 or more).  No sequence is longer than 2^30 keys: a
// window that with the first keys reaches as far hides nothing and is none, and without a window there are no first keys.
inline PagedLaunch paged_launch(AttnArgs &a, const lvr_paged_batch &b, int n_q, int n_kv, bool bf16, bool fp4 = false) {
    a.n_kv = n_kv;
    a.G = n_q / n_kv;
    a.g_shift = 28;
    while (1 << (a.g_shift - 28) < a.G) ++a.g_shift;
    a.g_mul = (uint32_t)((((uint64_t)1 << a.g_shift) + a.G - 1) / a.G);
    if ((int64_t)a.window + a.sinks >= 1 << 30) a.window = 0;
    if (!a.window) a.sinks = 0;
    a.uncut = fp4 ? UNCUT_FP4 : (bf16 && a.sinks ? UNCUT_BF16 : 0);
    const int64_t rows = (int64_t)b.n_tokens * a.G;
    a.narrow = bf16 && !(fp4 && rows <= NARROW_FP4_ALONE) ? NARROW_BF16 : NARROW_F32;
    if (b.n_tokens <= b.n_seqs || rows <= a.narrow) {
        a.target = (b.n_seqs * a.n_kv <= FEW_TILES ? ROWS16_PIECES_FEW : ROWS16_PIECES) / a.n_kv;   // n_kv is at most 256
        return {false, rows / 16 + b.n_seqs + a.target};
    }
    a.target = MIXED_PIECES / a.n_kv;
    // tiles enough to fill the device without cuts, or none longer than the shortest run
    if (rows / 128 * a.n_kv >= 8 * MIXED_PIECES || b.table_width <= MIN_RUN >> b.page_shift) a.target = 0;
    // tiles: a sequence's rows over 128 and one more, or at most narrow / 16
    return {true, rows / 128 + (int64_t)(a.narrow / 16) * b.n_seqs + 3 * a.target};
}

}  // namespace
