"""How the attention over pages divides a batch, with a wave of 64 lanes on the host: what the lanes of a wave tell each other (which of them has a
piece, whether all sequences go into as many runs) is part of the division, and a wave of one lane has none of it."""
import os
import random
import subprocess

import pytest

PROGRAM = r'''
#include <setjmp.h>
#include <ucontext.h>

#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <vector>
#include "paged_division.h"

// 64 lanes that run in turn, each until it has said something: what a lane says, it hears of all others when its turn comes again.  Two rows of what was
// said, since a lane may be a word ahead of the next one.
constexpr int N = 64;
static struct { ucontext_t start; jmp_buf at; std::vector<char> stack; bool started, done; } fiber[N];
static int current;
static jmp_buf back;
static double said[2][N];
static int words[N];
static void (*body)(int lane);
static void begin() {
    body(current);
    fiber[current].done = true;
    if (current == N - 1) _longjmp(back, 1);
    ++current;
    if (fiber[current].started) _longjmp(fiber[current].at, 1);
    fiber[current].started = true;
    setcontext(&fiber[current].start);
}
static void run(void (*f)(int)) {
    body = f;
    memset(words, 0, sizeof words);
    for (auto &x : fiber) {
        x.stack.resize(1 << 16);
        x.started = x.done = false;
        getcontext(&x.start);
        x.start.uc_stack.ss_sp = x.stack.data();
        x.start.uc_stack.ss_size = x.stack.size();
        x.start.uc_link = nullptr;
        makecontext(&x.start, begin, 0);
    }
    current = 0;
    fiber[0].started = true;
    if (!_setjmp(back)) setcontext(&fiber[0].start);
}
static const double *say(double v) {
    const int me = current, row = words[me]++ & 1;
    said[row][me] = v;
    if (!_setjmp(fiber[me].at)) {
        current = (me + 1) % N;
        if (fiber[current].done) { printf("a lane ended before the others\n"); exit(1); }
        if (fiber[current].started) _longjmp(fiber[current].at, 1);
        fiber[current].started = true;
        setcontext(&fiber[current].start);
    }
    return said[row];
}
static float off;   // how far the device's reciprocal is off the exact one, relative (it is good to a unit of the last place)
struct Lanes {
    static constexpr int LANES = N;
    static int lane() { return current; }
    static uint64_t ballot(bool v) {
        const double *x = say(v);
        uint64_t r = 0;
        for (int i = 0; i < N; ++i) r |= (uint64_t)(x[i] != 0) << i;
        return r;
    }
    static bool any(bool v) { return ballot(v) != 0; }
    static float sum(float v) {
        const double *x = say(v);
        float s = 0;
        for (int i = 0; i < N; ++i) s += (float)x[i];
        return s;
    }
    static int inclusive_sum(int v) {
        const int me = current;
        const double *x = say(v);
        int s = 0;
        for (int i = 0; i <= me; ++i) s += (int)x[i];
        return s;
    }
    static int of(int v, int lane) { return (int)say(v)[lane]; }
    static float of_first(float v) { return (float)say(v)[0]; }
    static float reciprocal(float v) { return (float)((1.0 / v) * (1.0 + off)); }
};

static int n_q, n_kv, type, page, width, window, sinks, n_seqs;   // type: 0 fp32, 1 bf16, 2 pages in 4 bits
static std::vector<int32_t> start, len;
static void fail(const char *what) {
    printf("%s: %d heads on %d, type %d, page %d, table of %d, window %d, sinks %d, %d sequences (new, held):", what, n_q, n_kv, type, page, width, window, sinks, n_seqs);
    for (int i = 0; i < n_seqs && i < 70; ++i) printf(" (%d, %d)", start[i + 1] - start[i], len[i]);
    printf("\n");
    exit(1);
}
#define OK(...) do { if (!(__VA_ARGS__)) fail("not " #__VA_ARGS__); } while (0)

static AttnArgs a;
static lvr_paged_batch b;
static PagedLaunch launch;
struct Found { bool is; Tile t; };
static std::vector<Found> found, cut;   // by piece; the tiles that the second launch merges

template <bool MIXED>
static void wave(int lane) {
    Division<MIXED, Lanes> d(a, b);
    OK(d.divide(a.target));
    for (int64_t x = 0; x < launch.pieces + 3; ++x) {
        Found f;
        memset(&f, 0, sizeof f);
        f.is = d.template locate<false>((int)x, f.t);
        if (lane == 0) found.push_back(f);
        else OK(f.is == found[x].is && (!f.is || !memcmp(&f.t, &found[x].t, sizeof(Tile))));   // all lanes find the same
    }
    for (int x = 0; MIXED && a.target > 0; ++x) {
        OK(x <= WIDE_ROOM);
        Found f;
        memset(&f, 0, sizeof f);
        f.is = d.template locate<true>(x, f.t);
        if (lane == 0) cut.push_back(f);
        if (!f.is) break;
    }
}

static long levelled;
static void check() {
    const bool MIXED = launch.mixed;
    found.clear();
    cut.clear();
    if (MIXED) run(wave<true>);
    else run(wave<false>);
    std::map<std::pair<int, int>, std::vector<Tile>> tiles;
    std::map<std::pair<int, int>, int> slots;
    int64_t pieces = 0;
    for (size_t x = 0; x < found.size(); ++x) {
        if (!found[x].is) continue;
        OK((int64_t)x < launch.pieces);
        tiles[{found[x].t.seq, found[x].t.row0}].push_back(found[x].t);
        ++pieces;
    }
    const int G = n_q / n_kv;
    const int64_t reach = (int64_t)width * page;
    size_t n_tiles = 0;
    bool alone = !MIXED && n_seqs <= N, even = true;   // one tile to a sequence; all as long
    int count = 0, held0 = -1;
    for (int s = 0; s < n_seqs; ++s) {
        const int tokens = start[s + 1] - start[s], rows = tokens * G, held = std::max(len[s], 0);
        const int height = MIXED && rows > a.narrow ? 128 : 16;
        if (rows > 0) {
            alone &= rows <= height;
            even &= held0 < 0 || held0 == held;
            held0 = held;
            ++count;
        }
        for (int row0 = 0; row0 < rows; row0 += height, ++n_tiles) {
            auto &p = tiles[{s, row0}];
            OK(!p.empty() && (int)p.size() == p[0].splits);
            std::sort(p.begin(), p.end(), [](const Tile &x, const Tile &y) { return x.split < y.split; });
            const int64_t p0 = (int64_t)held - tokens + row0 / G, p1 = (int64_t)held - tokens + (std::min(row0 + height, rows) - 1) / G;
            const int64_t end = std::min(p1 + 1, reach);
            std::vector<char> covered(std::max<int64_t>(end, 0) + 64);
            for (auto &x : p) {
                OK(x.height == height && x.rows == rows && x.first_token == start[s] && x.pos0 == held - tokens && x.hi == end);
                OK(x.begin % 64 == 0 && x.fold % 64 == 0 && x.shift % 64 == 0 && x.shift >= 0);
                OK(&x == &p[0] || (x.begin == (&x)[-1].end && x.split == (&x)[-1].split + 1));
                if (x.splits > 1) {
                    OK(x.slot >= x.split && x.slot - x.split == p[0].slot && ((int64_t)x.slot + 1) * n_kv <= (height == 128 ? WIDE_ROOM : NARROW_ROOM));
                    OK(!slots[{height, x.slot}]++);
                }
                for (int place = x.begin; place < x.end; ++place) {
                    const int64_t key = place + (place >= x.fold ? x.shift : 0);
                    if (key < x.hi) OK(key >= 0 && !covered[key]++);
                }
            }
            for (int64_t key = 0; key < end; ++key) OK(covered[key] || !(key < a.sinks || !a.window || key > p0 - a.window));
        }
    }
    OK(tiles.size() == n_tiles);
    // Batches of one length are cut into no more pieces than wanted, where that leaves two to a sequence.
    if (alone && even && count > 0 && a.target / count >= 2) {
        OK(pieces <= a.target);
        ++levelled;
    }
    std::map<std::pair<int, int>, Tile> merged;
    for (auto &f : cut)
        if (f.is) merged[{f.t.seq, f.t.row0}] = f.t;
    for (auto &x : tiles)
        if (x.second[0].height == 128 && x.second[0].splits > 1) {
            OK(merged.count(x.first) && merged[x.first].splits == x.second[0].splits && merged[x.first].slot == x.second[0].slot);
        }
}

int main() {
    long cases = 0;
    while (scanf("%d %d %d %d %d %d %d %d", &n_q, &n_kv, &type, &page, &width, &window, &sinks, &n_seqs) == 8) {
        start.assign(n_seqs + 1, 0);
        len.assign(n_seqs, 0);
        for (int i = 0; i < n_seqs; ++i) {
            int t;
            if (scanf("%d %d", &t, &len[i]) != 2) return 2;
            start[i + 1] = start[i] + t;
        }
        b = lvr_paged_batch{};
        b.seq_start = start.data();
        b.seq_len = len.data();
        b.n_seqs = n_seqs;
        b.n_tokens = start[n_seqs];
        b.table_width = width;
        b.page_shift = __builtin_ctz(page);
        b.n_pages = 1;
        if (b.n_tokens == 0) continue;   // nothing is launched
        a = AttnArgs{};
        a.window = window;
        a.sinks = sinks;
        launch = paged_launch(a, b, n_q, n_kv, type != 0, type == 2);
        static const float offs[] = {0.f, 1.2e-7f, -1.2e-7f};
        off = offs[cases++ % 3];
        check();
    }
    printf("%ld %ld\n", cases, levelled);
    return 0;
}
'''


@pytest.fixture(scope="module")
def division(tmp_path_factory):
    from paper_2605_06763_amd.build import CSRC

    def compiled(name, text):
        folder = tmp_path_factory.mktemp(name)
        src, exe = folder / (name + ".hip"), folder / name
        src.write_text(text)
        r = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "--offload-arch=gfx950", "-O1", "-std=c++17", "-I", CSRC, str(src), "-o", str(exe)],
                           capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        return exe
    return compiled


def size(rng, top):
    return int(2 ** rng.uniform(0, top))


def batch(rng, heads, lens, window=0, sinks=0, kind=None, page=None):
    page = page or rng.choice([16, 16, 64, 1024])
    pages = -(-max([1] + [n for _, n in lens]) // page)
    width = rng.choice([pages, pages, pages, pages + 3, max(1, pages // 2)])
    kind = rng.randint(0, 2) if kind is None else kind
    return " ".join(str(x) for x in (*heads, kind, page, width, window, sinks, len(lens), *(v for p in lens for v in p)))


def test_the_lanes_of_a_wave_divide_a_batch(division):
    """Batches of one length, with empty sequences and others among them, ragged ones, chunks beside single tokens, on both sides of as many sequences as a wave
    has lanes: every key that a row sees lies in one run, pieces have workgroups, partial results have places of their own."""
    exe = division("lanes", PROGRAM)
    rng = random.Random(77)
    lines = []
    for i in range(700):
        heads = rng.choice([(32, 8), (32, 8), (64, 8), (8, 8), (8, 1), (28, 4), (12, 4), (40, 8), (71, 1), (256, 256)])
        window = rng.choice([0, 0, 0, 1, size(rng, 8), size(rng, 13)])
        sinks = rng.choice([0, 0, 1, 4, 64, 65, size(rng, 10)])
        n_seqs = rng.choice([1, 2, 3, 5, 12, 20, size(rng, 6), 62, 63, 64, 65, 66, 130])
        n = size(rng, 15 if n_seqs < 30 else 11)
        what = rng.choice(["even", "even", "even", "ragged", "nearly", "chunk"])
        t = rng.choice([1, 1, 1, 2, size(rng, 5)])
        if what == "ragged":
            lens = [(m, m + size(rng, 13) - 1) for m in (rng.choice([1, 1, t, size(rng, 8)]) for _ in range(n_seqs))]
        elif what == "chunk":
            lens = [(size(rng, 9), size(rng, 13))] + [(1, size(rng, 12)) for _ in range(n_seqs - 1)]
            lens[0] = (lens[0][0], max(lens[0]))
        else:
            lens = [(t, max(t, n))] * n_seqs
        if what == "nearly":
            lens = [p if rng.random() < 0.8 else rng.choice([(0, n), (0, 0), (t, max(t, n // 2)), (t, t)]) for p in lens]
        lines.append(batch(rng, heads, lens, window, sinks))
    r = subprocess.run([str(exe)], input="\n".join(lines), capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout + r.stderr
    assert int(r.stdout.split()[0]) > 600 and int(r.stdout.split()[1]) > 60


def test_single_tokens_of_one_length_over_lengths(division):
    """Every number of sequences up to one more than a wave has lanes, lengths around multiples of the shortest run, all types."""
    exe = division("even", PROGRAM)
    rng = random.Random(78)
    lines = []
    for n_seqs in range(1, 66):
        for heads in ((32, 8), (8, 8), (12, 2)):
            n = rng.choice([63, 64, 65, 255, 256, 257, 512, 513, 1363, 1630, 4096, size(rng, 14)])
            lens = [(1, n)] * n_seqs
            if rng.random() < 0.3:
                lens += [(0, n)] * rng.randint(0, 64 - min(n_seqs, 64))
            lines.append(batch(rng, heads, lens, kind=rng.randint(0, 2)))
    r = subprocess.run([str(exe)], input="\n".join(lines), capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout + r.stderr
    assert int(r.stdout.split()[0]) == len(lines) and int(r.stdout.split()[1]) > 60
