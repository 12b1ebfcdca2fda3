"""How the attention over pages divides a batch into pieces: the device's own arithmetic, compiled for the host with a wave of one lane.

Every batch has to be divided in a bounded number of steps, into pieces that the launch has workgroups for, whose partial results lie
within the work space and apart from each other, and that cover every (row, key) once."""
import importlib.util
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r'''
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <vector>
#include "paged_division.h"

static long asked, may_ask;   // sums over the batch, three to a step of the division
static float off;             // how far the device's reciprocal is off the exact one, relative (it is good to a unit of the last place)
static void fail(const char *what);
struct Alone {
    static constexpr int LANES = 1;
    static int lane() { return 0; }
    static bool any(bool v) { return v; }
    static uint64_t ballot(bool v) { return v; }
    static float sum(float v) { return v; }
    static int inclusive_sum(int v) { if (++asked > may_ask) fail("the division does not end"); return v; }
    static int of(int v, int) { return v; }
    static float of_first(float v) { return v; }
    static float reciprocal(float v) { return (float)((1.0 / v) * (1.0 + off)); }
};

static int n_q, n_kv, bf16, page, width, window, n_seqs;
static std::vector<int32_t> start, len;
static long cases, grown, most;   // cases; those that took more than one step; most steps

static void fail(const char *what) {
    printf("%s: %d heads on %d, %s, page %d, table of %d, window %d, %d sequences (new, held):", what, n_q, n_kv, bf16 ? "bf16" : "f32", page, width, window, n_seqs);
    for (int i = 0; i < n_seqs && i < 40; ++i) printf(" (%d, %d)", start[i + 1] - start[i], len[i]);
    printf("\n");
    exit(1);
}
#define OK(...) do { if (!(__VA_ARGS__)) fail("not " #__VA_ARGS__); } while (0)

template <bool MIXED>
static void check(AttnArgs &a, const lvr_paged_batch &b, const PagedLaunch &launch, bool pieces_too) {
    Division<MIXED, Alone> d(a, b);
    asked = 0;
    may_ask = 3L * std::max(n_seqs, 1) * 64;
    OK(d.divide(a.target));
    const long steps = MIXED && n_seqs ? asked / (3L * n_seqs) : 1;
    grown += steps > 1;
    most = std::max(most, steps);
    may_ask = 1L << 60;
    int64_t all = 0, cut_wide = 0, cut_narrow = 0;
    for (int i = 0; i < n_seqs; ++i) {
        d.look(i);
        d.cut();
        all += (int64_t)d.tiles * d.runs;
        if (d.runs > 1) (d.is_wide() ? cut_wide : cut_narrow) += (int64_t)d.tiles * d.runs;
    }
    OK(all <= launch.pieces);
    OK(cut_wide * n_kv <= WIDE_ROOM);
    OK(cut_narrow * n_kv <= NARROW_ROOM);
    if (!pieces_too) return;
    if (n_seqs == 1) d.look(0), d.cut();   // what a wave keeps of a batch that it looks at once

    std::map<std::pair<int, int>, std::vector<Tile>> tiles;
    Tile t;
    for (int64_t x = 0; x < launch.pieces; ++x)
        if (d.template locate<false>((int)x, t)) tiles[{t.seq, t.row0}].push_back(t);
    for (int64_t x = launch.pieces; x < launch.pieces + 8; ++x) OK(!d.template locate<false>((int)x, t));
    const int G = n_q / n_kv;
    const int64_t reach = (int64_t)width * page;
    size_t n_tiles = 0;
    std::map<std::pair<int, int>, int> slots;   // (height, slot) -> taken
    for (int s = 0; s < n_seqs; ++s) {
        const int tokens = start[s + 1] - start[s], rows = tokens * G, held = std::min(std::max(len[s], 0), 1 << 30);
        const int height = MIXED && rows > a.narrow ? 128 : 16;
        for (int row0 = 0; row0 < rows; row0 += height, ++n_tiles) {
            auto &p = tiles[{s, row0}];
            OK(!p.empty());
            std::sort(p.begin(), p.end(), [](const Tile &x, const Tile &y) { return x.split < y.split; });
            const int last = std::min(row0 + height, rows) - 1;
            const int64_t p0 = (int64_t)held - tokens + row0 / G, p1 = (int64_t)held - tokens + last / G;
            const int64_t hi = std::min(p1 + 1, reach), lo = window ? std::max<int64_t>(0, p0 - window + 1) : 0;
            OK((int)p.size() == p[0].splits);
            int64_t at = lo & ~63;
            for (int i = 0; i < (int)p.size(); ++i) {
                const Tile &x = p[i];
                OK(x.height == height && x.rows == rows && x.first_token == start[s] && x.pos0 == held - tokens);
                OK(x.hi == hi && x.lo == lo && x.split == i && x.splits == (int)p.size());
                OK(x.begin == at && x.begin % 64 == 0);
                OK(i + 1 < (int)p.size() ? x.end > x.begin : x.end == hi);
                at = x.end;
                if (x.splits == 1) continue;
                OK(x.slot - x.split == p[0].slot && x.slot >= 0);
                OK(((int64_t)x.slot + 1) * n_kv <= (height == 128 ? WIDE_ROOM : NARROW_ROOM));
                OK(!slots[{height, x.slot}]++);
            }
        }
    }
    OK(tiles.size() == n_tiles);
    if (!MIXED || a.target == 0) return;
    std::map<std::pair<int, int>, bool> merged;   // the second launch finds every cut tile of 128 rows, and its partial results
    for (int x = 0; d.template locate<true>(x, t); ++x) {
        OK(x <= WIDE_ROOM);
        auto &p = tiles[{t.seq, t.row0}];
        OK(t.height == 128 && !p.empty() && p[0].splits == t.splits && (t.splits == 1 || p[0].slot == t.slot));
        merged[{t.seq, t.row0}] = true;
    }
    for (auto &x : tiles)
        if (x.second[0].height == 128 && x.second[0].splits > 1) OK(merged[x.first]);
}

static void one(bool pieces_too) {
    lvr_paged_batch b = {};
    b.seq_start = start.data();
    b.seq_len = len.data();
    b.n_seqs = n_seqs;
    b.n_tokens = start[n_seqs];
    b.table_width = width;
    b.page_shift = __builtin_ctz(page);
    b.n_pages = 1;
    if (b.n_tokens == 0 || n_seqs == 0) return;   // nothing is launched
    AttnArgs a = {};
    a.window = window;
    const PagedLaunch launch = paged_launch(a, b, n_q, n_kv, bf16);
    static const float offs[] = {0.f, 1.2e-7f, -1.2e-7f};
    off = offs[cases++ % 3];
    if (launch.mixed) check<true>(a, b, launch, pieces_too);
    else check<false>(a, b, launch, pieces_too);
}

// Batches of `seqs` prompts of n tokens behind `before` keys, with a table of just the pages they take.
static void prompts(int seqs, int n, int before) {
    n_seqs = seqs;
    start.assign(seqs + 1, 0);
    for (int i = 0; i < seqs; ++i) start[i + 1] = start[i] + n;
    len.assign(seqs, n + before);
    width = (n + before + page - 1) / page;
    one(false);
}

int main(int argc, char **argv) {
    if (argc > 1 && !strcmp(argv[1], "prompts")) {
        static const int heads[][2] = {{32, 8}, {64, 8}, {16, 8}, {8, 8}, {8, 2}, {8, 1}, {24, 8}, {12, 4}, {40, 8}, {28, 4}, {64, 4}, {96, 8}, {71, 1}, {256, 256}};
        for (auto &h : heads)
            for (bf16 = 0; bf16 < 2; ++bf16)
                for (int w = 0; w < 3; ++w)
                    for (int n = 1; n <= 4096; ++n) {
                        n_q = h[0], n_kv = h[1], page = w == 1 ? 64 : 16, window = w == 2 ? 1 + n / 3 : 0;
                        prompts(1, n, 0);
                        prompts(2 + n % 63, n, 0);
                        if (n <= 512) for (int s = 2; s <= 64; ++s) prompts(s, n, 0);
                        prompts(1, n, 1 + n * 7 % 3000);
                        prompts(1 + n % 5, n, 20000);
                    }
    } else {   // n_q n_kv bf16 page width window n_seqs (new held)...
        while (scanf("%d %d %d %d %d %d %d", &n_q, &n_kv, &bf16, &page, &width, &window, &n_seqs) == 7) {
            start.assign(n_seqs + 1, 0);
            len.assign(n_seqs, 0);
            for (int i = 0; i < n_seqs; ++i) {
                int t;
                if (scanf("%d %d", &t, &len[i]) != 2) return 2;
                start[i + 1] = start[i] + t;
            }
            one(true);
        }
    }
    printf("%ld %ld %ld\n", cases, grown, most);
    return 0;
}
'''


@pytest.fixture(scope="module")
def divide(tmp_path_factory):
    """Runs the program over batches (or over its own prompts); cases, those whose runs had to be made longer, and the most steps."""
    from paper_2605_06763_amd.build import CSRC
    folder = tmp_path_factory.mktemp("division")
    src, exe = folder / "division.hip", folder / "division"
    src.write_text(PROGRAM)
    r = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "--offload-arch=gfx950", "-O1", "-std=c++17", "-I", CSRC, str(src), "-o", str(exe)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def run(batches=None):
        text = None if batches is None else "\n".join(
            " ".join(str(x) for x in (*heads, int(dtype == "bf16"), page, width, window, len(lens), *(v for pair in lens for v in pair)))
            for heads, dtype, page, width, window, lens in batches)
        r = subprocess.run([str(exe)] + (["prompts"] if batches is None else []), input=text, capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stdout
        cases, grown, most = (int(x) for x in r.stdout.split())
        assert batches is None or cases >= len([b for b in batches if sum(t for t, _ in b[5])])
        return cases, grown, most

    return run


def batch(heads, lens, dtype="bf16", page=16, window=0, width=None):
    return heads, dtype, page, max([1] + [-(-n // page) for _, n in lens]) if width is None else width, window, lens


# prompts whose partial results do not fit the work space with the shortest runs
PROMPTS_TO_LENGTHEN = [((64, 8), 1, 352), ((64, 8), 1, 356), ((64, 8), 1, 360), ((32, 8), 8, 165), ((32, 8), 8, 170), ((32, 8), 2, 352), ((64, 8), 4, 170),
                       ((28, 4), 1, 546), ((12, 4), 1, 820), ((96, 8), 1, 292)]


@pytest.mark.parametrize("heads, seqs, n", PROMPTS_TO_LENGTHEN)
def test_runs_are_made_longer_until_the_partial_results_fit(divide, heads, seqs, n):
    divide([batch(heads, [(n, n)] * seqs, dtype, page) for dtype in ("bf16", "f32") for page in (16, 64)])


def test_prompts_of_every_length(divide):
    cases, grown, most = divide()
    assert cases > 1000000 and grown > 1000 and most <= 40


def test_batches_as_they_are_timed(divide):
    """The batches of the timed cases, listed and drawn."""
    spec = importlib.util.spec_from_file_location("timed_operators", os.path.join(ROOT, "perf", "operators.py"))
    O = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(O)
    cases = [c for c in O.listed() if c["kind"] == "attention"]
    rng = random.Random(11)
    while len(cases) < 3000:
        c = O.draw(rng)
        if c["kind"] == "attention":
            cases.append(c)
    divide([batch((c["hq"], c["hkv"]), list(zip(*O._lengths(c))), c["dtype"], c["page"], c["window"]) for c in cases])


def test_batches_of_every_kind(divide):
    """Many sequences and few, none and many new tokens, tokens before the cache, lengths beyond the table and at the ends of their range."""
    rng = random.Random(12)
    size = lambda top: int(2 ** rng.uniform(0, top)) if rng.random() < 0.9 else 0   # noqa: E731
    batches = []
    for _ in range(3000):
        heads = rng.choice([(32, 8), (64, 8), (8, 8), (8, 1), (28, 4), (12, 4), (96, 8), (1, 1), (71, 1), (256, 256), (1024, 1)])
        few, top = rng.random() < 0.7, 10 if heads[0] < 200 else 6
        lens = []
        for _ in range(rng.randint(1, 6) if few else rng.randint(7, 200)):
            t = size(top if few else 6)
            lens.append((t, t if rng.random() < 0.3 else rng.choice([0, t // 2, t + size(15), t + size(15), 2 ** 31 - 1 if rng.random() < 0.1 else t + 1])))
        page = rng.choice([16, 16, 64, 1024])
        pages = -(-max(min(n, 1 << 20) for _, n in lens) // page)
        width = rng.choice([pages, pages, pages + 3, max(1, pages // 2), 1, 0])
        batches.append(batch(heads, lens, rng.choice(["bf16", "f32"]), page, rng.choice([0, 0, 1, 50, 3000]), width))
    divide(batches)


def test_chunks_longer_than_their_table(divide):
    """Every sequence counts for the keys it can see: a chunk of more than twice the tokens its table has room for is divided as fast as others, and
    so are the sequences beside it."""
    batches = [batch((1, 1), [(5000, 5000)], width=125), batch((1, 1), [(100000, 100000)], width=2500), batch((8, 8), [(30000, 30000), (90, 9000)], width=500),
               batch((1, 1), [(20000, 20000)] + [(5, 4000)] * 40, width=250), batch((8, 2), [(9000, 2 ** 30)], "f32", width=100)]
    cases, _, most = divide(batches)
    assert cases == len(batches) and most <= 2
