"""The paged cache's pages in 4 bits, windows with first keys that stay visible, and norms, without a GPU: configurations and arguments that are
refused, where a row's codes and scales lie, and how a batch is divided when first keys stay visible."""
import ctypes as C
import os
import random
import subprocess

import pytest
import torch


@pytest.fixture(scope="module")
def L():
    import paper_2605_06763_amd as L
    if not os.path.exists(L.binding.LIB_PATH):
        from paper_2605_06763_amd.build import build_library
        build_library()
    return L


def compiled(tmp_path_factory, name, text):
    from paper_2605_06763_amd.build import CSRC
    folder = tmp_path_factory.mktemp(name)
    src, exe = folder / (name + ".hip"), folder / name
    src.write_text(text)
    r = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "--offload-arch=gfx950", "-O1", "-std=c++17", "-I", CSRC, str(src), "-o", str(exe)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return exe


OK = dict(n_q_heads=32, n_kv_heads=8, page_size=16, n_pages=100, rot_dim=128)
PAGE = 8 * 16 * 68


@pytest.mark.parametrize("bad, code", [
    (dict(page_strides=(PAGE - 16, 16 * 64, 64)), "INVALID"), (dict(page_strides=(PAGE + 8, 16 * 64, 64)), "INVALID"),
    (dict(page_strides=(PAGE, 16 * 64, 48)), "INVALID"), (dict(page_strides=(-PAGE, 16 * 64, 64)), "INVALID"),
    (dict(page_strides=(PAGE, 16 * 64 + 64, 64)), "UNSUPPORTED"), (dict(page_strides=(PAGE, 16 * 68, 68)), "INVALID"),
    (dict(page_strides=(PAGE, 64, 8 * 64 + 64)), "UNSUPPORTED"), (dict(page_strides=(PAGE, 16 * 128, 128)), "UNSUPPORTED"),
    (dict(head_dim=64, rot_dim=64), "UNSUPPORTED"), (dict(page_size=8), "UNSUPPORTED"), (dict(n_kv_heads=5), "INVALID"),
])
def test_bad_configurations_of_pages_in_4_bits_are_refused(L, bad, code):
    cfg = L.make_paged_config(kv_dtype=L.LVR_FP4, **dict(OK, **bad))
    assert L.lvr_paged_bytes(cfg) == 0
    freq, h = (C.c_double * 64)(*[0.5] * 64), C.c_void_p()
    assert L.lib().lvr_paged_create(C.byref(cfg), freq, None, C.byref(h)) == getattr(L, "LVR_E_" + code) and not h.value


def test_configurations_of_pages_in_4_bits(L):
    for more in (dict(), dict(layout="token"), dict(page_strides=(PAGE + 4096, 16 * 64, 64)), dict(n_kv_heads=1), dict(n_kv_heads=1, layout="token"),
                 dict(n_kv_heads=256, n_q_heads=256, page_size=65536)):
        cfg = L.make_paged_config(kv_dtype=L.LVR_FP4, **dict(OK, **more))
        assert L.lvr_paged_bytes(cfg) > 0
        assert L.paged_page_bytes(cfg) == cfg.n_kv_heads * cfg.page_size * 68 <= cfg.page_strides[0]
    for dtype in (2, 3, 5, -1):
        assert L.lvr_paged_bytes(L.make_paged_config(kv_dtype=dtype, **OK)) == 0
    # 4 bits are for pages alone
    assert L.lvr_arena_bytes(L.make_config(batch=1, n_q_heads=32, n_kv_heads=8, capacity=1024, kv_dtype=L.LVR_FP4)) == 0


def test_calls_without_a_handle_are_refused(L):
    lib = L.lib()
    assert lib.lvr_paged_norm_append(*[None] * 10, 1e-6, *[None] * 4, 0, 0, 0, None) == L.LVR_E_INVALID
    assert lib.lvr_paged_sink_attention(*[None] * 4, 0, None, None, None, 0, 0, 0, 0, 0, None, None) == L.LVR_E_INVALID


def handle(L, **more):
    h = L.PagedHandle()
    h.cfg, h.dtype = L.make_paged_config(**dict(OK, **more)), torch.bfloat16
    h.cfg_at, h.device = C.addressof(h.cfg), 0
    return h


def test_host_tensors_are_refused(L):
    i, table = torch.zeros(2, dtype=torch.int32), torch.zeros(1, 4, dtype=torch.int32)
    kv, q = torch.zeros(3, 8, 128, dtype=torch.bfloat16), torch.zeros(3, 32, 128, dtype=torch.bfloat16)
    for h, pool in ((handle(L), torch.zeros(100, 8, 16, 128, dtype=torch.bfloat16)), (handle(L, kv_dtype=L.LVR_FP4), torch.zeros(100, PAGE, dtype=torch.uint8))):
        for call in (lambda: L.lvr_paged_norm_append(h, pool, pool, kv, kv, i, i[:1], table), lambda: L.lvr_paged_append(h, pool, pool, kv, kv, i, i[:1], table),
                     lambda: L.lvr_paged_sink_attention(h, pool, pool, q, i, i[:1], table, q, 16, 4), lambda: L.lvr_paged_attention(h, pool, pool, q, i, i[:1], table, q),
                     lambda: L.lvr_paged_gather(h, pool, pool, i[:1], table, q, q)):
            with pytest.raises(ValueError, match="must be a device tensor"):
                call()


def test_pools_in_4_bits_are_checked(L, monkeypatch):
    monkeypatch.setattr(L.binding, "_tensor", lambda h, t, name: t)
    h = handle(L, kv_dtype=L.LVR_FP4)
    pool = torch.zeros(100, PAGE, dtype=torch.uint8)
    assert L.binding._pool(h, pool, "k_pages") == pool.data_ptr()
    for bad in (pool[:99], pool[:, :-16], pool.view(100, 8, 16, 68), pool.view(torch.int8), torch.zeros(100, PAGE + 64, dtype=torch.uint8)[:, :PAGE]):
        with pytest.raises(ValueError, match="k_pages must be"):
            L.binding._pool(h, bad, "k_pages")
    wide = handle(L, kv_dtype=L.LVR_FP4, page_strides=(PAGE + 64, 16 * 64, 64))
    pool = torch.zeros(100, PAGE + 64, dtype=torch.uint8)[:, :PAGE]
    assert L.binding._pool(wide, pool, "k_pages") == pool.data_ptr()


def test_windows_and_first_keys_are_checked(L, monkeypatch):
    monkeypatch.setattr(L.binding, "_pool", lambda *a: 0)
    monkeypatch.setattr(L.binding, "_tensor", lambda h, t, name: t)
    h, i, table = handle(L), torch.zeros(2, dtype=torch.int32), torch.zeros(1, 4, dtype=torch.int32)
    q = torch.zeros(3, 32, 128, dtype=torch.bfloat16)
    for window, sinks, what in ((-1, 4, "window"), (1 << 31, 4, "window"), (16, -1, "sinks"), (16, 1 << 31, "sinks")):
        with pytest.raises(ValueError, match=what):
            L.lvr_paged_sink_attention(h, None, None, q, i, i[:1], table, q, window, sinks)


def test_where_codes_and_scales_lie(tmp_path_factory):
    """Every row of a page has 64 bytes of codes and 4 of scales of its own, all of them within the page."""
    exe = compiled(tmp_path_factory, "places", r'''
#include <vector>
#include "paged.h"
int main() {
    for (int heads : {1, 3, 8}) for (int shift = 4; shift < 8; ++shift) for (int token = 0; token < 2; ++token) for (int extra : {0, 64}) {
        const int page = 1 << shift;
        lvr_paged_batch b = {};
        b.page_shift = shift;
        b.n_pages = 3;
        b.page_stride = (int64_t)heads * page * 68 + extra;
        b.head_stride = token ? 64 : 64 * page;
        b.row_stride = token ? 64 * heads : 64;
        b.scales = (int64_t)heads * page * 64;
        std::vector<char> taken(3 * b.page_stride);
        for (int p = 0; p < 3; ++p) for (int h = 0; h < heads; ++h) for (int64_t pos = page * 5; pos < page * 6; ++pos) {
            const int64_t at = lvr_row_at(b, p, h, pos), sc = lvr_scales_at(b, p, h, pos), in = pos % page;
            if (at % 64 || sc % 4) return 1;
            if (sc - p * b.page_stride - b.scales != 4 * (token ? in * heads + h : h * page + in)) return 2;
            for (int i = 0; i < 64; ++i) if (at + i < p * b.page_stride || at + i >= p * b.page_stride + b.scales || taken[at + i]++) return 3;
            for (int i = 0; i < 4; ++i) if (sc + i < p * b.page_stride + b.scales || sc + i >= (p + 1) * b.page_stride - extra || taken[sc + i]++) return 4;
        }
    }
    return 0;
}
''')
    assert subprocess.run([str(exe)]).returncode == 0


DIVISION = r'''
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <vector>
#include "paged_division.h"

struct Alone {
    static constexpr int LANES = 1;
    static int lane() { return 0; }
    static bool any(bool v) { return v; }
    static uint64_t ballot(bool v) { return v; }
    static float sum(float v) { return v; }
    static int inclusive_sum(int v) { return v; }
    static int of(int v, int) { return v; }
    static float of_first(float v) { return v; }
    static float reciprocal(float v) { return 1.f / v; }
};

static int n_q, n_kv, type, page, width, window, sinks, n_seqs;   // type: 0 fp32, 1 bf16, 2 pages in 4 bits
static std::vector<int32_t> start, len;
static void fail(const char *what) {
    printf("%s: %d heads on %d, type %d, page %d, table of %d, window %d, sinks %d, %d sequences (new, held):", what, n_q, n_kv, type, page, width, window, sinks, n_seqs);
    for (int i = 0; i < n_seqs && i < 40; ++i) printf(" (%d, %d)", start[i + 1] - start[i], len[i]);
    printf("\n");
    exit(1);
}
#define OK(...) do { if (!(__VA_ARGS__)) fail("not " #__VA_ARGS__); } while (0)

template <bool MIXED>
static void check(AttnArgs &a, const lvr_paged_batch &b, const PagedLaunch &launch) {
    Division<MIXED, Alone> d(a, b);
    OK(d.divide(a.target));
    int64_t all = 0, cut_wide = 0, cut_narrow = 0;
    for (int i = 0; i < n_seqs; ++i) {
        d.look(i);
        d.cut();
        all += (int64_t)d.tiles * d.runs;
        if (d.runs > 1) (d.is_wide() ? cut_wide : cut_narrow) += (int64_t)d.tiles * d.runs;
    }
    OK(all <= launch.pieces && cut_wide * n_kv <= WIDE_ROOM && cut_narrow * n_kv <= NARROW_ROOM);
    if (n_seqs == 1) d.look(0), d.cut();
    std::map<std::pair<int, int>, std::vector<Tile>> tiles;
    std::map<std::pair<int, int>, int> slots;
    Tile t;
    for (int64_t x = 0; x < launch.pieces; ++x)
        if (d.template locate<false>((int)x, t)) tiles[{t.seq, t.row0}].push_back(t);
    const int G = n_q / n_kv;
    const int64_t reach = (int64_t)width * page;
    for (int s = 0; s < n_seqs; ++s) {
        const int tokens = start[s + 1] - start[s], rows = tokens * G, held = std::max(len[s], 0);
        const int height = MIXED && rows > a.narrow ? 128 : 16;
        for (int row0 = 0; row0 < rows; row0 += height) {
            auto &p = tiles[{s, row0}];
            OK(!p.empty() && (int)p.size() == p[0].splits);
            std::sort(p.begin(), p.end(), [](const Tile &x, const Tile &y) { return x.split < y.split; });
            const int64_t p0 = (int64_t)held - tokens + row0 / G, p1 = (int64_t)held - tokens + (std::min(row0 + height, rows) - 1) / G;
            const int64_t end = std::min(p1 + 1, reach);
            std::vector<char> covered(std::max<int64_t>(end, 0) + 64);
            int work = 0;
            for (auto &x : p) {
                OK(x.begin % 64 == 0 && x.fold % 64 == 0 && x.shift % 64 == 0 && x.shift >= 0);
                OK(x.hi == end && x.begin == (&x == &p[0] ? x.begin : (&x)[-1].end));
                if (x.splits > 1) {
                    OK(x.slot - x.split == p[0].slot && ((int64_t)x.slot + 1) * n_kv <= (height == 128 ? WIDE_ROOM : NARROW_ROOM));
                    OK(!slots[{height, x.slot}]++);
                }
                for (int place = x.begin; place < x.end; ++place, ++work) {
                    const int64_t key = place + (place >= x.fold ? x.shift : 0);
                    if (key >= x.hi) continue;   // a kernel looks no page up
                    OK(key >= 0 && !covered[key]++);
                }
            }
            for (int64_t key = 0; key < end; ++key) {
                const bool seen = key < sinks || !window || key > p0 - window;   // by some row of the tile
                OK(!seen || covered[key]);
            }
            OK(height == 128 || p.size() == 1 || (window ? std::min(held, window + 128 + (sinks + 63) / 64 * 64) : held) > a.uncut);
            // no more than what the rows see and the ends of their tiles of 64
            if (window) OK(work <= window + sinks + height + 192);
        }
    }
    if (!MIXED || a.target == 0) return;
    std::map<std::pair<int, int>, bool> merged;
    for (int x = 0; d.template locate<true>(x, t); ++x) merged[{t.seq, t.row0}] = true;
    for (auto &x : tiles)
        if (x.second[0].height == 128 && x.second[0].splits > 1) OK(merged[x.first]);
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
        lvr_paged_batch b = {};
        b.seq_start = start.data();
        b.seq_len = len.data();
        b.n_seqs = n_seqs;
        b.n_tokens = start[n_seqs];
        b.table_width = width;
        b.page_shift = __builtin_ctz(page);
        b.n_pages = 1;
        AttnArgs a = {};
        a.window = window;
        a.sinks = sinks;
        a.uncut = type == 2 ? UNCUT_FP4 : (type == 1 && sinks ? UNCUT_BF16 : 0);
        const PagedLaunch launch = paged_launch(a, b, n_q, n_kv, type != 0, type == 2);
        if (launch.mixed) check<true>(a, b, launch);
        else check<false>(a, b, launch);
        ++cases;
    }
    printf("%ld\n", cases);
    return 0;
}
'''


def test_every_key_a_row_sees_lies_in_one_run(tmp_path_factory):
    """Windows with first keys that stay visible, apart from the window and meeting it, over tables that end before either."""
    exe = compiled(tmp_path_factory, "division", DIVISION)
    rng = random.Random(21)
    size = lambda top: int(2 ** rng.uniform(0, top))   # noqa: E731
    lines = []
    for _ in range(4000):
        heads = rng.choice([(32, 8), (64, 8), (8, 8), (8, 1), (28, 4), (12, 4), (1, 1), (71, 1), (256, 256)])
        lens = []
        for _ in range(rng.choice([1, 1, 2, 3, 20, 80])):
            t = rng.choice([1, 1, size(9 if heads[0] < 200 else 5)])
            lens.append((t, t + rng.choice([0, size(6), size(14), size(17)]) if rng.random() < 0.95 else t // 2))
        page = rng.choice([16, 16, 64, 1024])
        pages = -(-max(n for _, n in lens) // page)
        width = rng.choice([pages, pages, pages + 3, max(1, pages // 2), 1])
        window = rng.choice([0, 1, 16, size(8), size(13), size(13)])
        sinks = rng.choice([1, 4, 63, 64, 65, size(10), size(13)]) if window else 0
        lines.append(" ".join(str(x) for x in (*heads, rng.randint(0, 2), page, width, window, sinks, len(lens), *(v for p in lens for v in p))))
    r = subprocess.run([str(exe)], input="\n".join(lines), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout
    assert int(r.stdout) == len(lines)
