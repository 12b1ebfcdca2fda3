"""The paged cache without a GPU: configurations and arguments that are refused, and where the kernels look for a row."""
import ctypes as C
import os
import re
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def L():
    import paper_2605_06763_amd as L
    if not os.path.exists(L.binding.LIB_PATH):
        from paper_2605_06763_amd.build import build_library
        build_library()
    return L


OK = dict(n_q_heads=32, n_kv_heads=8, page_size=16, n_pages=100, rot_dim=128)


def test_config_struct_matches_header(L):
    text = open(os.path.join(ROOT, "include", "louver.h")).read()
    body = re.search(r"typedef struct lvr_paged_config \{(.*?)\} lvr_paged_config;", text, flags=re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    fields = re.findall(r"\b(?:int32_t|int64_t|float)\s+([a-z_]+)(?:\[3\])?\s*;", body)
    assert fields == [f for f, _ in L.lvr_paged_config._fields_]


@pytest.mark.parametrize("bad, code", [
    (dict(n_q_heads=30), "INVALID"), (dict(n_q_heads=0), "INVALID"), (dict(n_kv_heads=0), "INVALID"), (dict(kv_dtype=2), "INVALID"),
    (dict(page_size=0), "INVALID"), (dict(page_size=-16), "INVALID"), (dict(n_pages=0), "INVALID"), (dict(rot_dim=-16), "INVALID"),
    (dict(rot_dim=144), "INVALID"), (dict(rot_dim=33), "INVALID"), (dict(rot_axes=0), "INVALID"), (dict(rot_axes=5), "INVALID"),
    (dict(rot_pairs=2), "INVALID"), (dict(scale=-1.0), "INVALID"), (dict(scale=float("nan")), "INVALID"),
    (dict(scale=float("inf")), "INVALID"),
    (dict(page_strides=(8 * 16 * 128, 16 * 128, 127)), "INVALID"), (dict(page_strides=(8 * 16 * 128, 16 * 128, 132)), "INVALID"),
    (dict(page_strides=(-128, 16 * 128, 128)), "INVALID"), (dict(page_strides=(8 * 16 * 128, 16 * 128, 120)), "INVALID"),
    (dict(head_dim=64, rot_dim=64), "UNSUPPORTED"), (dict(rot_dim=72), "UNSUPPORTED"), (dict(page_size=8), "UNSUPPORTED"),
    (dict(page_size=48), "UNSUPPORTED"), (dict(page_size=1 << 17), "UNSUPPORTED"), (dict(n_q_heads=2048), "UNSUPPORTED"),
    (dict(n_q_heads=512, n_kv_heads=512), "UNSUPPORTED"), (dict(n_pages=1 << 31), "UNSUPPORTED"),
    (dict(page_strides=(8 * 16 * 128, 128, (1 << 24) + 8)), "UNSUPPORTED"),
])
def test_bad_configurations_are_refused(L, bad, code):
    cfg = L.make_paged_config(**dict(OK, **bad))
    assert L.lvr_paged_bytes(cfg) == 0
    half = 64
    freq, h = (C.c_double * half)(*[0.5] * half), C.c_void_p()
    assert L.lib().lvr_paged_create(C.byref(cfg), freq, None, C.byref(h)) == getattr(L, "LVR_E_" + code) and not h.value


def test_rotations_are_checked(L):
    cfg = L.make_paged_config(**dict(OK, rot_axes=3))
    assert L.lvr_paged_bytes(cfg) > 0
    make = L.lib().lvr_paged_create
    h, good = C.c_void_p(), (C.c_double * 64)(*[0.1] * 64)
    for value in (float("nan"), float("inf")):
        bad = (C.c_double * 64)(*[0.1] * 63, value)
        assert make(C.byref(cfg), bad, None, C.byref(h)) == L.LVR_E_INVALID
    for value in (-1, 3):
        axis = (C.c_int32 * 64)(*[0] * 63, value)
        assert make(C.byref(cfg), good, axis, C.byref(h)) == L.LVR_E_INVALID
    assert make(C.byref(cfg), None, None, C.byref(h)) == L.LVR_E_INVALID
    assert make(C.byref(cfg), good, None, None) == L.LVR_E_INVALID
    assert make(None, good, None, C.byref(h)) == L.LVR_E_INVALID and not h.value
    with pytest.raises(ValueError, match="64 entries"):
        L.lvr_paged_create(cfg, inv_freq=[0.1] * 63)
    with pytest.raises(ValueError, match="64 entries"):
        L.lvr_paged_create(cfg, inv_freq=[0.1] * 64, axis=[0] * 3)
    with pytest.raises(ValueError, match="layout"):
        L.make_paged_config(**OK, layout="row")


def test_calls_without_a_handle_are_refused(L):
    lib = L.lib()
    assert lib.lvr_paged_destroy(None) == L.LVR_E_INVALID
    assert lib.lvr_paged_append(*[None] * 12, 0, 0, 0, None) == L.LVR_E_INVALID
    assert lib.lvr_paged_attention(*[None] * 4, 0, None, None, None, 0, 0, 0, 0, None, None) == L.LVR_E_INVALID
    assert lib.lvr_paged_gather(*[None] * 5, 0, 0, 0, None, None, None) == L.LVR_E_INVALID


def test_host_tensors_are_refused(L):
    h = L.PagedHandle()
    h.cfg, h.dtype = L.make_paged_config(**OK), torch.bfloat16
    h.cfg_at, h.device = C.addressof(h.cfg), 0
    pool, kv = torch.zeros(100, 8, 16, 128, dtype=torch.bfloat16), torch.zeros(3, 8, 128, dtype=torch.bfloat16)
    q, i = torch.zeros(3, 32, 128, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    table = torch.zeros(1, 4, dtype=torch.int32)
    for call in (lambda: L.lvr_paged_append(h, pool, pool, kv, kv, i, i[:1], table), lambda: L.lvr_paged_attention(h, pool, pool, q, i, i[:1], table, q),
                 lambda: L.lvr_paged_gather(h, pool, pool, i[:1], table, pool, pool)):
        with pytest.raises(ValueError, match="must be a device tensor"):
            call()


def test_every_row_the_kernels_look_up_lies_in_the_pool(L, tmp_path):
    """The kernels' own look-up of pages and rows, compiled for the host, over tables with entries outside the pool and positions
    outside the table."""
    src = tmp_path / "rows.hip"
    src.write_text('''
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "paged.h"
int main() {
    srand(5);
    for (int round = 0; round < 2000; ++round) {
        const int shift = 4 + rand() % 5, heads = 1 + rand() % 8, width = rand() % 9, seqs = 1 + rand() % 4, pages = 1 + rand() % 7;
        const bool token = rand() & 1;
        std::vector<int32_t> table(seqs * width + 1);
        const int32_t odd[] = {-1, INT32_MIN, INT32_MAX, pages, pages + 1};
        for (auto &e : table) e = rand() % 3 ? rand() % pages : odd[rand() % 5];
        lvr_paged_batch b = {};
        b.table = table.data();
        b.table_width = width; b.n_seqs = seqs; b.page_shift = shift; b.n_pages = pages;
        b.page_stride = (int64_t)heads * (256 << shift);
        b.head_stride = token ? 256 : 256 << shift;
        b.row_stride = token ? 256 * heads : 256;
        const int64_t size = pages * b.page_stride, end = (int64_t)width << shift;
        const int64_t at[] = {-1, INT64_MIN / 2, end, end + 1, INT32_MAX, (int64_t)1 << 40, 0, end - 1, end / 2, end ? rand() % end : 0};
        for (int s = 0; s < seqs; ++s)
            for (int64_t p : at) {
                const int32_t page = lvr_page_of(b, s, p);
                const int32_t entry = p >= 0 && p < end ? table[s * width + (p >> shift)] : -1;
                if (page != (entry >= 0 && entry < pages ? entry : -1)) return 1;
                if (page < 0) continue;
                for (int h = 0; h < heads; ++h) {
                    const int64_t row = lvr_row_at(b, page, h, p);
                    if (row < 0 || row + 256 > size) return 2;
                    if (row != page * b.page_stride + h * b.head_stride + (p % (1 << shift)) * b.row_stride) return 3;
                }
            }
    }
    return 0;
}
''')
    exe = tmp_path / "rows"
    from paper_2605_06763_amd.build import CSRC
    r = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "--offload-arch=gfx950", "-O1", "-std=c++17", "-I", CSRC, str(src), "-o", str(exe)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert subprocess.run([str(exe)]).returncode == 0


def test_the_stride_of_a_single_head_or_page_says_nothing(L, monkeypatch):
    """A pool of one KV head (or one page) is the same memory whatever stride its only head has: torch's contiguous() leaves it as it is."""
    monkeypatch.setattr(L.binding, "_tensor", lambda h, t, name: t)
    h = L.PagedHandle()
    h.dtype = torch.bfloat16
    for layout, heads, pages in (("head", 1, 9), ("token", 1, 9), ("token", 1, 1), ("head", 4, 1)):
        h.cfg = L.make_paged_config(n_q_heads=4, n_kv_heads=heads, page_size=16, n_pages=pages, layout=layout)
        p = torch.zeros(pages, heads, 16, 128, dtype=torch.bfloat16)
        views = [p, p.as_strided(p.shape, (p.stride(0) if pages > 1 else 8, p.stride(1) if heads > 1 else 24, 128, 1))]
        if heads == 1:
            views += [v.transpose(1, 2).contiguous() for v in views]
        for v in views:
            assert L.binding._pool(h, v, "k_pages") == p.data_ptr()
        with pytest.raises(ValueError):
            L.binding._pool(h, p.repeat(1, 1, 2, 1)[:, :, ::2], "k_pages")


def _two_pi(bits):
    """2 pi * 2^bits: pi = 20 atan(1/7) + 8 atan(3/79), summed in integers."""
    b = bits + 64

    def atan(p, q):
        term, k, total = (p << b) // q, 1, 0
        while term:
            total += -(term // k) if k % 4 == 3 else term // k
            term, k = term * p * p // (q * q), k + 2
        return total

    return (2 * (20 * atan(1, 7) + 8 * atan(3, 79))) >> 64


def test_turns_per_position_of_any_frequency(L, tmp_path):
    """Frequencies become turns per position without the whole ones, to a unit of 2^-64, however many whole ones there are."""
    import random
    from fractions import Fraction
    rng = random.Random(3)
    freqs = [0.0, 1.0, -1.0, 0.75, 9.5, -9.5, 1e6, 1e17, 1.7976931348623157e308, -1.7976931348623157e308, 5e-324, -5e-324, 1e-300, 2.0 ** 63, 2.0 ** 64 - 2048,
             6.283185307179586, 6.283185307179587, -6.283185307179586, 10000.0 ** (-1 / 64), 2.0 ** -60, 2.0 ** -64, 2.0 ** 971, 2.0 ** 970 * 1.5]
    freqs += [rng.choice([1, -1]) * rng.uniform(1, 2) * 2.0 ** rng.uniform(-70, 70) for _ in range(3000)]
    freqs += [rng.choice([1, -1]) * rng.uniform(1, 2) * 2.0 ** rng.uniform(-1070, 1022) for _ in range(3000)]
    src, exe = tmp_path / "turns.hip", tmp_path / "turns"
    src.write_text('#include <cstdio>\n#include "paged.h"\nint main() {\n    double f;\n    while (scanf("%la", &f) == 1) printf("%llu\\n", (unsigned long long)lvr_turns_of(f));\n}\n')
    from paper_2605_06763_amd.build import CSRC
    r = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "--offload-arch=gfx950", "-O1", "-std=c++17", "-I", CSRC, str(src), "-o", str(exe)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    got = subprocess.run([str(exe)], input="\n".join(f.hex() for f in freqs), capture_output=True, text=True).stdout.split()
    assert len(got) == len(freqs)
    bits = 1300
    two_pi = _two_pi(bits)
    for f, g in zip(freqs, got):
        x = Fraction(f)
        want = ((x.numerator << (bits + 64)) // (x.denominator * two_pi)) % (1 << 64)
        off = (int(g) - want) % (1 << 64)
        assert min(off, (1 << 64) - off) <= 1, (f, int(g), want)
