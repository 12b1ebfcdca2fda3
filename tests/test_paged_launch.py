"""What a launch of the attention over pages makes of a call before the batch is divided on the device."""
import os
import subprocess

import pytest


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


def test_what_a_launch_makes_of_a_call(division):
    """Windows that hide nothing, first keys without a window, and the keys up to which a tile is not cut, by the type: as paged_launch sets them."""
    exe = division("launch", r'''
#include <cstdio>
#include "paged_division.h"
int main() {
    int type, window, sinks;
    while (scanf("%d %d %d", &type, &window, &sinks) == 3) {
        lvr_paged_batch b = {};
        b.n_seqs = 1, b.n_tokens = 1, b.table_width = 4, b.page_shift = 6;
        AttnArgs a = {};
        a.window = window, a.sinks = sinks, a.uncut = -7;
        paged_launch(a, b, 32, 8, type != 0, type == 2);
        printf("%d %d %d\n", a.window, a.sinks, a.uncut);
    }
    return 0;
}
''')
    top = 2 ** 31 - 1
    want = {
        (0, 0, 0): (0, 0, 0), (1, 0, 0): (0, 0, 0), (2, 0, 0): (0, 0, 512),
        (0, 100, 4): (100, 4, 0), (1, 100, 4): (100, 4, 256), (2, 100, 4): (100, 4, 512), (1, 100, 0): (100, 0, 0),
        (1, 0, 4): (0, 0, 0), (1, top, 0): (0, 0, 0), (1, 1, top): (0, 0, 0), (1, top, top): (0, 0, 0),
        (1, 2 ** 30 - 4, 4): (0, 0, 0), (1, 2 ** 30 - 5, 4): (2 ** 30 - 5, 4, 256), (0, 2 ** 30 - 1, 0): (2 ** 30 - 1, 0, 0), (0, 2 ** 30, 0): (0, 0, 0),
    }
    r = subprocess.run([str(exe)], input="\n".join("%d %d %d" % k for k in want), capture_output=True, text=True, timeout=60)
    assert r.returncode == 0
    assert [tuple(map(int, line.split())) for line in r.stdout.splitlines()] == list(want.values())
