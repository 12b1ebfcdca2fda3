"""What the compiler makes of the append's stores, from the library's own flags and source."""
import os
import re
import subprocess

import pytest


@pytest.fixture(scope="module")
def listing(tmp_path_factory):
    from paper_2605_06763_amd.build import CSRC, HIPCC_FLAGS
    out = tmp_path_factory.mktemp("code") / "paged.s"
    r = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *HIPCC_FLAGS, "--cuda-device-only", "-S", os.path.join(CSRC, "paged.hip"), "-o", str(out)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return out.read_text()


@pytest.mark.parametrize("pairs", [0, 1])
def test_stores_of_fp32_rows_do_not_wait_for_each_other(listing, pairs):
    """A wave that appends six pairs of pieces has them all before the first store: behind that it waits for no access to memory."""
    name = f"paged_append_kernelI9lvr_f32_tLb{pairs}ELi6ELb1ELb0ELb0EE"
    body = re.search(r"^_ZN\S*" + name + r"\S*:.*?^\.Lfunc_end", listing, re.M | re.S).group(0)
    code = [line.split(";")[0].strip() for line in body.splitlines()]
    stores = [i for i, x in enumerate(code) if x.startswith("global_store")]
    assert len(stores) == 12
    assert not [x for x in code[stores[0]:] if x.startswith("s_waitcnt") and "vmcnt" in x]


@pytest.mark.parametrize("kernel, n", [("paged_gather_kernelI", 4), ("paged_gather_fp4_kernelI", 2)])
def test_gathers_read_two_lines_of_arguments(listing, kernel, n):
    """Nothing of what the runtime puts behind a kernel's own arguments, which are two lines of 64 bytes."""
    sizes = re.findall(r"\.amdhsa_kernel \S*" + kernel + r".*?\.amdhsa_kernarg_size (\d+)", listing, re.S)
    assert [int(x) for x in sizes] == [128] * n
