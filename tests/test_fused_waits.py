"""Waits of the large-tile kernels with an epilogue and of e4m3, followed as in test_grouped_waits.py:
no wave passes a bare barrier with an LDS access of its own under way."""
import re
import subprocess

import pytest
from test_grouped_waits import under_way_at_barriers

from paper_2509_17863_amd import _build

# (source, kernel, how many of it): gathered or not, and the way back; gathered or not, with
# rows of scales in multiples of 16 bytes or not
KERNELS = [("grouped_swiglu.hip", "grouped_pp_kernel", 3), ("grouped_fp8.hip", "grouped_fp8_kernel", 4),
           ("grouped_fp8.hip", "grouped_fp8_mid_kernel", 1)]


def kernels(source, out):
    subprocess.run([_build.hipcc(), *_build.FLAGS, "-I", str(_build.PKG.parent / "include"),
                    "--cuda-device-only", "-S", str(_build.CSRC / source), "-o", str(out)],
                   check=True, capture_output=True)
    found, name = {}, None
    for line in out.read_text().splitlines():
        line = line.split(";")[0].strip()
        m = re.match(r"(_Z\w+):$", line)
        if m:
            name = m.group(1)
            found[name] = []
        elif line.startswith(".Lfunc_end"):
            name = None
        elif name and line and (not line.startswith(".") or line.endswith(":")):
            found[name].append(line)
    return found


@pytest.mark.parametrize("source,kernel,count", KERNELS)
def test_no_lds_access_is_under_way_at_a_barrier(source, kernel, count, tmp_path):
    large = {n: k for n, k in kernels(source, tmp_path / "a.s").items() if kernel in n}
    assert len(large) == count
    for name, lines in large.items():
        assert lines.count("s_barrier") >= 4, name
        assert under_way_at_barriers(lines) == [], name
