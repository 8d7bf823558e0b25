"""Waits of the large-tile kernels, read from the assembly that the compiler makes
of them.

Their barriers are bare (the loads into LDS stay in flight across them), so a wave
has to wait for its own LDS reads and writes before it passes one: what it still
has under way there could meet the loads that another wave starts into the same
stage behind the barrier.  Followed over every path of the kernel: an LDS access is
under way from its instruction to the next wait for lgkmcnt(0).
"""
import re
import subprocess

import pytest

from paper_2509_17863_amd import _build


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """Lines of every kernel of grouped_fast.hip by its symbol."""
    out = tmp_path_factory.mktemp("asm") / "grouped_fast.s"
    subprocess.run([_build.hipcc(), *_build.FLAGS, "-I", str(_build.PKG.parent / "include"),
                    "--cuda-device-only", "-S", str(_build.CSRC / "grouped_fast.hip"), "-o",
                    str(out)], check=True, capture_output=True)
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


def under_way_at_barriers(lines):
    """Numbers of the barriers that some path reaches with an LDS access under way."""
    at = {line[:-1]: i for i, line in enumerate(lines) if line.endswith(":")}
    seen, todo, bad = set(), [(0, False)], set()
    while todo:
        i, pending = todo.pop()
        while i < len(lines) and (i, pending) not in seen:
            seen.add((i, pending))
            op, _, args = lines[i].partition(" ")
            if op.startswith("ds_"):
                pending = True
            elif op == "s_waitcnt" and "lgkmcnt(0)" in args:
                pending = False
            elif op == "s_barrier" and pending:
                bad.add(i)
            elif op.startswith("s_cbranch"):
                todo.append((at[args.strip()], pending))
            elif op == "s_branch":
                i = at[args.strip()]
                continue
            elif op == "s_endpgm":
                break
            assert op not in ("s_setpc_b64", "s_swappc_b64"), "a jump that is not followed"
            i += 1
    return sorted(bad)


def test_the_walk_finds_what_it_looks_for():
    loop = ["top:", "s_barrier", "s_cbranch_execz skip", "ds_read_b128 v[0:3], v4",
            "s_waitcnt vmcnt(0) lgkmcnt(0)", "skip:", "s_branch top"]
    assert under_way_at_barriers(loop) == []
    assert under_way_at_barriers([*loop[:4], "s_waitcnt vmcnt(0)", *loop[5:]]) == [1]
    assert under_way_at_barriers(["ds_write_b64 v0, v[2:3]", "s_cbranch_scc1 out",
                                  "s_waitcnt lgkmcnt(0)", "out:", "s_barrier", "s_endpgm"]) == [4]


def test_no_lds_access_is_under_way_at_a_barrier(kernels):
    large = {n: k for n, k in kernels.items() if "grouped_pp_kernel" in n}
    assert len(large) == 7  # forward, 8-bit and dW with and without gather; dx
    for name, lines in large.items():
        assert lines.count("s_barrier") >= 4, name
        assert under_way_at_barriers(lines) == [], name
