"""The forward of a few tokens streams weights into LDS some steps ahead and waits, by
the number of vector loads that may still be out, for the oldest step's to land. The
wait holds only if every later step has issued at least as many vector loads as it
counts, which is the compiler's doing: loads that are the same for many lanes (scales)
may become scalar ones. Checked here in the assembly of the kernels (CPU-only)."""
import os
import re
import subprocess

import pytest

from paper_2601_01310_amd import build

GUARD = re.compile(r"s_waitcnt vmcnt\((\d+)\)$")  # with the empty asm behind it: the wait in stream()
WIDE = re.compile(r"(buffer_load_dwordx4|global_load_dwordx4|global_load_lds_dwordx4)\b")


def streams(asm):
    """[(function, the wait's count, wide loads before the first of its waits and between
    one and the next)] of each unrolled loop of steps."""
    found, name, wide = [], None, 0
    lines = [x.strip() for x in asm.split("\n")]
    for line, after in zip(lines, lines[1:]):
        if line.startswith("_ZN") and line.split()[0].endswith(":"):
            name, wide = line.split(":")[0], 0
        guard = GUARD.match(line)
        if WIDE.match(line):
            wide += 1
        elif guard and after.startswith(";;#ASMSTART"):
            n = int(guard.group(1))
            if found and found[-1][:2] == (name, n) and wide < found[-1][2][0]:
                found[-1][2].append(wide)
            else:
                found.append((name, n, [wide]))
            wide = 0
    return found


def short(found):
    """Those whose wait counts more than the later steps' wide loads: `ring` steps are
    issued ahead of a loop of as many."""
    return [(name, n, loads) for name, n, loads in found
            if len(set(loads[1:])) != 1 or n > (len(loads) - 1) * loads[1]]


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("asm") / "ew_few.s")
    subprocess.run([build.HIPCC, *build.COMMON, *build.DEVICE, "-x", "hip", "--cuda-device-only", "-S",
                    os.path.join(build.CSRC, "ew_few.hip"), "-o", out], check=True, capture_output=True)
    with open(out) as f:
        return f.read()


def test_waits_count_only_loads_that_stay_vector_loads(asm):
    found = streams(asm)
    # Rings of 7 and of 3 steps; bf16 and 8 bits; fused, or of three shapes.
    assert sorted(len(loads) for _, _, loads in found) == [3] * 2 + [3] * 8 + [7] * 6
    assert not short(found)


def test_the_check_sees_a_wait_that_counts_too_much(asm):
    name, n, loads = next(x for x in streams(asm) if len(x[2]) == 7)
    assert short([(name, n + 1, loads)])
    assert short([(name, n, loads[:-1] + [loads[-1] - 1])])
