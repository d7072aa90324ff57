"""CPU check of how attention over the 8-bit cache is cut into shares and merged: a small C++ program compiled against the kernels' own arithmetic."""
import os
import shutil
import subprocess

import pytest

from tests.test_gpu_kvq_kernels import CASES as KERNEL_CASES, IDS as KERNEL_IDS
from tests.test_gpu_kvq_merge import CASES, IDS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not (os.path.exists(hipcc) or shutil.which(hipcc)):
        pytest.skip("hipcc not available")
    exe = str(tmp_path_factory.mktemp("host") / "kvq_shares_check")
    r = subprocess.run([hipcc, "--offload-arch=gfx950", "-O1", "-std=c++17", "-Wno-unused-result", os.path.join(ROOT, "tests", "host", "kvq_shares_check.cpp"), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]

    def run(*args):
        r = subprocess.run([exe, *map(str, args)], capture_output=True, text=True)
        assert r.returncode == 0, r.stdout + r.stderr
        return r.stdout
    return run


def test_parts_follow_each_other_and_merges_read_what_was_published(program):
    assert program().startswith("ok ")


def _lone_levels(n, f):
    """Levels on which the last of n parts has no neighbour."""
    return {level for level in range(5) if f ** level < n and -(-n // f ** level) % f == 1}


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_the_cases_of_the_gpu_test_reach_their_merges(program, case):
    Hq, Hkv, D, ctx, counts, wanted = case
    pages = -(-max(c + n for c, n in zip(ctx, counts)) // 64)
    out = program(int(len(ctx) > 3), Hkv, Hq // Hkv, max(counts), pages, *[v for pair in zip(ctx, counts) for v in pair]).split()
    threads, reached = 512 if len(ctx) > 3 else 256, set()
    for unit in out:
        parts, rows = map(int, unit.split(":"))
        few = rows * (D // 4) <= threads
        reached |= {(few, level) for level in _lone_levels(parts, 8 if few else 4)}
    assert wanted <= reached, (wanted, reached, out)


@pytest.mark.parametrize("case", KERNEL_CASES, ids=KERNEL_IDS)
def test_the_cases_of_both_kernels_run_them(program, case):
    Hq, Hkv, D, ctx, counts, besides = case
    longest = max(c + n for c, n in zip(ctx, counts))
    for wide, most in ((1, max(longest, besides)), (0, longest)):
        program(wide, Hkv, Hq // Hkv, max(counts), -(-most // 64), *[v for pair in zip(ctx, counts) for v in pair])
