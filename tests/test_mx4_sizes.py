"""Products of 4-bit matrices without a GPU: the rule that chooses their kernels, and the room that they ask for."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    """Runs the host program on the given numbers; -> what it prints."""
    exe = str(tmp_path_factory.mktemp("mx4") / "mx4_rules")
    # (signed overflow ends the program instead of wrapping)
    cmd = ["g++", "-std=c++17", "-O2", "-fsanitize=signed-integer-overflow", "-fsanitize-undefined-trap-on-error",
           "-I", os.path.join(ROOT, "paper_2508_15706_amd", "csrc"), os.path.join(HERE, "host", "mx4_rules.cpp"), "-o", exe]
    subprocess.run(cmd, check=True)

    def call(*numbers):
        r = subprocess.run([exe, *map(str, numbers)], capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stdout + r.stderr
        return r.stdout
    return call


def test_room(rules):
    assert rules().strip() == "ok"


def test_every_kernel_has_its_tests(rules):
    """The GPU tests' sizes reach the kernels that they are there for."""
    import test_gpu_mx4_sizes as gpu
    for tile, sizes in gpu.TILES.items():
        lines = rules(*(z for s in sizes for z in s)).splitlines()
        assert len(lines) == len(sizes) and all(line.startswith(f"{tile} 1 ") for line in lines)
    for waves, widths in gpu.FEW.items():
        lines = rules(*(z for n in widths for m, k in gpu.FEW_ROWS for z in (m, n, k))).splitlines()
        assert len(lines) == len(widths) * len(gpu.FEW_ROWS) and all(line.endswith(f" 1 {waves}") for line in lines)


@pytest.mark.parametrize("m, n, k", [(2000, 512, 8192), (512, 2048, 8192), (512, 1024, 8192), (70, 700, 16384), (16, 2048, 8192)])
def test_room_for_the_most_rows_serves_fewer(m, n, k):
    from paper_2508_15706_amd import binding as sl
    most = sl.sl_mx4_workspace_bytes(m, n, k)
    assert all(sl.sl_mx4_workspace_bytes(rows, n, k) <= most for rows in range(1, m))
    assert all(sl.sl_mx4_workspace_bytes(m, cols, k) <= most for cols in range(1, n, 7))
    assert all(sl.sl_mx4_workspace_bytes(m, n, length) <= most for length in range(1, k, 31))
