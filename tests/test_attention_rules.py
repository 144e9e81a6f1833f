"""Where attention's calls place what they keep in a workspace, checked on the CPU over the sizes that they take."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


def test_workspaces(tmp_path):
    exe = str(tmp_path / "attention_rules")
    # (signed overflow ends the program instead of wrapping)
    cmd = ["g++", "-std=c++17", "-O2", "-fsanitize=signed-integer-overflow", "-fsanitize-undefined-trap-on-error",
           "-I", os.path.join(ROOT, "paper_2508_15706_amd", "csrc"), os.path.join(HERE, "host", "attention_rules.cpp"), "-o", exe]
    subprocess.run(cmd, check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert (r.returncode, r.stdout.strip()) == (0, "ok"), r.stdout + r.stderr
