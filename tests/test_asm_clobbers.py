"""Instructions that are written out in the kernels' sources: a register that one of them sets by name is declared, so that the
compiler does not keep a value of its own there."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_registers_set_by_name_are_declared():
    statements = []
    for path in glob.glob(os.path.join(ROOT, "paper_2508_15706_amd", "csrc", "*")):
        statements += re.findall(r"\basm volatile\((.*?)\);", open(path).read(), re.S)
    assert statements
    for text in statements:
        for register in re.findall(r"[sv]_mov_b32 ([a-z]+\d*)\b", text):
            assert f'"{register}"' in text, text
