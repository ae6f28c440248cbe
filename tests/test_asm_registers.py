"""Assembly in the kernels' sources names every register that it writes by name: the compiler keeps values there otherwise."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1910_10929_amd", "csrc")


def test_written_registers_are_declared():
    found = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        with open(path) as f:
            text = f.read()
        for statement in re.findall(r"\basm volatile\((.*?)\);", text, re.S):
            template, rest = (re.split(r'"\s*:', statement, maxsplit=1) + [""])[:2]
            clobbers = rest[rest.rfind(":"):] if ":" in rest else ""
            for register in set(re.findall(r"(?:^|\\n\\t|\")[a-z_0-9]+ (m0|vcc|exec|s\d+|v\d+)\b", template)):
                found += 1
                assert f'"{register}"' in clobbers, (os.path.basename(path), register, statement)
    assert found
