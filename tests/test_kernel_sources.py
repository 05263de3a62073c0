"""What the kernels' sources may not hold."""
import glob
import os
import re

from conftest import ROOT

CSRC = os.path.join(ROOT, "paper_2607_13500_amd", "csrc")


def statements(text):
    """The templates of the inline assembly of a source, joined where they are split."""
    for m in re.finditer(r"\basm\s*(?:volatile)?\s*\(((?:\s*\"(?:[^\"\\]|\\.)*\")+)", text):
        yield "".join(re.findall(r"\"((?:[^\"\\]|\\.)*)\"", m.group(1)))


def test_inline_assembly_reads_no_results():
    """Vector arithmetic in inline assembly: the compiler counts the waits between a
    matrix instruction (or an exponential) and the reader of its result for its own
    instructions, not for those of inline assembly, which then read what the
    registers held before."""
    found, seen = [], 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        with open(path) as f:
            for template in statements(f.read()):
                seen += 1
                ops = [line.split()[0] for line in re.split(r"\\n(?:\\t)?|;", template) if line.split()]
                found += [(os.path.basename(path), op) for op in ops if op.startswith("v_")]
    assert seen > 5 and not found, found
