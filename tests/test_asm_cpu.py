"""Inline assembly in the kernels says which registers it uses: a load to LDS
reads its base from m0, so m0 is an operand of the statement that the compiler
sets, and no statement writes m0 behind the compiler's back."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_15380_amd", "csrc")
STRING = r'"(?:[^"\\]|\\.)*"'
STATEMENT = re.compile(r"asm\s+volatile\s*\(((?:[^()\"]|" + STRING + r"|\([^()]*\))*)\)")


def statements():
    """(file, instructions, operands and clobbers) of every statement."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        with open(path) as f:
            for m in STATEMENT.finditer(f.read()):
                code = re.match(r"(?:\s*" + STRING + ")+", m.group(1)).group(0)
                yield os.path.basename(path), code.replace("\\n", "\n").replace("\\t", "\t"), m.group(1)[len(code):]


def test_m0_is_an_operand():
    found = list(statements())
    loads = [(name, code, rest) for name, code, rest in found if re.search(r"_lds_|\blds\b", code)]
    assert loads                         # (dense.hip's are there)
    for name, code, rest in loads:
        assert '"{m0}"' in rest, (name, code)
    for name, code, rest in found:
        assert not re.search(r"\bs_\w+\s+m0\b", code), (name, code)
