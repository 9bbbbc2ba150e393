"""Rules that the compiler cannot check in the kernels' sources."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1606_05688_amd", "csrc")


def _assembly():
    """(file, statement) of every asm statement."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        if path.endswith((".h", ".hip")):
            with open(path) as f:
                text = f.read()
            for m in re.finditer(r"\basm\s+volatile\s*\(", text):
                yield os.path.basename(path), text[m.start():text.index(";\n", m.start())]


def test_assembly_names_the_special_registers_that_it_writes():
    """m0 is no operand: what a statement does to it, the compiler knows from the statement's list alone."""
    writes = [(f, a) for f, a in _assembly() if re.search(r"s_mov_b32\s+m0\b", a)]
    assert writes
    for f, a in writes:
        lists = re.sub(r'^.*?"\s*::', "::", a, flags=re.S)
        assert '"m0"' in lists, (f, a)
