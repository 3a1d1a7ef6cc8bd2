"""Inline assembly in the kernels: a register that a statement writes by its name is among its clobbers, since the compiler keeps values of its own in such registers.  m0 cannot be
one (the compiler takes it as reserved): it is an operand wherever an instruction reads it, and never written by name."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2103_15195_amd", "csrc")
NAMED = re.compile(r"^\s*[sv]_\w+\s+(m0|vcc(?:_lo|_hi)?|exec(?:_lo|_hi)?|[sv]\d+|[sv]\[\d+:\d+\])\b")


def statements(text):
    """(instructions, what stands behind them) of every asm statement."""
    for m in re.finditer(r"\basm\s+volatile\s*\(", text):
        depth, at = 1, m.end()
        while depth:
            depth += {"(": 1, ")": -1}.get(text[at], 0)
            at += 1
        body = text[m.end():at - 1]
        code = re.match(r'\s*((?:"(?:[^"\\]|\\.)*"\s*)+)', body)
        lines = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', code.group(1))).replace("\\n", "\n").replace("\\t", "\t").split("\n")
        yield lines, body[code.end():]


def all_statements():
    for path in sorted(glob.glob(os.path.join(CSRC, "*.hip")) + glob.glob(os.path.join(CSRC, "*.h"))):
        for lines, rest in statements(open(path).read()):
            yield os.path.basename(path), lines, rest


def test_registers_written_by_name_are_clobbers():
    for path, lines, rest in all_statements():
        for line in lines:
            name = NAMED.match(line)
            if name:
                assert name.group(1) != "m0" and f'"{name.group(1)}"' in rest.split(":")[-1], (path, line)


def test_copies_to_lds_have_m0_as_an_operand():
    copies = [rest for _, lines, rest in all_statements() if any(re.search(r"buffer_load\w* .*\blds\b", line) for line in lines)]
    assert len(copies) == 2 and all('"{m0}"(' in rest for rest in copies)
