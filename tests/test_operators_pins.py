"""What the layer operators' kernels rest on, checked without a GPU."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2506_08520_amd", "csrc")


def asm_statements():
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h*"))):
        with open(path) as f:
            text = re.sub(r"//[^\n]*", "", f.read())
        for m in re.finditer(r"\basm\b[^;(]*\(", text):
            depth, i, quoted = 1, m.end(), False
            while depth:
                ch = text[i]
                if ch == '"' and text[i - 1] != "\\":
                    quoted = not quoted
                if not quoted:
                    depth += (ch == "(") - (ch == ")")
                i += 1
            yield os.path.basename(path), text[m.end():i - 1]


def test_assembly_declares_the_registers_that_it_uses():
    """A register that a statement names stands among its operands or clobbers, and the loads
    to LDS take m0 as an operand: the compiler has uses of its own for it."""
    loads = 0
    for name, body in asm_statements():
        body = body.replace(r"\n", " ").replace(r"\t", " ")
        strings = re.findall(r'"((?:[^"\\]|\\.)*)"', body)
        for reg in re.findall(r"\b[sv]_\w+\s+(m0|vcc|exec|scc|s\d+|v\d+)\b", body):
            assert reg in strings[1:], f"{name}: {reg} is written but not declared: {body}"
        if re.search(r"\blds_dword|_load_lds_", body):
            loads += 1
            assert "{m0}" in strings, f"{name}: m0 is not an operand: {body}"
    assert loads >= 2
