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


def test_assembly_declares_the_registers_that_it_writes():
    """A register that a statement names stands among its operands or clobbers: the compiler
    has uses of its own for m0."""
    for name, body in asm_statements():
        body = body.replace(r"\n", " ").replace(r"\t", " ")
        strings = re.findall(r'"((?:[^"\\]|\\.)*)"', body)
        for reg in re.findall(r"\b[sv]_\w+\s+(m0|vcc|exec|scc|s\d+|v\d+)\b", body):
            assert {reg, "=&{%s}" % reg} & set(strings[1:]), f"{name}: {reg}: {body}"


def test_loads_to_lds_read_scalars_of_their_own():
    """The base and m0 of a load in assembly are written in the statement, by scalar
    instructions, with one between m0's and the load: wait states that the compiler does not
    count there."""
    loads = 0
    for name, body in asm_statements():
        code = re.search(r'"((?:[^"\\]|\\.)*)"', body)[1].replace(r"\t", "").split(r"\n")
        if "_load_lds_" not in body:
            continue
        loads += 1
        base = re.fullmatch(r"global_load_lds_\w+ %\d, (%\d)", code[-1])[1]
        scalars = [re.match(r"s_mov_b(?:32|64) (m0|%\d), %\d$", c)[1] for c in code[:-1]]
        assert scalars == ["m0", base], f"{name}: {body}"
    assert loads == 2
