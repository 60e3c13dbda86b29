"""Inline assembly in the kernels' sources names the fixed registers that it changes."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2412_04358_amd", "csrc")


def statements(text):
    """(code, what is named behind the operands) of each asm statement."""
    for m in re.finditer(r"\basm\s+(?:volatile\s*)?\(", text):
        depth, end, quoted = 1, m.end(), False
        while depth:
            c = text[end]
            if c == "\\" and quoted:
                end += 1
            elif c == '"':
                quoted = not quoted
            elif not quoted:
                depth += (c == "(") - (c == ")")
            end += 1
        body = text[m.end():end - 1]
        strings = re.findall(r'"((?:[^"\\]|\\.)*)"', body)
        code = strings[0] if strings else ""
        parts = re.sub(r'"(?:[^"\\]|\\.)*"', lambda s: s.group(0).replace(":", ";"), body).replace("::", ": :").split(":")
        yield code, parts[3] if len(parts) > 3 else ""


def written(code):
    """Fixed scalar registers that its instructions have as their destinations."""
    found = set()
    for line in re.split(r"\\n\\t|\\n|;", code):
        m = re.match(r"\s*s_\w+\s+(m0|vcc|exec|scc|s\d+)\b", line)
        if m:
            found.add(m.group(1))
    return found


def test_a_register_that_is_not_named_is_found():
    code, named = next(statements('asm volatile("s_mov_b32 m0, %0\\n\\ts_nop 0" ::"s"(x) : "memory");'))
    assert written(code) == {"m0"} and "m0" not in named


def test_sources():
    count = 0
    for path in glob.glob(os.path.join(CSRC, "*")):
        with open(path) as f:
            for code, named in statements(f.read()):
                count += 1
                for register in written(code):
                    assert '"%s"' % register in named, (os.path.basename(path), code)
    assert count > 2
