"""Inline assembly of the HIP sources names the registers that it writes beside its operands, so that the compiler does not count on what
it had there."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_24786_amd", "csrc")
WRITTEN = re.compile(r"^\s*[sv]_\w+\s+(m0|vcc|exec|scc|s\d+|v\d+|s\[\d+:\d+\]|v\[\d+:\d+\])\b")


def _statements(text):
    """(template, rest of the statement) of every asm statement."""
    for m in re.finditer(r"\basm\s+volatile\s*\(|\basm\s*\(", text):
        depth, i, quoted = 1, m.end(), False
        while depth:
            ch = text[i]
            if ch == '"' and text[i - 1] != "\\":
                quoted = not quoted
            elif not quoted:
                depth += {"(": 1, ")": -1}.get(ch, 0)
            i += 1
        body = text[m.end():i - 1]
        head = re.match(r'(?:\s*"(?:[^"\\]|\\.)*")+', body)
        yield head.group(0), body[head.end():]


def test_registers_written_by_name_are_named_as_clobbered():
    found = 0
    for name in sorted(os.listdir(CSRC)):
        with open(os.path.join(CSRC, name)) as f:
            text = f.read()
        for template, rest in _statements(text):
            lines = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', template)).replace("\\t", "").split("\\n")
            clobbers = rest.split(":")[3] if rest.count(":") >= 3 else ""
            for line in lines:
                written = WRITTEN.match(line)
                if written:
                    found += 1
                    assert f'"{written.group(1)}"' in clobbers, f"{name}: {line.strip()!r} writes {written.group(1)}, which the statement does not name"
    assert found >= 2
