"""Inline assembly of the HIP sources leaves the compiler no wrong belief about a register."""
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


def test_registers_written_by_name():
    """Ordinary ones are named as clobbered.  m0 and exec are reserved: the compiler promises nothing for one on that list, so they are operands
    that it writes itself ("{m0}"), or left alone."""
    statements = 0
    for name in sorted(os.listdir(CSRC)):
        with open(os.path.join(CSRC, name)) as f:
            text = f.read()
        for template, rest in _statements(text):
            statements += 1
            lines = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', template)).replace("\\t", "").split("\\n")
            operands = rest.split(":")
            clobbers = operands[3] if len(operands) > 3 else ""
            for line in lines:
                written = WRITTEN.match(line)
                if written:
                    register = written.group(1)
                    assert register not in ("m0", "exec"), f"{name}: {line.strip()!r} writes a reserved register"
                    assert f'"{register}"' in clobbers, f"{name}: {line.strip()!r} writes {register}, which the statement does not name"
            if any("_load_lds_" in line for line in lines):                     # takes its address in LDS from m0
                assert '"{m0}"' in operands[2], f"{name}: {lines} needs m0"
    assert statements > 3
