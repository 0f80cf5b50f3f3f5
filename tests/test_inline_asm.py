"""Inline assembly of the kernels says what it writes (CPU: the sources are read)."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_22312_amd", "csrc")


def statements():
    """Every asm statement of the sources: file, template and what follows it, up to the closing parenthesis."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*.hip")) + glob.glob(os.path.join(CSRC, "*.h"))):
        with open(path) as f:
            text = f.read()
        for m in re.finditer(r"\basm\s+(?:volatile\s*)?\(", text):
            depth, at = 1, m.end()
            while depth:
                depth += {"(": 1, ")": -1}.get(text[at], 0)
                at += 1
            body = text[m.end():at - 1]
            template = re.match(r'\s*((?:"(?:[^"\\]|\\.)*"\s*)+)', body)
            yield os.path.basename(path), template.group(1), body[template.end():]


def test_writes_of_m0_are_named():
    """A statement that writes m0 names it as clobbered: the compiler may hold a number of its own there."""
    found = 0
    for name, template, rest in statements():
        if re.search(r"\bs_mov_b32\s+m0\b", template):
            assert '"m0"' in rest.rsplit(":", 1)[-1], (name, template)
            found += 1
    assert found >= 2
