"""Inline assembly that sets a register by its name has to tell the compiler: nothing else keeps it from holding a value of
its own there."""
import glob
import os
import re

import paper_2602_06502_amd._build as B


def _statements(text):
    """asm statements with literal templates: (template, what follows it)."""
    for m in re.finditer(r"\basm\s*(?:volatile)?\s*\(", text):
        depth, i = 1, m.end()
        while depth:
            depth += {"(": 1, ")": -1}.get(text[i], 0)
            i += 1
        body = text[m.end():i - 1]
        t = re.match(r'\s*((?:"(?:[^"\\]|\\.)*"\s*)+)', body)
        yield "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', t.group(1))), body[t.end():]


def test_special_registers_that_are_written_are_named():
    found = 0
    for f in sorted(glob.glob(os.path.join(B.CSRC, "*.hip")) + glob.glob(os.path.join(B.CSRC, "*.h"))):
        text = re.sub(r"//[^\n]*", "", open(f).read())
        text = "\n".join(l for l in text.splitlines() if not l.rstrip().endswith("\\"))  # (macros have tests of their own)
        for template, rest in _statements(text):
            for ins in re.split(r"\\n\\t|\\n|;", template):
                m = re.match(r"\s*s_\w+\s+(m0|vcc|exec|scc)\b", ins)
                if m:
                    found += 1
                    assert '"%s"' % m.group(1) in rest.rsplit(":", 1)[-1], (os.path.basename(f), template)
    assert found >= 2
