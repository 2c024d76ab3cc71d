"""Inline assembly names the registers that it writes: what it does not name, the compiler may keep a value in."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2005_13789_amd", "csrc")


def statements():
    """(file, instructions, clobbers) of every asm statement: its text up to the closing parenthesis, cut at the colons outside of quotes."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*.hip")) + glob.glob(os.path.join(CSRC, "*.h"))):
        text = open(path, encoding="utf-8").read()
        for m in re.finditer(r"\basm\s+volatile\s*\(", text):
            parts, depth, quoted, i = [""], 1, False, m.end()
            while depth:
                c = text[i]
                if c == '"':
                    quoted = not quoted
                if not quoted:
                    depth += (c == "(") - (c == ")")
                if c == ":" and not quoted and depth == 1:
                    parts.append("")
                else:
                    parts[-1] += c
                i += 1
            yield os.path.basename(path), parts[0], parts[3] if len(parts) > 3 else ""


def test_assembly_that_writes_m0_names_it():
    found = list(statements())
    assert len(found) >= 5
    writers = [s for s in found if re.search(r"\b[sv]_\w+\s+m0\s*,", s[1])]
    assert writers, "the loads to LDS write m0"
    for name, code, clobbers in writers:
        assert '"m0"' in clobbers, (name, code)
