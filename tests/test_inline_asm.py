"""Inline assembly that writes m0 gives it back: the compiler may hold a value there
and cannot be told of the change (m0 is a reserved register in a clobber list)."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_10264_amd", "csrc")


def _statements():
    for name in sorted(os.listdir(CSRC)):
        with open(os.path.join(CSRC, name)) as f:
            text = f.read()
        for m in re.finditer(r"\basm\s+volatile\s*\(", text):
            # the template: the string literals up to the first colon outside them
            lits, at = [], m.end()
            while (lit := re.compile(r'\s*"((?:[^"\\]|\\.)*)"').match(text, at)) is not None:
                lits.append(lit.group(1))
                at = lit.end()
            yield name, [x.strip() for x in re.split(r"\\n|\\t", "".join(lits)) if x.strip()]


def test_m0_is_given_back():
    found = 0
    for name, lines in _statements():
        if not any(re.match(r"s_mov_b32 m0,", x) for x in lines):
            continue
        found += 1
        saved = re.fullmatch(r"s_mov_b32 (%\d+), m0", lines[0])
        assert saved and lines[-1] == f"s_mov_b32 m0, {saved.group(1)}", (name, lines)
    assert found >= 3
