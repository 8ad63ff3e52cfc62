"""Inline assembly tells the compiler which registers it writes besides its outputs: m0 here, which the compiler is free to use for instructions of its own."""
import glob
import os
import re

SOURCES = glob.glob(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2507_17133_amd", "csrc", "*.h*"))


def _statements(text):
    text = re.sub(r"//[^\n]*", "", text)
    return re.findall(r"\basm\s*(?:volatile)?\s*\(.*?\)\s*;", text, re.S)


def test_m0_is_named_where_it_is_written():
    found = 0
    for path in SOURCES:
        for s in _statements(open(path).read()):
            template = re.match(r"\basm\s*(?:volatile)?\s*\(\s*((?:\"(?:[^\"\\]|\\.)*\"\s*)+)", s).group(1)
            if not re.search(r"\bm0\b", template):
                continue
            found += 1
            clobbers = s[s.index(template) + len(template):].split(":")[3:]        # : outputs : inputs : clobbers
            assert any('"m0"' in c for c in clobbers), (os.path.basename(path), s)
    assert found == 2
