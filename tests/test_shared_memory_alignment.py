"""Arrays in LDS that are read or written 16 bytes at a time have that alignment by their declaration, not by where the compiler happens to put them."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2510_24211_amd", "csrc")


def test_arrays_for_whole_eights_are_aligned():
    found = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*.hip"))):
        text = open(path).read()
        for m in re.finditer(r"__shared__\s+([^;=]*?)(\w+)\s*\[[^;]*;", text):
            kind, name = m.groups()
            if not re.search(r"\b(?:load|store|put)_eight<[^>]*>\(\s*%s\b" % name, text):
                continue
            found += 1
            align = re.search(r"aligned\((\d+)\)", kind)
            assert re.search(r"\bf32x[48]\b", kind) or (align and int(align.group(1)) >= 16), (os.path.basename(path), kind, name)
    assert found >= 1
