"""The kernel sources use no atomics (no GPU): what the library documents of its results."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _code(src):
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", src, flags=re.S)


def test_no_atomics():
    files = glob.glob(os.path.join(ROOT, "paper_2606_28560_amd", "csrc", "*"))
    assert len(files) >= 10
    for path in files:
        found = re.findall(r"\w*atomic\w*", _code(open(path).read()), flags=re.I)
        assert not found, (os.path.basename(path), found)
    assert re.findall(r"\w*atomic\w*", _code("if (x) atomicOr(&y, 1u);  // no atomics"), flags=re.I) == ["atomicOr"]
