"""What the sources of the packed-sequence kernels promise the compiler.  No GPU needed."""
import glob
import os
import re

from paper_2606_27748_amd import build as B


def _assembly():
    for path in glob.glob(os.path.join(B.CSRC, "*.h*")):
        text = open(path).read()
        for at in re.finditer(r"\basm\s+volatile\s*\(", text):
            yield os.path.basename(path), text[at.start():text.index(";", at.end())]


def test_assembly_writes_no_register_behind_the_compilers_back():
    """No assembly statement writes m0 by itself: as an operand the compiler sets it, and knows what it holds."""
    loads = 0
    for name, text in _assembly():
        assert not re.search(r"\bs_\w+\s+m0\b", text), (name, text)
        if re.search(r"\blds\b", text):
            loads += 1
            assert '"{m0}"' in text, (name, text)
    assert loads == 3   # rows and floats of a window, and linear copies
