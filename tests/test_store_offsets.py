"""Wide stores and what follows them.  No GPU needed."""
import glob
import os
import re
import subprocess

import pytest

from paper_2606_27748_amd import build as B

WIDE = re.compile(r"buffer_store_dwordx[34] v\[(\d+):(\d+)\], \S+, s\[\S+\], s\d+")


def _scalar_offsets(path):
    """Stores of 16 bytes whose scalar offset is not the literal zero."""
    text = open(path).read()
    calls = [text[at.start():text.index(";", at.start())] for at in re.finditer(r"raw_buffer_store_b(96|128)\(", text)]
    return [c for c in calls if not re.search(r",\s*0,\s*0\)$", c)]


def test_wide_stores_have_no_scalar_offset():
    """With one, the first word of a store has been seen overwritten by the instruction behind it."""
    found = {os.path.basename(p) for p in glob.glob(os.path.join(B.CSRC, "*.h*")) if _scalar_offsets(p)}
    assert found <= {"flex_decode.hip"}, found


@pytest.mark.parametrize("source", ["flex_decode.hip"])
def test_stored_registers_are_left_alone(source, tmp_path):
    """Where a wide store does have a scalar offset, none of the three instructions behind it writes what it stores."""
    out = tmp_path / "kernels.s"
    subprocess.run([B.HIPCC] + B.FLAGS + B.FILE_FLAGS.get(source, []) + ["--cuda-device-only", "-S", os.path.join(B.CSRC, source),
                   "-o", str(out)], check=True, capture_output=True)
    code = [l.strip() for l in out.read_text().splitlines() if re.match(r"\t[a-z]", l)]
    stores = 0
    for i, line in enumerate(code):
        m = WIDE.match(line)
        if not m:
            continue
        stores += 1
        for after in code[i + 1:i + 4]:
            w = re.match(r"v_\w+ v\[?(\d+)(?::(\d+))?", after)
            assert not (w and int(w[1]) <= int(m[2]) and int(w[2] or w[1]) >= int(m[1])), (line, after)
    assert stores > 0
