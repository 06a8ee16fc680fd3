"""What a reader of the HIP sources can check without a GPU."""
import glob
import os
import re

from paper_2011_13635_amd import build


def _asm_statements():
    for path in sorted(glob.glob(os.path.join(build.CSRC, "*"))):
        if not path.endswith((".hip", ".h")):
            continue
        with open(path) as f:
            text = f.read()
        for m in re.finditer(r"\basm\s+(?:volatile\s*)?\((.*?)\);", text, re.S):
            yield os.path.basename(path), m.group(1)


def test_asm_that_writes_m0_says_so():
    """The compiler may set M0 once for several uses of its own: a statement that changes it has to name it among what it changes."""
    writes = [(path, s) for path, s in _asm_statements() if re.search(r"\bs_mov_b32\s+m0\b", s)]
    assert writes
    for path, s in writes:
        assert re.search(r':[^:]*"m0"[^:]*$', s), f"{path}: {s}"
